// mla_pages_*: the pages of paged caches, counted and given out on the device.
//
// Who gets which page is a matter of ranks, not of atomics, so that every run
// gives the same tables: the free pages (and, compacting, the used ones) are ranked
// in index order by prefix sums, the pages wanted in the order of the call's rows.
// One cluster of 8 CTAs (a CTA, where that does) plans: each of its 256 warps counts over a range of rows
// and of pages (a ballot counts 32 pages), the counts are summed over the CTA and,
// through distributed shared memory, over the cluster, and each warp then knows the
// ranks of what it has.  (1024 rows of 2 to 130 pages from cold caches: one CTA planned
// in 19 us and a second launch filled the rows in 5; the cluster does both in 13.  The
// whole GPU would need a second launch or a grid barrier.)  Copies are made by a
// second launch over all SMs; 1024 partial pages in four layers' caches, 33 MB
// written, take 13 us, and moving 415 MB of the latent cache's pages 71 us, 5.8 TB/s.  The only atomics are integer counts, whose
// order changes nothing.
#include <limits.h>

#include "common.cuh"
#include "internal.h"
#include "tc.cuh"

namespace gbmla {
namespace {

constexpr int kPlanThreads = 1024, kMaxPlanCtas = 8, kCtaWarps = kPlanThreads / 32;
constexpr int kLook = 16;  // ballots of 32 pages a warp takes at a time
constexpr int kWorkThreads = 256, kCopyCtas = 6;
constexpr int kChunk = 4 * kWorkThreads;  // vectors of a step of a compaction's copies
constexpr int kHead = 16;  // ints before the workspace's lists

// Workspace: [0] pages moved, [1] pages looked at; then a table row's copy each (source
// page, page of its own or -1, rows); then one int a page each: free list or
// destinations, sources, new places (-1: nothing counts the page)
// or which pages were free, a bit each.
struct Ws {
    int32_t *head;
    int4 *copy;
    int32_t *list, *src, *to;
    __host__ __device__ Ws(int32_t *ws, const mla_page_pool &p)
    {
        head = ws;
        copy = reinterpret_cast<int4 *>(ws + kHead);
        list = ws + kHead + 4 * static_cast<size_t>(p.num_rows);
        src = list + p.num_pages;
        to = src + p.num_pages;
    }
};

struct PlanShared {
    int2 warp[kCtaWarps];
    int2 cta[2][kMaxPlanCtas];
};

// A warp's part in the plan of a cluster (the grid is one; it may be one CTA).
struct Plan {
    PlanShared &sh;
    int lane, own, rank, warp, ctas, warps;  // warp in the CTA, CTA, warp in the cluster, CTAs, warps
    int par = 0;
    __device__ __forceinline__ explicit Plan(PlanShared &s)
        : sh(s), lane(threadIdx.x & 31), own(threadIdx.x >> 5), rank(blockIdx.x), warp(rank * kCtaWarps + own), ctas(gridDim.x), warps(ctas * kCtaWarps)
    {
        if (ctas > 1) tc::cluster_sync();  // (its peers' shared memory is there)
    }
    // What the plan's threads wrote before is seen after.
    __device__ __forceinline__ void sync() const
    {
        if (ctas > 1)
            tc::cluster_sync();
        else
            __syncthreads();
    }
    // The first page that the warp looks at, where it looks at kLook x 32.
    __device__ __forceinline__ int64_t first_look() const { return static_cast<int64_t>(warp) * kLook * 32; }
    // The warp's share of n things: [first, last).
    __device__ __forceinline__ int2 share(int n, int multiple) const
    {
        const int64_t per = ((int64_t{n} + warps - 1) / warps + multiple - 1) / multiple * multiple, first = warp * per;
        return make_int2(static_cast<int>(first < n ? first : n), static_cast<int>(first + per < n ? first + per : n));
    }
    // Exclusive prefix sums of two counts over the cluster's warps; the totals.
    // What the cluster wrote to memory before is seen after.
    __device__ __forceinline__ int2 scan(int a, int b, int2 *total)
    {
        if (lane == 0) sh.warp[own] = make_int2(a, b);
        __syncthreads();
        if (own == 0) {
            const int2 v = sh.warp[lane];
            int2 s = v;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int x = __shfl_up_sync(0xffffffffu, s.x, o), y = __shfl_up_sync(0xffffffffu, s.y, o);
                if (lane >= o) s.x += x, s.y += y;
            }
            sh.warp[lane] = make_int2(s.x - v.x, s.y - v.y);
            const int x = __shfl_sync(0xffffffffu, s.x, 31), y = __shfl_sync(0xffffffffu, s.y, 31);
            if (lane < ctas) {
                uint32_t to;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(smem_u32(&sh.cta[par][rank])), "r"(lane));
                asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(to), "r"(x), "r"(y) : "memory");
            }
        }
        sync();
        int2 before = sh.warp[own], all = make_int2(0, 0);
        for (int c = 0; c < ctas; ++c) {
            const int2 v = sh.cta[par][c];
            if (c < rank) before.x += v.x, before.y += v.y;
            all.x += v.x, all.y += v.y;
        }
        par ^= 1;
        __syncthreads();  // (sh.warp is written again)
        *total = all;
        return before;
    }
};

__device__ __forceinline__ int pages_of(int len, int page) { return (len + page - 1) / page; }

// Table row of group i % groups of the call's sequence i / groups, -1 if there is none.
__device__ __forceinline__ int row_of(const mla_page_pool &p, const int32_t *seqs, int i)
{
    const int s = seqs[i / p.groups];
    return s >= 0 && s < p.num_rows / p.groups ? s * p.groups + i % p.groups : -1;
}
__device__ __forceinline__ bool len_ok(const mla_page_pool &p, int len)
{
    return len >= 0 && len <= p.bt_stride * p.page_size;
}

// The warp's kLook x 32 pages from `page0` on: their counts (1 from page `end` on),
// and which are free, word j for the pages from page0 + 32 j on.
struct Look {
    int refs[kLook];
    unsigned free[kLook];
    __device__ __forceinline__ void load(const mla_page_pool &p, int64_t page0, int end)
    {
#pragma unroll
        for (int j = 0; j < kLook; ++j) {
            const int64_t page = page0 + 32 * j + (threadIdx.x & 31);
            refs[j] = page < end ? p.refs[page] : 1;
        }
    }
    __device__ __forceinline__ int count()
    {
        int n = 0;
#pragma unroll
        for (int j = 0; j < kLook; ++j) {
            free[j] = __ballot_sync(0xffffffffu, refs[j] == 0);
            n += __popc(free[j]);
        }
        return n;
    }
};

// Ranks the warp's `mine` wanted pages among the cluster's and puts the lowest free
// pages into list, as many as are wanted; the first rank, *found pages are there.
// `look` has loaded the warp's first pages.  Where `bits` is given, which pages were
// free is left there, a word for every 32 pages up to *looked.
__device__ __forceinline__ int rank_pages(const mla_page_pool &p, Plan &plan, Look &look, int mine, int32_t *list, int *found,
                                          int32_t *bits = nullptr, int32_t *looked = nullptr)
{
    const int64_t round = int64_t{plan.warps} * kLook * 32;
    int at = 0, want = 0, have = 0;
    for (int64_t p0 = 0; p0 == 0 || (have < want && p0 < p.num_pages); p0 += round) {
        const int64_t page0 = p0 + plan.first_look();
        if (p0 > 0) look.load(p, page0, p.num_pages);
        const int n = look.count();
        int2 total;
        const int2 before = plan.scan(p0 == 0 ? mine : 0, n, &total);
        if (p0 == 0) at = before.x, want = total.x;
        int r = have + before.y;
#pragma unroll
        for (int j = 0; j < kLook; ++j) {
            const int to = r + __popc(look.free[j] & ((1u << plan.lane) - 1u));
            if ((look.free[j] >> plan.lane & 1) && to < want) list[to] = static_cast<int>(page0) + 32 * j + plan.lane;
            r += __popc(look.free[j]);
            if (bits && plan.lane == j && page0 + 32 * j < p.num_pages) bits[page0 / 32 + j] = static_cast<int32_t>(look.free[j]);
        }
        have += total.y;
        if (bits && plan.warp == 0 && plan.lane == 0) *looked = static_cast<int>(min(p0 + round, int64_t{p.num_pages}));
    }
    plan.sync();  // the list is written
    *found = min(have, want);
    return at;
}

// The pages that n sequences' rows still want: a warp a few rows.
__global__ void __launch_bounds__(kPlanThreads) reserve_kernel(mla_page_pool p, int n, const int32_t *seqs,
                                                              const int32_t *lens, int32_t *ws, unsigned *status)
{
    __shared__ PlanShared sh;
    griddep_wait();
    const Ws w(ws, p);
    Plan plan(sh);
    Look look;
    look.load(p, plan.first_look(), p.num_pages);
    const int2 rows = plan.share(n * p.groups, 1);
    // lane r: the i0 + r-th row's entries (an offset into the table) and how many it needs (0: no such row)
    auto row_at = [&](int i0, int *need, bool report) {
        const int i = i0 + plan.lane;
        *need = 0;
        if (i >= rows.y) return 0;
        const int row = row_of(p, seqs, i), len = lens[i / p.groups];
        if (row < 0 || !len_ok(p, len)) {
            if (report) record_status(status, kStatusBounds);
            return 0;
        }
        *need = pages_of(len, p.page_size);
        return row * p.bt_stride;
    };
    // entries lane, lane + 32 of four rows from k0 on, loaded together (0: past what is needed)
    auto entries = [&](int entry, int need, int r0, int k0, int (&e)[4][2]) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int32_t *row = p.block_table + __shfl_sync(0xffffffffu, entry, r0 + r);
            const int end = __shfl_sync(0xffffffffu, need, r0 + r);
#pragma unroll
            for (int j = 0; j < 2; ++j) e[r][j] = k0 + 32 * j + plan.lane < end ? row[k0 + 32 * j + plan.lane] : 0;
        }
    };
    int mine = 0, e[4][2];
    for (int i0 = rows.x; i0 < rows.y; i0 += 32) {
        int need, count = 0;
        const int entry = row_at(i0, &need, true);
        for (int r0 = 0; r0 < min(32, rows.y - i0); r0 += 4) {
            int miss[4] = {0, 0, 0, 0};
            const int most = __reduce_max_sync(0xffffffffu, plan.lane >> 2 == r0 >> 2 ? need : 0);
            for (int k0 = 0; k0 < most; k0 += 64) {
                entries(entry, need, r0, k0, e);
#pragma unroll
                for (int r = 0; r < 4; ++r) miss[r] += (e[r][0] == -1) + (e[r][1] == -1);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int all = __reduce_add_sync(0xffffffffu, miss[r]);
                if (plan.lane == r0 + r) count = all;
                mine += all;
            }
        }
        if (i0 + plan.lane < rows.y) w.copy[i0 + plan.lane].x = count;
    }
    int found, at = rank_pages(p, plan, look, mine, w.list, &found);
    for (int i0 = rows.x; i0 < rows.y; i0 += 32) {
        int need, count = i0 + plan.lane < rows.y ? w.copy[i0 + plan.lane].x : 0, incl = count;
        const int entry = row_at(i0, &need, false);
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, incl, o);
            if (plan.lane >= o) incl += x;
        }
        const int first = at + incl - count;  // lane r: its row's first rank
        at += __shfl_sync(0xffffffffu, incl, 31);
        for (int r0 = 0; r0 < min(32, rows.y - i0); r0 += 4) {
            int rank[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) rank[r] = __shfl_sync(0xffffffffu, first, r0 + r);
            const int most = __reduce_max_sync(0xffffffffu, plan.lane >> 2 == r0 >> 2 ? need : 0);
            for (int k0 = 0; k0 < most; k0 += 64) {
                entries(entry, need, r0, k0, e);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int row = __shfl_sync(0xffffffffu, entry, r0 + r);
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const bool miss = e[r][j] == -1;
                        if (e[r][j] < -1 || e[r][j] >= p.num_pages) record_status(status, kStatusBounds);
                        const unsigned who = __ballot_sync(0xffffffffu, miss);
                        if (miss) {
                            const int to = rank[r] + __popc(who & ((1u << plan.lane) - 1u));
                            if (to < found) {
                                const int page = __ldcg(w.list + to);
                                p.block_table[row + k0 + 32 * j + plan.lane] = page;
                                p.refs[page] = 1;
                            } else {
                                record_status(status, kStatusBounds);  // no free page is left
                            }
                        }
                        rank[r] += __popc(who);
                    }
                }
            }
        }
    }
}

__global__ void __launch_bounds__(kWorkThreads) release_kernel(mla_page_pool p, int n, const int32_t *seqs,
                                                              const int32_t *lens, unsigned *status)
{
    griddep_wait();
    const int i = blockIdx.x;
    const int row = row_of(p, seqs, i), len = lens[i / p.groups];
    if (row < 0 || !len_ok(p, len)) {
        if (threadIdx.x == 0) record_status(status, kStatusBounds);
        return;
    }
    int32_t *e = p.block_table + static_cast<int64_t>(row) * p.bt_stride;
    for (int k = pages_of(len, p.page_size) + threadIdx.x; k < p.bt_stride; k += kWorkThreads) {
        const int page = e[k];
        if (page == -1) continue;
        if (page < 0 || page >= p.num_pages) {
            record_status(status, kStatusBounds);
            continue;
        }
        e[k] = -1;
        if (atomicSub(&p.refs[page], 1) <= 0) {  // the table held a page that was not counted
            atomicAdd(&p.refs[page], 1);
            record_status(status, kStatusBounds);
        }
    }
}

// The pages of their own that children copy a partial last page to: a lane a unit
// (a table row of a pair).
__global__ void __launch_bounds__(kPlanThreads) fork_plan_kernel(mla_page_pool p, int n, const int32_t *parents,
                                                                const int32_t *children, const int32_t *lens,
                                                                int32_t *ws, unsigned *status)
{
    __shared__ PlanShared sh;
    griddep_launch_dependents();  // (its only one is the launch that copies, which waits)
    griddep_wait();
    const Ws w(ws, p);
    Plan plan(sh);
    Look look;
    look.load(p, plan.first_look(), p.num_pages);
    const int2 units = plan.share(n * p.groups, 32);
    // The unit's source page: that of its partial last one (-1: nothing to copy, or a
    // fault).  Asked before any page is given out, for a page that nothing counts may be.
    auto source = [&](int i) {
        const int from = row_of(p, parents, i), to = row_of(p, children, i), len = lens[i / p.groups];
        if (from < 0 || to < 0 || from == to || !len_ok(p, len)) {
            record_status(status, kStatusBounds);
            return -1;
        }
        if (len % p.page_size == 0) return -1;
        const int k = len / p.page_size;
        const int src = p.block_table[static_cast<int64_t>(from) * p.bt_stride + k];
        if (src >= 0 && src < p.num_pages && p.refs[src] > 0 && p.block_table[static_cast<int64_t>(to) * p.bt_stride + k] == -1)
            return src;
        record_status(status, kStatusBounds);
        return -1;
    };
    int mine = 0;
    for (int i0 = units.x; i0 < units.y; i0 += 32) {
        const int i = i0 + plan.lane;
        if (i >= units.y) break;
        const int src = source(i);
        w.copy[i].x = src;
        mine += src >= 0;
    }
    __syncwarp();
    int found, at = rank_pages(p, plan, look, __reduce_add_sync(0xffffffffu, mine), w.list, &found, w.to, &w.head[1]);
    for (int i0 = units.x; i0 < units.y; i0 += 32) {
        const int i = i0 + plan.lane;
        const int src = i < units.y ? w.copy[i].x : -1;
        const unsigned who = __ballot_sync(0xffffffffu, src >= 0);
        int page = -1, rows = 0;
        if (src >= 0) {
            const int r = at + __popc(who & ((1u << plan.lane) - 1u)), len = lens[i / p.groups];
            if (r < found) {
                page = __ldcg(w.list + r);
                rows = len % p.page_size;
                p.block_table[static_cast<int64_t>(row_of(p, children, i)) * p.bt_stride + len / p.page_size] = page;
                p.refs[page] = 1;
            } else {
                record_status(status, kStatusBounds);
            }
        }
        at += __popc(who);
        if (i < units.y) w.copy[i] = make_int4(src, page, rows, 0);
    }
}

// Vectors [first, last) of the first `rows` rows of page src to page dst (both
// parts of the cache, one after the other), four of a thread's in flight.
__device__ __forceinline__ void copy_rows(const PageCache &c, const int (&width)[2], int64_t src, int64_t dst, int rows,
                                          int first, int last)
{
    const int n0 = rows * (width[0] / 8), n = min(last, n0 + rows * (width[1] / 8));
    for (int i0 = first + threadIdx.x; i0 < n; i0 += 4 * kWorkThreads) {
        uint4 v[4];
        uint16_t *to[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int i = i0 + u * kWorkThreads;
            if (i < n) {
                const int part = i >= n0, j = i - part * n0;
                const int64_t blk = part ? c.blk[1] : c.blk[0], tok = part ? c.tok[1] : c.tok[0];
                const int wide = part ? width[1] : width[0];
                int64_t at = static_cast<int64_t>(j) * 8;
                if (tok != wide) {  // (rows one behind the other need no division)
                    const int r = j / (wide / 8);
                    at += r * (tok - wide);
                }
                uint16_t *base = static_cast<uint16_t *>(part ? c.base[1] : c.base[0]) + at;
                v[u] = *reinterpret_cast<const uint4 *>(base + src * blk);
                to[u] = base + dst * blk;
            }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (i0 + u * kWorkThreads < n) *reinterpret_cast<uint4 *>(to[u]) = v[u];
    }
}

// Block (unit, layer): the unit's partial page in that layer's caches; behind the
// layers the full pages are shared.
__global__ void __launch_bounds__(kWorkThreads) fork_kernel(mla_page_pool p, const __grid_constant__ PageCaches c, int n,
                                                           const int32_t *parents, const int32_t *children,
                                                           const int32_t *lens, int32_t *ws, unsigned *status)
{
    griddep_wait();
    const Ws w(ws, p);
    const int i = blockIdx.x, layer = blockIdx.y;
    if (layer < c.n) {
        const int4 job = w.copy[i];
        if (job.y >= 0) copy_rows(c.c[layer], c.width, job.x, job.y, job.z, 0, INT_MAX);
        return;
    }
    const int from = row_of(p, parents, i), to = row_of(p, children, i), len = lens[i / p.groups];
    if (from < 0 || to < 0 || from == to || !len_ok(p, len)) return;
    const int full = len / p.page_size, looked = w.head[1];
    const int32_t *src = p.block_table + static_cast<int64_t>(from) * p.bt_stride;
    int32_t *dst = p.block_table + static_cast<int64_t>(to) * p.bt_stride;
    for (int k = threadIdx.x; k < full; k += kWorkThreads) {
        const int page = src[k];
        // (a page that nothing counts may have been given out since: what the plan saw tells)
        if (page < 0 || page >= p.num_pages || dst[k] != -1 ||
            (page < looked ? w.to[page / 32] >> (page % 32) & 1 : p.refs[page] <= 0)) {
            record_status(status, kStatusBounds);
            continue;
        }
        dst[k] = page;
        atomicAdd(&p.refs[page], 1);
    }
}

__global__ void __launch_bounds__(kPlanThreads) compact_plan_kernel(mla_page_pool p, int32_t *ws)
{
    __shared__ PlanShared sh;
    griddep_launch_dependents();  // (its only one is the launch that copies, which waits)
    griddep_wait();
    const Ws w(ws, p);
    Plan plan(sh);
    const int2 pages = plan.share(p.num_pages, 32);
    // a range of kLook x 32 pages at most is looked at once for all that follows
    const bool once = pages.y - pages.x <= 32 * kLook;
    Look look;
    int live = 0;
    for (int64_t page0 = pages.x; page0 < pages.y; page0 += 32 * kLook) {
        look.load(p, page0, pages.y);
        live += static_cast<int>(min(pages.y - page0, int64_t{32 * kLook})) - look.count();
    }
    int2 total;
    plan.scan(live, 0, &total);
    const int used = total.x;
    // free below `used` (a hole) and in use above it (to be moved): as many of the one as of the other
    auto parts = [&](int64_t page0, unsigned f, unsigned *holes, unsigned *moves) {
        const int64_t below = min(max(used - page0, int64_t{0}), int64_t{32}), in = min(pages.y - page0, int64_t{32});
        const unsigned low = below == 32 ? ~0u : (1u << below) - 1u, valid = in == 32 ? ~0u : (1u << in) - 1u;
        *holes = f & low & valid;
        *moves = ~f & ~low & valid;
    };
    int holes = 0, moves = 0;
    unsigned h, m;
    for (int64_t page0 = pages.x; page0 < pages.y; page0 += 32 * kLook) {
        if (!once) {
            look.load(p, page0, pages.y);
            look.count();
        }
#pragma unroll
        for (int j = 0; j < kLook; ++j) {
            if (page0 + 32 * j >= pages.y) break;
            parts(page0 + 32 * j, look.free[j], &h, &m);
            holes += __popc(h);
            moves += __popc(m);
        }
    }
    int2 at = plan.scan(holes, moves, &total);
    const unsigned lower = (1u << plan.lane) - 1u;
    for (int64_t page0 = pages.x; page0 < pages.y; page0 += 32 * kLook) {
        if (!once) {
            look.load(p, page0, pages.y);
            look.count();
        }
#pragma unroll
        for (int j = 0; j < kLook; ++j) {
            const int page = static_cast<int>(page0) + 32 * j + plan.lane;
            if (page0 + 32 * j >= pages.y) break;
            parts(page0 + 32 * j, look.free[j], &h, &m);
            if (h >> plan.lane & 1) w.list[at.x + __popc(h & lower)] = page;
            if (m >> plan.lane & 1)
                w.src[at.y + __popc(m & lower)] = page;
            else if (page < pages.y)
                w.to[page] = look.free[j] >> plan.lane & 1 ? -1 : page;  // (nothing counts a free one)
            at.x += __popc(h);
            at.y += __popc(m);
        }
    }
    plan.sync();  // the lists are written, and nothing counts any more
    for (int i = plan.warp * 32 + plan.lane; i < total.y; i += plan.warps * 32) {
        const int src = __ldcg(w.src + i), dst = __ldcg(w.list + i);
        w.to[src] = dst;
        p.refs[dst] = p.refs[src];
        p.refs[src] = 0;
    }
    if (plan.warp == 0 && plan.lane == 0) w.head[0] = total.y;
}

// The table's entries, then the moved pages, 1024 vectors of a layer's page a step.
__global__ void __launch_bounds__(kWorkThreads, kCopyCtas) compact_kernel(mla_page_pool p, const __grid_constant__ PageCaches c,
                                                                         int32_t *ws, unsigned *status)
{
    griddep_wait();
    const Ws w(ws, p);
    const int moves = w.head[0];
    const int64_t entries = static_cast<int64_t>(p.num_rows) * p.bt_stride;
    for (int64_t i = blockIdx.x * kWorkThreads + threadIdx.x; i < entries; i += gridDim.x * kWorkThreads) {
        const int page = p.block_table[i];
        if (page == -1) continue;
        const int to = page >= 0 && page < p.num_pages ? w.to[page] : -1;
        if (to < 0)
            record_status(status, kStatusBounds);  // no such page, or one that nothing counts
        else if (to != page)
            p.block_table[i] = to;
    }
    const int vectors = p.page_size * ((c.width[0] + c.width[1]) / 8), chunks = (vectors + kChunk - 1) / kChunk;
    const int64_t jobs = static_cast<int64_t>(moves) * c.n * chunks;
    for (int64_t j = blockIdx.x; j < jobs; j += gridDim.x) {
        const int64_t page = j / chunks;
        const int chunk = static_cast<int>(j - page * chunks), i = static_cast<int>(page / c.n), layer = static_cast<int>(page - static_cast<int64_t>(i) * c.n);
        copy_rows(c.c[layer], c.width, w.src[i], w.list[i], p.page_size, chunk * kChunk, (chunk + 1) * kChunk);
    }
}

}  // namespace

namespace {
// CTAs of a plan: one, whose barriers cost less, where each of its 32 warps has no more
// than four rows (of `rows`) and 512 pages to go through, else a cluster.  Reserving
// for 4 sequences of 8 rows from 200 pages 6.8 us against 7.9; a compaction, which
// moves pages' counts too, is better off with a cluster from 4096 pages on (12 900
// pages of the latent cache: 95 us with one CTA, 90 so).
int plan_ctas(const mla_page_pool &p, int64_t rows, int pages = kCtaWarps * kLook * 32)
{
    return rows <= 4 * kCtaWarps && p.num_pages <= pages ? 1 : kMaxPlanCtas;
}
}  // namespace

size_t pages_workspace_ints(const mla_page_pool &p)
{
    return kHead + 4 * static_cast<size_t>(p.num_rows) + 3 * static_cast<size_t>(p.num_pages);
}

// (none of a call's last launches triggers its dependents early: attention kernels
// read tables and caches before their wait)
cudaError_t launch_pages_release(const mla_page_pool &p, int n, const int32_t *seqs, const int32_t *lens,
                                 unsigned *status, cudaStream_t st)
{
    return launch_dependent(release_kernel, dim3(n * p.groups), dim3(kWorkThreads), 0, st, 1, p, n, seqs, lens, status);
}

cudaError_t launch_pages_reserve(const mla_page_pool &p, int n, const int32_t *seqs, const int32_t *lens, int32_t *ws,
                                 unsigned *status, cudaStream_t st)
{
    const int ctas = plan_ctas(p, static_cast<int64_t>(n) * p.groups);
    return launch_dependent(reserve_kernel, dim3(ctas), dim3(kPlanThreads), 0, st, ctas, p, n, seqs, lens, ws, status);
}

cudaError_t launch_pages_fork(const mla_page_pool &p, const PageCaches &c, int n, const int32_t *parents,
                              const int32_t *children, const int32_t *lens, int32_t *ws, unsigned *status,
                              cudaStream_t st)
{
    const int ctas = plan_ctas(p, static_cast<int64_t>(n) * p.groups / 8);  // (a lane a row)
    const cudaError_t e = launch_dependent(fork_plan_kernel, dim3(ctas), dim3(kPlanThreads), 0, st, ctas, p, n, parents, children, lens, ws, status);
    if (e != cudaSuccess) return e;
    return launch_dependent(fork_kernel, dim3(n * p.groups, c.n + 1), dim3(kWorkThreads), 0, st, 1, p, c, n, parents,
                            children, lens, ws, status);
}

cudaError_t launch_pages_compact(const mla_page_pool &p, const PageCaches &c, int32_t *ws, unsigned *status, int sms,
                                 cudaStream_t st)
{
    const int ctas = plan_ctas(p, 0, 4096);
    const cudaError_t e = launch_dependent(compact_plan_kernel, dim3(ctas), dim3(kPlanThreads), 0, st, ctas, p, ws);
    if (e != cudaSuccess) return e;
    return launch_dependent(compact_kernel, dim3(kCopyCtas * sms), dim3(kWorkThreads), 0, st, 1, p, c, ws, status);
}

}  // namespace gbmla
