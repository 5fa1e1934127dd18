// mla_gqa_prompt_attn: causal attention of packed prompts over the original GQA
// layer's caches (Sec. 3.1, Eqs. 2-4), on the tensor cores.
//
// An item is two tiles ("halves") of up to 128 query rows each: floor(128 / hpg)
// consecutive tokens of a sequence times the hpg heads of one KV group, so that a
// key tile read once serves every head of its group.  Per 128-key tile and half
//     S[rows, keys] = Q (K-major smem) x K^T (K-major smem)        fp32 in TMEM
//     P             = 2^(S scale - base), bf16, written back to TMEM
//     O[rows, D]   += P (TMEM) x V (MN-major smem)                 fp32 in TMEM
// with one query row a TMEM lane and a softmax thread: maxima and sums need no
// exchange between threads.  The two halves take turns: while the tensor core
// works for one, the other's softmax runs.
//
// One CTA an SM, one partition a CTA: all items' key tiles, in order, form one
// list, which the partitions cut evenly (as the decode path cuts its own), so
// that prompts of any lengths keep all SMs busy to the end.  An item that a cut
// falls into leaves partials, joined afterwards.
//
// Warps: 0 the TMA producer, 1 and 2 the MMA issuers of halves 0 and 1, 3 the
// scheduler, which finds the partition's pieces (items, or their parts) and
// hands them to the others, 4-7 and 8-11 the softmax of halves 0 and 1.  Loads,
// products and softmax run on from one piece into the next.  TMEM, D = 64: S of
// both halves, O of both, P of both, 512 columns in all, so that the next S is
// made while P is still being made; D = 128: O takes 256 columns and P lies over
// its own S.
//
// Bound.  A half's tile costs the tensor pipe 525 cycles at D = 64 and 1025 at 128,
// and the exponential units 512 (32 lanes a clock).  D = 128 comes close: 8191 tokens
// of 24 heads in 272 to 279 us from box to box, 1.48 to 1.52 PFLOP/s, 2320 cycles a
// tile of both halves.  D = 64 is bound by the chain of one half's softmax, with this
// layout (128-key tiles, P beside S, two halves, whose warps store their own rows):
// wait, 128 scores out of TMEM (170 cycles),
// maximum (500), weights (950), store, hand over; 1930 cycles a tile of both halves,
// the tensor pipe 53 % and the issue slots 57 % busy.  Chunks of 125 to 475 tokens
// behind prefixes of 4000 to 16000 (14 heads, 2 groups) take 84 us, 32 prompts of 17
// to 1009 tokens (32 heads, 8 groups) 88 us, where an item's ends (3400 cycles) weigh
// as much as two tiles.  Tried: twice the softmax warps, each half of a row's scores
// (102 us for the chunks: the chain's waits double, its arithmetic does not halve);
// no maximum after the first tile, a sum's overflow asking for another base instead
// (the scores must outlive the weights, and registers spill: 92 us); the first half of
// the weights handed over early (D = 64: nothing waits for its products).
#include <cudaTypedefs.h>
#include <limits.h>
#include <math.h>

#include "common.cuh"
#include "internal.h"
#include "tc.cuh"

namespace gbmla {
namespace {

constexpr int kTile = 128;                 // keys a tile, rows a half
constexpr int kPage = 64;
constexpr int kAtom = kTile * 128;         // 128 rows x 64 columns, 128-byte swizzle
constexpr int kThreads = 384;
constexpr int kProducer = 0, kIssuer = 1, kScheduler = 3, kSoftmax = 4;  // warps
// Registers a thread of 12 warps: 168 at launch, three warps a quarter of the
// SM; the softmax warps, with a row of 128 scores each, take what the first four
// warps give: 104 + 2 x 200 = 504 = 3 x 168.
constexpr int kFewRegs = 104, kMoreRegs = 200;
// An item's own cost in the list, in keys: its queries in, its rows out.  (Least
// squares over the CTAs of a launch: a tile of both halves 1930 cycles, an item 3430,
// a cut 410 at D = 64; 2320, 5820, 1640 at D = 128.)
template <int D>
constexpr int kItemUnits = D == 64 ? 2 * kTile : 3 * kTile;
constexpr int kLeastTiles = 4;             // a piece of an item is at least this many tiles (2: prompts of 17 to 1009 tokens + 3 %)
constexpr int kPieces = 4;                 // pieces handed out ahead

template <int D>
constexpr int kSlots = D == 64 ? 8 : 5;    // ring slots, one tile of keys or values each
template <int D>
constexpr int kQBufs = D == 64 ? 2 : 1;    // query buffers, both halves of an item each
template <int D>
constexpr size_t kSmem = 1024 + (static_cast<size_t>(2 * kQBufs<D> + kSlots<D>) * (D / 64) + (D == 64 ? 2 : 0)) * kAtom;

struct Args {
    int batch, total, groups, hpg, max_kv;
    int parts;                             // partitions
    int tpt;                               // tokens of a half
    int item;                              // kItemUnits
    int cut;                               // items are cut (else partitions begin and end with them)
    int paged, bt_stride, num_pages;
    float scale_log2;
    const int32_t *cu, *kv_len, *block_table;
    uint16_t *o;
    float *lse, *o_part, *lse_part;
    struct Cut *cuts;                      // one a partition, for the join
    unsigned *status;
};

// What the join needs of a partition: the item that its end cuts (last: the last
// partition with a piece of it, -1 where none begins here), and whether its own
// first piece goes on with another partition's item.
struct Cut {
    int tok, ntok, pos, g, last, goes_on, pad[2];
};

// What the warps work on next: an item's key tiles [t0, t0 + n), n the larger of
// its halves' n0 and n1.
struct Piece {
    int u, g, kv;                          // unit (-1: no piece is left), group, cached tokens
    int tok, ntok, pos;                    // first packed token, tokens, position of the first
    int t0, n0, n1;
    int slot;                              // partial slot, -1: the whole item
};

static_assert(sizeof(Cut) == kPromptCutBytes && kPromptPartRows == 4 * kTile, "two items a partition");

struct __align__(8) Bars {
    uint64_t full[8], empty[8];            // ring
    uint64_t piece_full[kPieces], piece_empty[kPieces];
    uint64_t q_full[2][2], q_free[2][2], drain[2];  // (buffer, half)
    uint64_t turn[2][4];                   // the exponentials of a half's warp, after the other half's
    uint64_t out_ready[2][2], out_free[2];  // the rows on their way out; ready: stores in turn, for a warp may be one ahead
    uint64_t s_full[2], s_free[2], p_full[2][2], pv_done[2], o_free[2];  // p_full: the first and the last 64 keys' weights
};

struct Shared {
    Bars bars;
    Piece pieces[kPieces];
    uint32_t tmem;
};

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint64_t pack2(float lo, float hi)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float &lo, float &hi)
{
    asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b)
{
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    const __nv_bfloat162 h2 = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h2);
}

__device__ __forceinline__ float max3(float a, float b, float c)
{
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ float max32(const uint32_t *x)
{
    float m[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) m[i] = fmaxf(__uint_as_float(x[i]), __uint_as_float(x[i + 4]));
#pragma unroll
    for (int i = 8; i < 32; i += 2) m[(i / 2) % 4] = max3(m[(i / 2) % 4], __uint_as_float(x[i]), __uint_as_float(x[i + 1]));
    return fmaxf(max3(m[0], m[1], m[2]), m[3]);
}

// A wait of a whole warp, as few instructions as it takes: waits stand at every
// turn of the roles' loops, and with the clock read between looks (mbar_wait_warp)
// and the loops unrolled they made 245 KB of code, which the instruction caches do
// not hold.  At 3.8 us a look (measured where nothing ever arrives) these are 0.94 s.
constexpr int kLooks = 250000;
__device__ __forceinline__ bool wait_warp(uint32_t bar, int phase) { return mbar_wait_looks<kLooks>(bar, phase & 1); }

// Whether a phase has ended, for the lanes to agree on later (`all`): a wait costs
// some 130 cycles even where there is nothing to wait for, and a look that is made
// ahead of other work costs next to nothing.  (The phase before has been waited for.)
__device__ __forceinline__ uint32_t looked(const uint64_t *bar, int phase)
{
    uint32_t done;
    asm volatile("{\n .reg .pred p;\n mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
                 : "=r"(done)
                 : "r"(smem_u32(bar)), "r"(phase & 1)
                 : "memory");
    return done;
}
__device__ __forceinline__ bool all(uint32_t done) { return __all_sync(0xffffffffu, done); }

// ---------------------------------------------------------------- the list of tiles
// Items in the order sequence, group, tokens; an item's units are kItemUnits<D> of its
// own and the keys that its last token sees (so that sums over items are arithmetic
// series).  Partition k begins at unit k q, q about T / S, at the tile that holds it; a
// cut close to an item's ends moves there.

// Tokens of sequence b (0 where its offsets are faulty), and its cached tokens (0 where its length is).
__device__ __forceinline__ int tokens_of(const Args &a, int b)
{
    const int first = a.cu[b], end = a.cu[b + 1];
    return first >= 0 && end >= first && end <= a.total ? end - first : 0;
}
__device__ __forceinline__ int cached_of(const Args &a, int b)
{
    const int kv = a.kv_len[b];
    return kv >= 0 && kv <= a.max_kv ? kv : 0;
}

struct Seq {
    int n, p0, items;  // tokens, position of the first, items a group
    int full, dark;    // items of as many tokens as an item has, and those of them that see no key
};
__device__ __forceinline__ Seq seq_of(const Args &a, int b)
{
    Seq s{0, 0, 0, 0, 0};
    if (b < a.batch) {
        const int per = 2 * a.tpt;
        s.n = tokens_of(a, b);
        s.p0 = cached_of(a, b) - s.n;
        s.full = s.n / per;
        s.items = s.full + (s.n > s.full * per);
        s.dark = s.p0 >= 0 ? 0 : min(s.full, -s.p0 / per);
    }
    return s;
}
// Keys that item k's last token sees, and their tiles.
__device__ __forceinline__ int keys_of(const Seq &s, int per, int k) { return max(0, s.p0 + min((k + 1) * per, s.n)); }
__device__ __forceinline__ int tiles_of(const Seq &s, int per, int k) { return (keys_of(s, per, k) + kTile - 1) / kTile; }
// Units of a group's first m items.
__device__ __forceinline__ int64_t units_before(const Args &a, const Seq &s, int m)
{
    const int per = 2 * a.tpt;
    const int whole = min(m, s.full), k0 = min(whole, s.dark);
    const int64_t c = whole - k0;
    int64_t u = c * s.p0 + per * ((static_cast<int64_t>(k0) + 1 + whole) * c / 2);
    if (m > whole) u += keys_of(s, per, whole);
    return u + static_cast<int64_t>(a.item) * m;
}

// Where a partition begins: at tile t of item k of group g of sequence b (b ==
// batch: past the list); `at` is the item's first unit.  The same in every lane.
struct Place {
    int b, g, k, t;
    Seq s;
    int64_t at;
    // on to the next item
    __device__ void next(const Args &a)
    {
        t = 0;
        at += a.item + keys_of(s, 2 * a.tpt, k);
        if (++k < s.items) return;
        k = 0;
        if (++g < a.groups) return;
        g = 0;
        do {
            ++b;
            s = seq_of(a, b);
        } while (b < a.batch && s.items == 0);
    }
    __device__ bool same(const Place &o) const { return b == o.b && g == o.g && k == o.k; }
};

// The list's length, a partition's, and the fewest tiles of a piece of an item (a
// 64th of a partition more or less, rather than two partials; a sixteenth: chunks
// behind long prefixes 84.5 us, 83.3 so).  Quotients in
// fp32: every CTA has the same ones, and an int64 division is a long piece of code.
struct List {
    int64_t T, q;
    int least;
    __device__ __forceinline__ List(const Args &a, int64_t units) : T(units)
    {
        const float f = static_cast<float>(units), parts = static_cast<float>(a.parts);
        q = max(int64_t{1}, static_cast<int64_t>(f / parts));
        least = max(kLeastTiles, static_cast<int>(f / (64.f * parts * kTile)));
    }
    __device__ __forceinline__ int64_t begin(const Args &a, int k) const { return k < a.parts ? min(k * q, T) : T; }
    // The partition that holds unit x.
    __device__ __forceinline__ int part_of(const Args &a, int64_t x) const
    {
        int k = min(static_cast<int>(static_cast<float>(x) / static_cast<float>(q)), a.parts - 1);
        while (begin(a, k) > x) --k;
        while (begin(a, k + 1) <= x) ++k;
        return k;
    }
};

// The tile of the item at unit `at` that unit x falls into (0: or before it).
__device__ __forceinline__ int tile_at(const Args &a, int64_t x, int64_t at)
{
    const int64_t k = x - at - a.item;
    return k < 0 ? 0 : static_cast<int>(k / kTile);
}

// 32 sequences, one a lane: the units of a group of theirs, and of all groups up to
// and with theirs.
struct Chunk {
    int b0;
    Seq s;
    int64_t w, incl;
    __device__ __forceinline__ void fill(const Args &a, int b)
    {
        const int lane = threadIdx.x & 31;
        b0 = b;
        s = seq_of(a, b + lane);
        w = units_before(a, s, s.items);
        incl = w * a.groups;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t v = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += v;
        }
    }
};

// Partition `part`: where it begins and ends.  A warp, converged.  Three rounds of
// one piece of code, which runs once a launch and comes from far away: the list's
// length, then the partition's ends.
__device__ __forceinline__ List locate(const Args &a, int part, Place &from, Place &to)
{
    const int lane = threadIdx.x & 31, per = 2 * a.tpt;
    Chunk c;
    c.b0 = -1;
    List list(a, 0);
#pragma unroll 1
    for (int round = 0; round < 3; ++round) {
        const int64_t x = round == 0 ? INT64_MAX : list.begin(a, part + round - 1);
        int64_t base = 0;
        Place p{a.batch, 0, 0, 0, {0, 0, 0, 0, 0}, list.T};
#pragma unroll 1
        for (int b = 0; b < a.batch && (round == 0 || x < list.T); b += 32) {
            if (c.b0 != b) c.fill(a, b);
            const unsigned hit = __ballot_sync(0xffffffffu, base + c.incl > x);
            if (hit == 0) {
                base += __shfl_sync(0xffffffffu, c.incl, 31);
                continue;
            }
            const int src = __ffs(hit) - 1;
            p.b = b + src;
            p.s.n = __shfl_sync(0xffffffffu, c.s.n, src);
            p.s.p0 = __shfl_sync(0xffffffffu, c.s.p0, src);
            p.s.items = __shfl_sync(0xffffffffu, c.s.items, src);
            p.s.full = __shfl_sync(0xffffffffu, c.s.full, src);
            p.s.dark = __shfl_sync(0xffffffffu, c.s.dark, src);
            const int64_t one = __shfl_sync(0xffffffffu, c.w, src);
            base += __shfl_sync(0xffffffffu, c.incl, src) - one * a.groups;
            int g = -1;  // the last group that begins at or before x
            for (int g0 = 0; g0 < a.groups; g0 += 32)
                g += __popc(__ballot_sync(0xffffffffu, g0 + lane < a.groups && base + (g0 + lane) * one <= x));
            p.g = g;
            base += g * one;
            // the last item that begins at or before x, 32 candidates at a time
            int lo = 0, cnt = p.s.items;
            while (cnt > 1) {
                const int step = (cnt + 31) / 32, k = lo + lane * step;
                const bool in = lane * step < cnt && base + units_before(a, p.s, k) <= x;
                const int top = 31 - __clz(__ballot_sync(0xffffffffu, in));
                lo += top * step;
                cnt = min(step, cnt - top * step);
            }
            p.k = lo;
            p.at = base + units_before(a, p.s, lo);
            const int nt = tiles_of(p.s, per, lo), least = a.cut ? list.least : nt + 1;
            p.t = tile_at(a, x, p.at);
            if (p.t < least)
                p.t = 0;
            else if (nt - p.t < least)
                p.next(a);
            break;
        }
        if (round == 0)
            list = List(a, base);
        else if (round == 1)
            from = p;
        else
            to = p;
    }
    return list;
}

// A place in the ring.
template <int NS>
struct RingPos {
    int slot, round;
    __device__ void advance()
    {
        if (++slot == NS) {
            slot = 0;
            ++round;
        }
    }
    __device__ RingPos plus(int d) const { return {(slot + d) % NS, round + (slot + d) / NS}; }
};

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
    prompt_attn_kernel(const __grid_constant__ Args a, const __grid_constant__ CUtensorMap map_q,
                       const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                       const __grid_constant__ CUtensorMap map_o, const __grid_constant__ CUtensorMap map_part)
{
    constexpr int KA = D / 64, NS = kSlots<D>, NQ = kQBufs<D>;
    constexpr bool SEP = D == 64;          // P beside S
    constexpr uint32_t kS = 0, kO = 256, kP = SEP ? 256 + 2 * D : 0, kPStep = SEP ? 64 : 128;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    __shared__ Shared sh;
    Bars &bars = sh.bars;
    // (values that the compiler sees to be the warp's own stay in uniform registers,
    // which the tensor instructions take their operands from)
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    if (tid == 0) {
        for (int s = 0; s < NS; ++s) {
            mbar_init(&bars.full[s], 1);
            mbar_init(&bars.empty[s], 8);
        }
        for (int s = 0; s < kPieces; ++s) {
            mbar_init(&bars.piece_full[s], 1);
            mbar_init(&bars.piece_empty[s], 11);  // the producer, two issuers, eight softmax warps
        }
        for (int h = 0; h < 2; ++h) {
            for (int q = 0; q < 2; ++q) {
                mbar_init(&bars.q_full[q][h], 1);
                mbar_init(&bars.q_free[q][h], SEP ? 4 : 1);
            }
            mbar_init(&bars.drain[h], 1);
            for (int q = 0; q < 4; ++q) mbar_init(&bars.turn[h][q], 1);
            mbar_init(&bars.s_full[h], 1);
            mbar_init(&bars.s_free[h], 4);
            mbar_init(&bars.p_full[h][0], 4);
            mbar_init(&bars.p_full[h][1], 4);
            mbar_init(&bars.pv_done[h], 1);
            mbar_init(&bars.o_free[h], 4);
            mbar_init(&bars.out_ready[h][0], 4);
            mbar_init(&bars.out_ready[h][1], 4);
            mbar_init(&bars.out_free[h], 1);
        }
        tc::fence_barrier_init();
        tc::prefetch_tensormap(&map_q);
        tc::prefetch_tensormap(&map_k);
        tc::prefetch_tensormap(&map_v);
    }
    if (warp == kIssuer) {
        tc::tmem_alloc(smem_u32(&sh.tmem), 512);
        tc::tmem_relinquish();
    }
    griddep_wait();
    griddep_launch_dependents();
    if (blockIdx.x == 0) {
        for (int b = tid; b < a.batch; b += kThreads) {
            const int kv = a.kv_len[b];
            if (a.cu[b] < 0 || a.cu[b + 1] < a.cu[b] || a.cu[b + 1] > a.total || kv < 0 || kv > a.max_kv)
                record_status(a.status, kStatusBounds);
        }
    }
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    const uint32_t tmem = __shfl_sync(0xffffffffu, sh.tmem, 0);
    const uint32_t q_s = (smem_u32(smem_raw) + 1023u) & ~1023u, ring = q_s + 2 * NQ * KA * kAtom, stage = SEP ? ring + NS * KA * kAtom : q_s;
    bool ok = true;
    auto wait = [&](uint64_t *bar, int phase) {
        if (ok) ok = wait_warp(smem_u32(bar), phase);
        return ok;
    };
    auto own = [](int x) { return __shfl_sync(0xffffffffu, x, 0); };
    // The idx-th piece once it is there; taken: this warp needs it no more.
    auto piece_at = [&](int idx) -> const Piece & {
        wait(&bars.piece_full[idx % kPieces], idx / kPieces);
        return sh.pieces[idx % kPieces];
    };
    auto taken = [&](int idx) {
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(smem_u32(&bars.piece_empty[idx % kPieces]));
    };

    if (warp < kSoftmax) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kFewRegs));
        if (warp == kScheduler) {
            const int part = blockIdx.x, per = 2 * a.tpt;
            Place at, end;
            const List list = locate(a, part, at, end);
            if (a.cut && lane == 0) {
                // (T > 0 where an end lies in an item)
                Cut c{0, 0, 0, 0, -1, at.t > 0 && !(at.same(end) && at.t >= end.t), {}};
                if (end.b < a.batch && end.t > 0 && !(at.same(end) && at.t > 0)) {
                    c.tok = a.cu[end.b] + end.k * per;
                    c.ntok = min(per, end.s.n - end.k * per);
                    c.pos = end.s.p0 + end.k * per;
                    c.g = end.g;
                    c.last = list.part_of(a, end.at + a.item + static_cast<int64_t>(tiles_of(end.s, per, end.k) - list.least + 1) * kTile - 1);
                }
                a.cuts[part] = c;
            }
            int idx = 0;
            for (bool more = true; ok; ++idx) {
                more = more && at.b < a.batch && !(at.same(end) && at.t >= end.t);
                if (idx >= kPieces && !wait(&bars.piece_empty[idx % kPieces], idx / kPieces - 1)) break;
                if (lane == 0) {
                    Piece p;
                    p.u = -1;
                    if (more) {
                        const int nt = tiles_of(at.s, per, at.k), t1 = at.same(end) ? end.t : nt;
                        p.u = at.b * a.groups + at.g;
                        p.g = at.g;
                        p.kv = at.s.p0 + at.s.n;
                        p.tok = a.cu[at.b] + at.k * per;
                        p.ntok = min(per, at.s.n - at.k * per);
                        p.pos = at.s.p0 + at.k * per;
                        p.t0 = at.t;
                        auto tiles_to = [&](int last) { return max(0, min(t1, last < 0 ? 0 : last / kTile + 1) - at.t); };
                        p.n0 = tiles_to(p.pos + min(p.ntok, a.tpt) - 1);
                        p.n1 = p.ntok > a.tpt ? tiles_to(p.pos + p.ntok - 1) : 0;
                        p.slot = at.t == 0 && t1 == nt ? -1 : at.t > 0 ? 2 * part : 2 * part + 1;
                    }
                    sh.pieces[idx % kPieces] = p;
                }
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(smem_u32(&bars.piece_full[idx % kPieces]));
                if (!more) break;
                if (lane < 2 * KA) {  // the queries as far as the L2
                    const Piece &p = sh.pieces[idx % kPieces];
                    if ((lane < KA ? p.n0 : p.n1) > 0)
                        tc::tma_prefetch_3d(&map_q, 64 * (lane % KA), p.g * a.hpg, p.tok + (lane / KA) * a.tpt);
                }
                __syncwarp();
                if (at.same(end))
                    more = false;
                else
                    at.next(a);
            }
        } else if (warp == kProducer) {
            RingPos<NS> rp{0, 0};
            int issued = 0, loads[2] = {0, 0};  // ring loads, and query loads of each half
            const uint64_t policy = tc::policy_evict_last();
            const uint32_t box = static_cast<uint32_t>(a.tpt * a.hpg) * 128;
            for (int idx = 0; ok; ++idx) {
                const Piece p = piece_at(idx);
                if (!ok) break;
                taken(idx);
                if (p.u < 0) break;
                const int n = max(p.n0, p.n1);
                auto queries = [&](int h) {
                    if ((h ? p.n1 : p.n0) == 0) return;
                    const int i = loads[h], qb = i % NQ;
                    if (i >= NQ && !wait(&bars.q_free[qb][h], i / NQ - 1)) return;
                    const uint32_t bar = smem_u32(&bars.q_full[qb][h]);
                    tc::mbar_arrive_expect_tx_elect(bar, KA * box);
                    for (int k = 0; k < KA; ++k)
                        tc::tma_load_3d_elect(q_s + ((qb * 2 + h) * KA + k) * kAtom, &map_q, 64 * k, p.g * a.hpg, p.tok + h * a.tpt, bar);
                    ++loads[h];
                };
                queries(0);
                int page_0 = -64, page_id = 0;
                for (int j = 0; j < n && ok; ++j) {
                    const int key = (p.t0 + j) * kTile;
                    int blk[2] = {p.u, p.u}, boxes = 1;
                    if (a.paged) {
                        const int pg = key / kPage, pages = (p.kv + kPage - 1) / kPage;
                        if (pg + 1 >= page_0 + 32) {
                            page_0 = pg;
                            page_id = pg + lane < pages ? a.block_table[static_cast<int64_t>(p.u) * a.bt_stride + pg + lane] : 0;
                        }
                        boxes = pages - pg > 1 ? 2 : 1;
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            blk[x] = __shfl_sync(0xffffffffu, page_id, pg + x - page_0);
                            if (x < boxes && (blk[x] < 0 || blk[x] >= a.num_pages)) {
                                if (lane == 0) record_status(a.status, kStatusBounds);
                                boxes = x;
                            }
                        }
                    }
                    const uint32_t bytes = static_cast<uint32_t>(boxes) * (a.paged ? kPage : kTile) * 128 * KA;
#pragma unroll
                    for (int kvi = 0; kvi < 2; ++kvi, ++issued, rp.advance()) {  // keys, then values
                        const uint32_t full = smem_u32(&bars.full[rp.slot]), dst = ring + rp.slot * KA * kAtom;
                        if (rp.round > 0 && !wait(&bars.empty[rp.slot], rp.round - 1)) break;
                        tc::mbar_arrive_expect_tx_elect(full, bytes);
                        const CUtensorMap *map = kvi ? &map_v : &map_k;
                        for (int x = 0; x < boxes; ++x)
                            for (int k = 0; k < KA; ++k)
                                tc::tma_load_3d_hint_elect(dst + k * kAtom + x * kPage * 128, map, 64 * k, a.paged ? 0 : key, blk[x],
                                                           full, policy);
                    }
                    // (the second half's queries may be in use for a tile longer)
                    if (j == 0 && ok) queries(1);
                }
            }
            if (!ok) {
                // the loads in flight land before the shared memory goes
                for (int i = max(0, issued - NS); i < issued; ++i)
                    wait_warp(smem_u32(&bars.full[i % NS]), i / NS);
                for (int h = 0; h < 2; ++h)
                    for (int i = max(0, loads[h] - NQ); i < loads[h]; ++i)
                        wait_warp(smem_u32(&bars.q_full[i % NQ][h]), i / NQ);
            }
        } else {
            // An issuer a half: what it waits for and works out between its products is
            // hidden behind the other's.
            const int h = warp - kIssuer;
            constexpr uint32_t id_qk = tc::idesc_bf16_f32(128, kTile, false, false), id_pv = tc::idesc_bf16_f32(128, D, false, true);
            // descriptors (their low words) of Q and of the ring's first slot, as keys and
            // as values; a slot further is kSlot16 more
            constexpr uint32_t kSlot16 = KA * kAtom / 16;
            const uint32_t dq = tc::smem_desc_lo(q_s + h * KA * kAtom, 16), dk = tc::smem_desc_lo(ring, 16), dv = tc::smem_desc_lo(ring, kAtom);
            const uint32_t s_full = smem_u32(&bars.s_full[h]), pv_done = smem_u32(&bars.pv_done[h]);
            const uint32_t d_s = tmem + kS + h * 128, d_o = tmem + kO + h * D, d_p = tmem + kP + h * kPStep;
            int tile = 0, pieces = 0;  // this half's tiles and pieces so far
            // Few commits and no waits but for what is needed: the ring's slots are given
            // back by the softmax warps, which see the scores and the products complete
            // anyway.  The scores of this half's piece q with the keys at `at`, once S may
            // be written (D = 128: behind the products that read the last P).
            auto qk = [&](int q, RingPos<NS> at, bool first) {
                if (first && !wait(&bars.q_full[q % NQ][h], q / NQ)) return;
                if ((SEP || first) && !wait(&bars.full[at.slot], at.round)) return;
                if (SEP && tile > 0 && !wait(&bars.s_free[h], tile - 1)) return;
                tc::fence_after_sync();
                const uint32_t q0 = dq + q % NQ * 2 * kSlot16, k_0 = dk + at.slot * kSlot16;
#pragma unroll
                for (int k = 0; k < KA; ++k) tc::mma4_ss_sw128(d_s, q0 + k * (kAtom / 16), k_0 + k * (kAtom / 16), id_qk, k > 0);
                tc::commit_elect(s_full);
            };
            // What only the other half uses is waited for and given back here, for this
            // half's four softmax warps: whoever skipped a phase of a barrier could take the
            // one after the next for it.
            auto give_back = [&](uint64_t *bar) {
                if (lane == 0) tc::mbar_arrive(smem_u32(bar), 4);
            };
            RingPos<NS> base{0, 0};  // the piece's first keys
            bool ahead = false;      // its first scores have been issued
            for (int idx = 0; ok; ++idx) {
                const Piece &p = piece_at(idx);
                if (!ok) break;
                const int u = own(p.u), n0 = own(p.n0), n1 = own(p.n1), kv = own(p.kv), t0 = own(p.t0);
                taken(idx);
                if (u < 0) break;
                const int n = max(n0, n1), nh = h ? n1 : n0;
                if (n == 0) continue;
                const RingPos<NS> after = base.plus(2 * n);
                const int q = pieces;
                if (nh > 0 && !ahead) qk(q, base, true);
                ahead = false;
                // the next piece's first scores
                auto look = [&] {
                    const Piece &next = piece_at(idx + 1);
                    if (!ok) return;
                    const int nu = own(next.u), nn = own(h ? next.n1 : next.n0);
                    if (nu < 0 || nn == 0) return;
                    qk(q + 1, after, true);
                    ahead = true;
                };
                RingPos<NS> vp = base, kp = base;
                vp.advance();
                for (int j = 0; j < nh && ok; ++j) {
                    const bool last = j + 1 == nh;
                    ++tile;
                    kp.advance();
                    kp.advance();
                    if (SEP) {
                        if (!last)
                            qk(q, kp, false);
                        else
                            look();
                    } else if (!last && !wait(&bars.full[kp.slot], kp.round)) {
                        break;
                    }
                    if (!wait(&bars.full[vp.slot], vp.round)) break;
                    const uint32_t b = dv + vp.slot * kSlot16;
                    if (j == 0 && pieces > 0 && !wait(&bars.o_free[h], pieces - 1)) break;
                    // The keys' last tile: only the 16-key steps that hold cached rows are
                    // issued, and the rest of the last such step is cleared (its weights
                    // are 0, but the rows may hold anything, and 0 x NaN is NaN; both
                    // issuers clear them, each before its own products).
                    const int v = kv - (t0 + j) * kTile;
                    if (v >= kTile) {
                        if (!SEP) {
                            if (!wait(&bars.p_full[h][0], tile - 1)) break;
                            tc::fence_after_sync();
                            tc::mma4_ts_sw128(d_o, d_p, b, id_pv, j > 0);
                        }
                        if (!wait(&bars.p_full[h][1], tile - 1)) break;
                        tc::fence_after_sync();
                        if (SEP) tc::mma4_ts_sw128(d_o, d_p, b, id_pv, j > 0);
                        tc::mma4_ts_sw128(d_o, d_p + 32, b + 4 * 128, id_pv, 1);
                    } else {
                        const int v16 = (v + 15) / 16 * 16;
                        const uint32_t v_s = ring + vp.slot * KA * kAtom;
                        for (int x = lane; x < (v16 - v) * 8 * KA; x += 32) {
                            const int k = x / ((v16 - v) * 8), y = x - k * (v16 - v) * 8;
                            asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(v_s + k * kAtom + (v + y / 8) * 128 + (y % 8) * 16),
                                         "r"(0)
                                         : "memory");
                        }
                        tc::fence_proxy_async_smem();
                        __syncwarp();
                        if ((!SEP && !wait(&bars.p_full[h][0], tile - 1)) || !wait(&bars.p_full[h][1], tile - 1)) break;
                        tc::fence_after_sync();
                        for (int k = 0; k < v16 / 16; ++k) tc::mma_ts_sw128(d_o, d_p + 8 * k, b + k * 128, id_pv, j > 0 || k > 0);
                    }
                    if (SEP || last) tc::commit_elect(pv_done);  // (else the next S is full after it)
                    if (!SEP) {
                        if (!last)
                            qk(q, kp, false);
                        else
                            look();
                    }
                    vp.advance();
                    vp.advance();
                }
                for (int j = nh; j < n && ok; ++j) {
                    const RingPos<NS> k_at = base.plus(2 * j), v_at = base.plus(2 * j + 1);
                    if (!wait(&bars.full[k_at.slot], k_at.round)) break;
                    give_back(&bars.empty[k_at.slot]);
                    if (!wait(&bars.full[v_at.slot], v_at.round)) break;
                    give_back(&bars.empty[v_at.slot]);
                }
                pieces += nh > 0;
                base = after;
            }
            // every MMA has completed before TMEM goes
            tc::commit_elect(smem_u32(&bars.drain[h]));
            if (!wait_warp(smem_u32(&bars.drain[h]), 0)) ok = false;
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kMoreRegs));
        const int h = (warp - kSoftmax) >> 2, quarter = warp & 3, row = quarter * 32 + lane;
        const uint32_t lanes = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
        const uint32_t s_t = lanes + kS + h * 128, p_t = lanes + kP + h * kPStep, o_t = lanes + kO + h * D;
        const int rt = row / a.hpg, hh = row - rt * a.hpg, in = h * a.tpt + rt;
        const uint64_t scale = pack2(a.scale_log2, a.scale_log2);
        auto arrive = [&](uint64_t *bar) {
            // (a predicate, not a branch)
            asm volatile("{\n .reg .pred p;\n setp.eq.u32 p, %1, 0;\n @p mbarrier.arrive.shared::cta.b64 _, [%0];\n}\n"
                         ::"r"(smem_u32(bar)), "r"(lane)
                         : "memory");
        };
        int tile = 0, pieces = 0, step = 0, outs = 0, frees = 0;  // this half's tiles and pieces, both halves' turns, stores
        RingPos<NS> rp{0, 0};
        // The two halves' warps of a quarter of the SM share its exponential unit: they
        // take turns, so that one loads, compares and stores, and has its products made,
        // while the other's exponentials run.  (Left alone they run in step, and all of
        // that waits for one another: 8191 tokens at width 128 344 us, 295 so.)
        // (the first half's first turn is the phase before a barrier's first)
        auto my_turn = [&](uint32_t done) { return all(done) || wait(&bars.turn[h][quarter], step - (h == 0)); };
        auto look_turn = [&] { return looked(&bars.turn[h][quarter], step - (h == 0)); };
        uint32_t s_done = 0;
        for (int idx = 0; ok; ++idx) {
            const Piece &sp = piece_at(idx);
            if (!ok) break;
            const int u = own(sp.u), n0 = own(sp.n0), n1 = own(sp.n1), t0 = own(sp.t0), slot = own(sp.slot);
            const bool real = rt < a.tpt && in < sp.ntok;
            // (a row that is none masks nothing and never asks for another base: its
            // warp would go those ways on every tile)
            const int pos = real ? sp.pos + in : INT_MAX;
            const int tok = own(sp.tok), ntok = own(sp.ntok), g = own(sp.g);
            const int64_t t = tok + in;
            taken(idx);
            if (u < 0) break;
            const int n = max(n0, n1), nh = h ? n1 : n0;
            float m = real ? -INFINITY : INFINITY, l = 0.f;  // base (log2 domain) and sum
            int v_at = 0;  // V(j - 1)
            for (int j = 0; j < n; ++j, ++step) {
                const int k_at = rp.slot, v_old = v_at;
                rp.advance();
                if (j < nh) v_at = rp.slot;
                rp.advance();
                if (j >= nh) {  // a tile that only the other half uses
                    if (!my_turn(look_turn())) break;
                    arrive(&bars.turn[1 - h][quarter]);
                    continue;
                }
                if (!(SEP && all(s_done)) && !wait(&bars.s_full[h], tile)) break;
                ++tile;
                tc::fence_after_sync();
                uint32_t s[kTile];
#pragma unroll
                for (int c = 0; c < kTile; c += 32) tc::ld_32x32b_x32(s_t + c, s + c);
                arrive(&bars.empty[k_at]);
                if (!SEP && j > 0) arrive(&bars.empty[v_old]);  // (S(j) was made behind the products of V(j - 1))
                if (SEP && j + 1 == nh) arrive(&bars.q_free[pieces % NQ][h]);
#pragma unroll
                for (int c = 0; c < kTile; c += 32) tc::wait_ld_x32(s + c);
                if (SEP) {
                    tc::fence_before_sync();
                    __syncwarp();
                    arrive(&bars.s_free[h]);
                }
                const uint32_t turn = look_turn();
                const int lim = pos - (t0 + j) * kTile;  // last visible column
                if (__any_sync(0xffffffffu, lim < kTile - 1)) {
#pragma unroll
                    for (int c = 0; c < kTile; ++c) s[c] = c <= lim ? s[c] : 0xff800000u;
                }
                const float top = max3(max32(s), max32(s + 32), fmaxf(max32(s + 64), max32(s + 96))) * a.scale_log2;
                // The base is the maximum of the first tile, raised later only when a
                // score passes it by 2^8: fp32 and bf16 have the room, and relative
                // roundings are the same at any base.
                const uint32_t pv = SEP && j > 0 ? looked(&bars.pv_done[h], tile - 2) : 0;
                const bool up = top > m + (j == 0 ? 0.f : 8.f);
                if (__any_sync(0xffffffffu, up)) {
                    const float alpha = up ? ex2(m - top) : 1.f;  // (0 from a base of -inf)
                    m = up ? top : m;
                    l *= alpha;
                    if (j > 0) {
                        if (SEP) {
                            if (!wait(&bars.pv_done[h], tile - 2)) break;
                            tc::fence_after_sync();
                        }
#pragma unroll
                        for (int c = 0; c < D; c += 16) {
                            uint32_t o[16];
                            tc::ld_32x32b_x16(o_t + c, o);
                            tc::wait_ld();
#pragma unroll
                            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
                            tc::st_32x32b_x16(o_t + c, o);
                        }
                    }
                }
                if (SEP && j > 0) {  // P(j - 1) has been read
                    if (!all(pv) && !wait(&bars.pv_done[h], tile - 2)) break;
                    arrive(&bars.empty[v_old]);
                }
                const float nm = m == -INFINITY ? 0.f : -m;
                const uint64_t base = pack2(nm, nm);
                uint64_t sum[2] = {0, 0};
                // 32 keys' weights, their sums added, into TMEM
                auto weigh = [&](int c0) {
                    uint32_t p[16];
#pragma unroll
                    for (int c = 0; c < 32; c += 2) {
                        float x, y;
                        unpack2(fma2(pack2(__uint_as_float(s[c0 + c]), __uint_as_float(s[c0 + c + 1])), scale, base), x, y);
                        x = ex2(x);
                        y = ex2(y);
                        sum[(c >> 1) & 1] = add2(sum[(c >> 1) & 1], pack2(x, y));
                        p[c >> 1] = pack_bf16(x, y);
                    }
                    tc::st_32x32b_x16(p_t + c0 / 2, p);
                };
                auto publish = [&](int half) {
                    tc::wait_st();
                    tc::fence_before_sync();
                    __syncwarp();
                    arrive(&bars.p_full[h][half]);
                };
                if (!my_turn(turn)) break;
                weigh(0);
                weigh(32);
                if (!SEP) publish(0);  // (D = 64: nothing waits for the first half's products)
                weigh(64);
                arrive(&bars.turn[1 - h][quarter]);
                if (SEP) s_done = looked(&bars.s_full[h], tile);
                weigh(96);
                publish(1);
                float x, y;
                unpack2(add2(sum[0], sum[1]), x, y);
                l += x + y;
            }
            if (!ok) break;
            // ---- the rows
            // A row of an item's piece may see none of its keys, one of a whole item sees
            // none before position 0: 0.  What else has no sum, or NaN for one, shows.
            const bool none = l == 0.f && (slot >= 0 || pos < 0);
            const float inv = none ? 0.f : 1.f / l;
            const float lse = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
            const int64_t at = (t * a.groups + g) * a.hpg + hh;
            const int part_row = (slot * 2 + h) * kTile;
            if (real && slot >= 0) a.lse_part[part_row + row] = lse;
            if (real && slot < 0 && a.lse) a.lse[at] = lse;
            const bool part = slot >= 0 && nh > 0, whole = slot < 0 && nh > 0 && ntok >= (h + 1) * a.tpt;
            // Through shared memory and out by TMA, 128 bytes of every row at a time:
            // stored from here, each lane its row, they hold up everything else on the
            // SM that uses shared memory (two halves of 128 x 128: 3300 cycles).  D = 128
            // has no room for that but where this half's queries were.  Rolled up: code
            // that runs once an item comes from far away (unrolled, 5000 cycles).
            const int chunks = part || slot < 0 ? D / 32 : 0;
            auto let_go = [&] {
                if (quarter == 0 && lane == 0) {
                    tc::bulk_wait_read0();
                    tc::mbar_arrive(smem_u32(&bars.out_free[h]));
                }
                __syncwarp();
            };
            // (D = 64: the last item's store has long read its buffer)
            if (SEP && (part || whole) && outs > 0) let_go();
            if (nh > 0) {
                if (!wait(&bars.pv_done[h], SEP ? tile - 1 : pieces)) break;
                tc::fence_after_sync();
                arrive(&bars.empty[v_at]);
            }
#pragma unroll 1
            for (int c = 0; c < chunks; ++c) {
                uint32_t o[32];
                if (nh > 0) {
                    tc::ld_32x32b_x32(o_t + 32 * c, o);
                    tc::wait_ld_x32(o);
                } else {
#pragma unroll
                    for (int e = 0; e < 32; ++e) o[e] = 0;
                }
                if (c + 1 == chunks && nh > 0) {
                    tc::fence_before_sync();
                    __syncwarp();
                    arrive(&bars.o_free[h]);
                }
#pragma unroll
                for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * inv);
                uint32_t w[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) w[e] = pack_bf16(__uint_as_float(o[2 * e]), __uint_as_float(o[2 * e + 1]));
                if (!part && !whole) {  // a half that the sequence's end cuts short (or that saw no key): its rows one by one
                    if (real) {
                        uint4 *dst = reinterpret_cast<uint4 *>(a.o + at * D + 32 * c);
#pragma unroll
                        for (int e = 0; e < 4; ++e) dst[e] = make_uint4(w[4 * e], w[4 * e + 1], w[4 * e + 2], w[4 * e + 3]);
                    }
                    continue;
                }
                // 128 bytes a row: one chunk of fp32, two of bf16
                const int box = part ? c : c >> 1, sub = part ? 0 : (c & 1) * 4;
                const uint32_t buf = stage + (SEP ? h : 2 * h + (box & 1)) * kAtom, out = buf + row * 128;
                if (sub == 0 && (SEP ? outs > 0 : box >= 2)) {  // what was there has left
                    if (!SEP || c > 0) let_go();
                    if (!wait(&bars.out_free[h], frees++)) break;
                }
                auto put = [&](int i, uint32_t x, uint32_t y, uint32_t z, uint32_t u) {
                    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(out + ((i ^ (row & 7)) << 4)), "r"(x), "r"(y),
                                 "r"(z), "r"(u)
                                 : "memory");
                };
                if (part) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) put(i, o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) put(sub + i, w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
                    if (sub == 0) continue;
                }
                tc::fence_proxy_async_smem();
                __syncwarp();
                arrive(&bars.out_ready[h][outs & 1]);
                if (quarter == 0) {
                    if (!wait(&bars.out_ready[h][outs & 1], outs >> 1)) break;
                    if (lane == 0) {
                        if (part)
                            tc::tma_store_3d(&map_part, buf, 32 * c, part_row, 0);
                        else
                            tc::tma_store_3d(&map_o, buf, 64 * box, g * a.hpg, tok + h * a.tpt);
                        tc::bulk_commit();
                    }
                    __syncwarp();
                }
                ++outs;
            }
            if (nh > 0) {
                if (!SEP && quarter == 0 && lane == 0) {  // the next queries may come
                    tc::bulk_wait_read0();
                    tc::mbar_arrive(smem_u32(&bars.q_free[0][h]));
                }
                __syncwarp();
                ++pieces;
            }
        }
        if (quarter == 0 && lane == 0) tc::bulk_wait0();
        __syncwarp();
    }
    // A wait that runs out ends its warp's work, and with it the other warps', by
    // waits of their own that run out.
    if (!ok && lane == 0) record_status(a.status, kStatusTimeout);
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    if (warp == kIssuer) tc::tmem_dealloc(tmem, 512);
}

// The partials of the items that were cut, joined: block (partition, rows).  The
// partition in which a cut item begins takes its pieces, its own and those of the
// partitions after it: weights e^(lse - max) over their sum.  A thread takes 16
// columns of a row, D / 16 threads a row: with 4 columns each, what every thread
// finds out about its row anew was most of the work (2400 tokens behind long
// prefixes, 14 MB of partials: 8.5 us, 5 so).
constexpr int kJoinThreads = 256;
template <int D>
constexpr int kJoinRows = kJoinThreads / (D / 16);
template <int D>
__global__ void __launch_bounds__(kJoinThreads) prompt_join_kernel(const __grid_constant__ Args a)
{
    constexpr int TPR = D / 16;
    griddep_wait();
    griddep_launch_dependents();
    const int part = blockIdx.x;
    const Cut cut = a.cuts[part];
    if (cut.last < 0) return;
    const int r = blockIdx.y * kJoinRows<D> + threadIdx.x / TPR, c = threadIdx.x % TPR * 4;  // columns c + 4 TPR i
    const int h = r / kTile, row = r % kTile, rt = row / a.hpg, in = h * a.tpt + rt;
    if (rt >= a.tpt || in >= cut.ntok) return;
    float m = -INFINITY, w = 0.f, acc[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] = 0.f;
    for (int q = part; q <= cut.last; ++q) {
        const int64_t at = static_cast<int64_t>(q == part ? 2 * q + 1 : 2 * q) * 2 * kTile + r;
        const float s = a.lse_part[at];
        float4 v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const float4 *>(a.o_part + at * D + c + 4 * TPR * i);
        // a partition that begins and ends in one tile wrote nothing, nor did a piece of
        // which this row sees no key: whatever was there is not looked at
        if ((q > part && !a.cuts[q].goes_on) || s == -INFINITY) continue;
        const float top = fmaxf(m, s), f = ex2((m - top) * 1.4426950408889634f), e = ex2((s - top) * 1.4426950408889634f);
        m = top;
        w = w * f + e;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            acc[4 * i] = acc[4 * i] * f + e * v[i].x;
            acc[4 * i + 1] = acc[4 * i + 1] * f + e * v[i].y;
            acc[4 * i + 2] = acc[4 * i + 2] * f + e * v[i].z;
            acc[4 * i + 3] = acc[4 * i + 3] * f + e * v[i].w;
        }
    }
    const int64_t at = (static_cast<int64_t>(cut.tok + in) * a.groups + cut.g) * a.hpg + row % a.hpg;
    const float inv = w == 0.f && cut.pos + in < 0 ? 0.f : 1.f / w;  // (no key before position 0)
#pragma unroll
    for (int i = 0; i < 4; ++i)
        *reinterpret_cast<uint2 *>(a.o + at * D + c + 4 * TPR * i) =
            make_uint2(pack_bf16(acc[4 * i] * inv, acc[4 * i + 1] * inv), pack_bf16(acc[4 * i + 2] * inv, acc[4 * i + 3] * inv));
    if (a.lse && c == 0) a.lse[at] = w == 0.f ? -INFINITY : m + log2f(w) * 0.69314718055994531f;
}

PFN_cuTensorMapEncodeTiled_v12000 encoder()
{
    static const PFN_cuTensorMapEncodeTiled_v12000 fn = [] {
        cudaDriverEntryPointQueryResult q;
        void *p = nullptr;
        const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q);
        return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(e == cudaSuccess && q == cudaDriverEntryPointSuccess ? p : nullptr);
    }();
    return fn;
}

// Boxes of `box` columns (128 bytes: 64 of bf16, 32 of fp32) x r1 x r2 of a
// tensor [d2][d1][cols] with element strides s2, s1, 1.
cudaError_t encode(CUtensorMap *m, const void *base, int cols, int64_t d1, int64_t s1, int64_t d2, int64_t s2, int r1, int r2,
                   int box = 64)
{
    const auto fn = encoder();
    if (!fn) return cudaErrorNotSupported;
    const int bytes = 128 / box;
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(d1), static_cast<cuuint64_t>(d2)};
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(s1) * bytes, static_cast<cuuint64_t>(s2) * bytes};
    const cuuint32_t boxes[3] = {static_cast<cuuint32_t>(box), static_cast<cuuint32_t>(r1), static_cast<cuuint32_t>(r2)}, es[3] = {1, 1, 1};
    const CUresult r = fn(m, bytes == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3,
                          const_cast<void *>(base), dims, strides, boxes, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

// The most items of a call (the sequences' lengths are on the device), and
// whether any can have tiles enough to be cut.
int64_t most_items(int batch, int total, int groups, int hpg)
{
    return (static_cast<int64_t>(total) / (2 * (kTile / hpg)) + (batch < total ? batch : total)) * groups;
}
bool may_cut(int max_kv) { return (max_kv + kTile - 1) / kTile >= 2 * kLeastTiles; }

template <int D>
cudaError_t launch_d(const PromptAttn &p, cudaStream_t st)
{
    const CacheView &c = p.cache;
    const bool paged = c.block_table != nullptr;
    const int tpb = paged ? c.page_size : c.capacity, rows = paged ? kPage : kTile;
    const int64_t blocks = paged ? c.num_pages : static_cast<int64_t>(p.batch) * p.groups;
    Args a;
    a.batch = p.batch;
    a.total = p.total;
    a.groups = p.groups;
    a.hpg = p.hpg;
    a.max_kv = p.max_kv;
    a.parts = p.num_splits;
    a.tpt = kTile / p.hpg;
    a.item = kItemUnits<D>;
    a.cut = a.parts > 1 && may_cut(p.max_kv);
    a.paged = paged;
    a.bt_stride = c.bt_stride;
    a.num_pages = c.num_pages;
    a.scale_log2 = p.sm_scale * 1.4426950408889634f;
    a.cu = p.cu;
    a.kv_len = p.kv_len;
    a.block_table = c.block_table;
    a.o = static_cast<uint16_t *>(p.o);
    a.lse = p.lse;
    a.o_part = p.o_part;
    a.lse_part = p.lse_part;
    a.cuts = reinterpret_cast<Cut *>(p.lse_part + static_cast<size_t>(a.parts) * 4 * kTile);
    a.status = p.status;
    CUtensorMap mq, mk, mv, mo, mp;
    cudaError_t e;
    if ((e = encode(&mq, p.q, D, p.groups * p.hpg, D, p.total, p.q_stride, p.hpg, a.tpt)) != cudaSuccess) return e;
    if ((e = encode(&mk, c.k_rope, D, tpb, c.r_tok, blocks, c.r_blk, rows, 1)) != cudaSuccess) return e;
    if ((e = encode(&mv, c.c_kv, D, tpb, c.c_tok, blocks, c.c_blk, rows, 1)) != cudaSuccess) return e;
    const int heads = p.groups * p.hpg;
    if ((e = encode(&mo, p.o, D, heads, D, p.total, static_cast<int64_t>(heads) * D, p.hpg, a.tpt)) != cudaSuccess) return e;
    // partials: 32 fp32 columns of a half's rows
    mp = mo;
    if (a.cut && (e = encode(&mp, p.o_part, D, static_cast<int64_t>(a.parts) * 4 * kTile, D, 1, static_cast<int64_t>(a.parts) * 4 * kTile * D,
                             kTile, 1, 32)) != cudaSuccess)
        return e;
    if ((e = allow_smem<prompt_attn_kernel<D>>(kSmem<D>)) != cudaSuccess) return e;
    if ((e = launch_dependent(prompt_attn_kernel<D>, dim3(a.parts), dim3(kThreads), kSmem<D>, st, 1, a, mq, mk, mv, mo, mp)) != cudaSuccess)
        return e;
    if (!a.cut) return cudaSuccess;
    return launch_dependent(prompt_join_kernel<D>, dim3(a.parts, 2 * kTile / kJoinRows<D>), dim3(kJoinThreads), 0, st, 1, a);
}

}  // namespace

int prompt_splits(int batch, int total, int groups, int hpg, int max_kv, int sms)
{
    // one a SM, as far as there are pieces for them
    const int64_t pieces = most_items(batch, total, groups, hpg) * (1 + max_kv / (kLeastTiles * kTile));
    return pieces < 1 ? 1 : pieces < sms ? static_cast<int>(pieces) : sms;
}

size_t prompt_part_rows(int batch, int total, int groups, int hpg, int max_kv, int requested, int sms)
{
    const int most = requested > 0 ? requested : prompt_splits(batch, total, groups, hpg, max_kv, sms);
    return most > 1 && may_cut(max_kv) ? static_cast<size_t>(most) * kPromptPartRows : 0;
}

cudaError_t launch_prompt_attn(const PromptAttn &p, cudaStream_t st)
{
    if (p.head_dim == 64) return launch_d<64>(p, st);
    if (p.head_dim == 128) return launch_d<128>(p, st);
    return cudaErrorInvalidConfiguration;
}

}  // namespace gbmla
