// mla_token_logprobs: log probability of a given token, entropy, log-sum-exp and
// the likeliest alternatives of each row of logits, in one pass over them.
//
// A row goes to one CTA or to a cluster of 2 or 4, each a slice of its vocabulary.
// A thread keeps, over its vectors of 16 bytes, the maximum m and, over a base b
// that follows it loosely, S = sum 2^((x - b) log2 e) and T = the same sum with
// each term times x - b (which is finite where its product with log2 e is not);
// merged over the row,
//     lse = m + ln S,  entropy = ln S - T / S,  log p(y) = x_y - m - ln S.
// The alternatives need no second pass: the threads' maxima give a value that at
// least n_top logits of the slice reach.  A thread knows its best groups of
// vectors; those that reach that value are looked at again (a hundred of 4000) and
// what reaches it is put by, as keys (value, falling index), in shared memory and
// ranked; rank 0 merges the slices'.  Where more reach it than there is room for
// (plateaus), the slice is gone over in pieces, each merged into the best so far.
// (A filter within the pass, by a threshold from its beginning, let 800 of 128 256
// logits through, one for almost every vector that a warp looks at, and with that
// 640 rows took 105 us in place of 66.)
//
// Bound: memory, once the rows fill the SMs (912 rows of 128256 bf16 logits: 46 us
// or 5.0 TB/s with 20 alternatives; 640 rows, which are 1.4 waves, 39 us with them
// and 31 us without), then what a row costs in turn (reductions, barriers, the
// ranking: 2 us of which the next row's first loads hide a part; the whole next row
// prefetched into L2 meanwhile takes more from the rows under way: 912 rows 54 us).
// A few rows are bound by that latency: 5.7 us for 3 rows of 32000.  Issue is next
// (about five instructions a bf16 logit: unpacking, maximum, exponent, exponential
// and two sums, two-wide where that exists).
#include <math.h>

#include "common.cuh"
#include "internal.h"
#include "tc.cuh"

namespace gbmla {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kCtas = 3;                    // per SM
constexpr int kUnroll = 4;                  // vectors a thread loads together
constexpr int kMaxCluster = 4;
constexpr int kKeys = 4096;                 // keys put by in a slice
constexpr int kGroups = 2048;               // groups of vectors that are looked at again
constexpr int kRank = 512;                  // keys that are ranked one against the other
constexpr int kPiece = 2048;                // logits of a piece, where those do not do
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kMasked = -2e9f;            // logits at or below weigh nothing
constexpr float kFloor = -1e30f;            // what lower ones are raised to: 2^-inf would be 0, but 0 x inf is not
constexpr float kRaise = 16.f;              // a base is raised once a logit passes it by this much
static_assert(kKeys >= kPiece + kMaxTop, "a piece and the best so far");

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint64_t pk(float lo, float hi)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void upk(uint64_t v, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b)
{
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b)
{
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}

// Keys in the order of falling logits and rising indices (larger first; 0: none).
__device__ __forceinline__ uint64_t key_of(float x, int idx)
{
    uint32_t b = __float_as_uint(x + 0.f);  // (-0 is 0)
    b = b & 0x80000000u ? ~b : b | 0x80000000u;
    return static_cast<uint64_t>(b) << 32 | static_cast<uint32_t>(~idx);
}
__device__ __forceinline__ int index_of(uint64_t key) { return static_cast<int>(~static_cast<uint32_t>(key)); }
__device__ __forceinline__ float value_of(uint64_t key)
{
    const uint32_t b = static_cast<uint32_t>(key >> 32);
    return __uint_as_float(b & 0x80000000u ? b & 0x7fffffffu : ~b);
}
// fp32 values in the order of unsigned integers.
__device__ __forceinline__ uint32_t order_of(float x)
{
    const uint32_t b = __float_as_uint(x);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// A 16-byte vector of logits.
template <typename T>
struct Vec;
template <>
struct Vec<float> {
    static constexpr int n = 4;
    static constexpr uint32_t kNone = 0xff800000u;  // -inf
    __device__ static float one(const float *p) { return *p; }
    __device__ static uint4 lone(const float *p) { return make_uint4(__float_as_uint(*p), kNone, kNone, kNone); }
    __device__ static float at(const uint4 &v, int e) { return __uint_as_float(e == 0 ? v.x : e == 1 ? v.y : e == 2 ? v.z : v.w); }
    __device__ static float max(const uint4 &v)
    {
        return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
    }
    __device__ static float max4(const uint4 &a, const uint4 &b, const uint4 &c, const uint4 &d)
    {
        return fmaxf(fmaxf(max(a), max(b)), fmaxf(max(c), max(d)));
    }
    // (NaN stays)
    __device__ static float raise(uint32_t x)
    {
        float y;
        asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(__uint_as_float(x)), "f"(kFloor));
        return y;
    }
    __device__ static void pairs(const uint4 &v, uint64_t (&p)[2])
    {
        p[0] = pk(raise(v.x), raise(v.y));
        p[1] = pk(raise(v.z), raise(v.w));
    }
};
template <>
struct Vec<uint16_t> {
    static constexpr int n = 8;
    static constexpr uint32_t kNone = 0xff80ff80u;
    __device__ static float one(const uint16_t *p) { return bf16_bits_to_float(*p); }
    __device__ static uint4 lone(const uint16_t *p) { return make_uint4(0xff800000u | *p, kNone, kNone, kNone); }
    __device__ static float at(const uint4 &v, int e)
    {
        const uint32_t w = e < 2 ? v.x : e < 4 ? v.y : e < 6 ? v.z : v.w;
        return __uint_as_float(e & 1 ? w & 0xffff0000u : w << 16);
    }
    __device__ static uint32_t max2(uint32_t a, uint32_t b)
    {
        uint32_t r;
        asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    __device__ static float max(const uint4 &v)
    {
        const uint32_t w = max2(max2(v.x, v.y), max2(v.z, v.w));
        return fmaxf(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    }
    __device__ static float max4(const uint4 &a, const uint4 &b, const uint4 &c, const uint4 &d)
    {
        const uint32_t x = max2(max2(a.x, a.y), max2(a.z, a.w)), y = max2(max2(b.x, b.y), max2(b.z, b.w));
        const uint32_t z = max2(max2(c.x, c.y), max2(c.z, c.w)), u = max2(max2(d.x, d.y), max2(d.z, d.w));
        const uint32_t w = max2(max2(x, y), max2(z, u));
        return fmaxf(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    }
    __device__ static uint64_t pair(uint32_t w)
    {
        asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(w) : "r"(0xf14af14au));  // -1.0e30
        return pk(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    }
    __device__ static void pairs(const uint4 &v, uint64_t (&p)[4])
    {
        p[0] = pair(v.x);
        p[1] = pair(v.y);
        p[2] = pair(v.z);
        p[3] = pair(v.w);
    }
};

// Statistics of some logits: the maximum, and over the base b the sums of 2^y and
// of 2^y (x - b), y = (x - b) log2 e.  (The difference first: x log2 e - b log2 e in one
// FMA saves an instruction a pair, but leaves the rounding of b log2 e in y, 64 for
// logits of -1e9, and a lone token's probability is then not 1.)
struct Stat {
    float m, b, s, t;
};
// The same over another base.
__device__ __forceinline__ void rebase(Stat &a, float b)
{
    const float d = a.b - b, f = ex2(d * kLog2e);
    // (what weighs nothing any more may be large: no 0 x inf; but a sum that is NaN stays so)
    a.t = f > 0.f ? f * (a.t + d * a.s) : 0.f;
    a.s = f > 0.f ? f * a.s : a.s - a.s;
    a.b = b;
}
__device__ __forceinline__ Stat merged(Stat a, Stat c)
{
    const float m = fmaxf(a.m, c.m), b = fmaxf(m, kMasked);
    rebase(a, b);
    rebase(c, b);
    return {m, b, a.s + c.s, a.t + c.t};
}

// Over groups of 2 w lanes; every lane has the result, by the same sums.
__device__ __forceinline__ Stat merged_lanes(Stat r, int w)
{
    const int lane = threadIdx.x & 31;
    for (int o = w; o > 0; o >>= 1) {
        Stat q;
        q.m = __shfl_xor_sync(0xffffffffu, r.m, o);
        q.b = __shfl_xor_sync(0xffffffffu, r.b, o);
        q.s = __shfl_xor_sync(0xffffffffu, r.s, o);
        q.t = __shfl_xor_sync(0xffffffffu, r.t, o);
        r = lane & o ? merged(q, r) : merged(r, q);
    }
    return r;
}

// A thread's running statistics: the sums two-wide; the maxima of its three best
// groups of vectors, and where the first two of them are.
struct Run {
    float m, b, m1, m2;
    int at0, at1;
    uint64_t s, t;
};

// A group of the thread's vectors, which begins at vector at.
template <typename T, bool kRank, int N>
__device__ __forceinline__ void take(Run &r, const uint4 (&v)[N], int at)
{
    static_assert(N == 2 || N == 4);
    float m;
    if constexpr (N == 4)
        m = Vec<T>::max4(v[0], v[1], v[2], v[3]);
    else
        m = fmaxf(Vec<T>::max(v[0]), Vec<T>::max(v[1]));
    if (kRank) {
        r.m2 = fmaxf(r.m2, fminf(r.m1, m));
        const bool over = m > r.m, next = m > r.m1;
        r.at1 = over ? r.at0 : next ? at : r.at1;
        r.m1 = over ? r.m : next ? m : r.m1;
        r.at0 = over ? at : r.at0;
    }
    r.m = fmaxf(r.m, m);
    if (r.m > r.b + kRaise) {
        const float d = r.b - r.m, f = ex2(d * kLog2e);
        float s0, s1, t0, t1;
        upk(r.s, s0, s1);
        upk(r.t, t0, t1);
        // (what weighs nothing any more may be large: no 0 x inf; but a sum that is NaN stays so)
        r.t = f > 0.f ? pk(f * (t0 + d * s0), f * (t1 + d * s1)) : 0;
        r.s = f > 0.f ? pk(f * s0, f * s1) : pk(s0 - s0, s1 - s1);
        r.b = r.m;
    }
    const uint64_t L = pk(kLog2e, kLog2e), B = pk(-r.b, -r.b);
    constexpr int P = Vec<T>::n / 2;
#pragma unroll
    for (int u = 0; u < N; ++u) {
        uint64_t p[P];
        Vec<T>::pairs(v[u], p);
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const uint64_t d = add2(p[i], B);
            float a, b;
            upk(mul2(d, L), a, b);
            const uint64_t e = pk(ex2(a), ex2(b));
            r.s = add2(r.s, e);
            r.t = fma2(e, d, r.t);
        }
    }
}

struct Shared {
    uint64_t keys[kKeys];                        // what was put by, then the slice's best
    uint64_t best[kMaxTop];                      // the best so far, in order
    uint64_t all[2][kMaxCluster * kMaxTop];      // rank 0: every slice's k best (by row parity)
    Stat stats[2][kMaxCluster];                  // rank 0: every slice's statistics
    Stat warp_stats[kWarps];
    uint32_t hist[256];
    uint32_t floor[kWarps];
    int reach[kGroups];                          // groups of vectors whose maximum reaches far enough
    int groups, n;                               // how many; keys put by (they may be more than there is room for)
    int bin, need, in_bin;
};

// The k largest of keys[0 .. n), n <= kRank, in order, into best (0: none): each
// key's place is the number of larger ones.  (Two hundred keys: well below a
// microsecond; selecting them digit by digit, as below, takes 7.)  All threads.
__device__ void rank_best(const uint64_t *keys, int n, uint64_t *best, int k)
{
    const int tid = threadIdx.x;
    if (tid < kMaxTop) best[tid] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += kThreads) {
        const uint64_t key = keys[i];
        int above = 0;
#pragma unroll 8
        for (int j = 0; j < n; ++j) above += keys[j] > key;
        if (above < k && key) best[above] = key;
    }
    __syncthreads();
}

// The same of any number of sh.keys: one digit of 8 bits after the other.  All threads.
__device__ __noinline__ void select_best(Shared &sh, int n, int k)
{
    const int tid = threadIdx.x, lane = tid & 31;
    uint64_t prefix = 0, mask = 0;
    int need = k;
    for (int shift = 56; n > k && shift >= 0; shift -= 8) {
        sh.hist[tid] = 0;
        __syncthreads();
        for (int i = tid; i < n; i += kThreads)
            if ((sh.keys[i] & mask) == prefix) atomicAdd(&sh.hist[(sh.keys[i] >> shift) & 255], 1);
        __syncthreads();
        if (tid < 32) {  // lane l: the bins 255 - 8 l and down
            int c = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) c += sh.hist[255 - 8 * lane - i];
            int incl = c;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int x = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += x;
            }
            int before = incl - c;
            if (before < need && incl >= need) {
                for (int i = 0; i < 8; ++i) {
                    const int bin = 255 - 8 * lane - i, h = sh.hist[bin];
                    if (before + h >= need) {
                        sh.bin = bin;
                        sh.need = need - before;
                        sh.in_bin = h;
                        break;
                    }
                    before += h;
                }
            }
        }
        __syncthreads();
        prefix |= static_cast<uint64_t>(sh.bin) << shift;
        mask |= uint64_t{255} << shift;
        need = sh.need;
        if (sh.in_bin == need) break;  // all of the bin's
    }
    __syncthreads();
    if (tid == 0) sh.bin = 0;
    if (tid < kMaxTop) sh.best[tid] = 0;
    __syncthreads();
    // the k keys at or above the prefix into the histogram's place, then in order
    uint64_t *chosen = reinterpret_cast<uint64_t *>(sh.hist);
    for (int i = tid; i < n; i += kThreads) {
        const uint64_t key = sh.keys[i];
        if ((key & mask) >= prefix) chosen[atomicAdd(&sh.bin, 1)] = key;
    }
    __syncthreads();
    if (tid < 32) {
        const int got = min(n, k);
        const uint64_t key = lane < got ? chosen[lane] : 0;
        int above = 0;
#pragma unroll
        for (int l = 0; l < 32; ++l) above += __shfl_sync(0xffffffffu, key, l) > key;
        if (lane < got) sh.best[above] = key;
    }
    __syncthreads();
}

__device__ __forceinline__ uint32_t map_rank(const void *p, int rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(p)), "r"(rank));
    return r;
}
__device__ __forceinline__ void st_cluster64(uint32_t addr, uint64_t v)
{
    asm volatile("st.shared::cluster.b64 [%0], %1;" ::"r"(addr), "l"(v) : "memory");
}

// A CTA's slice of a row: up to 16 bytes of alignment (rank 0), vectors, and a
// rest (the last rank).
template <typename T>
struct Slice {
    const T *x;
    const uint4 *v;    // the slice's vectors
    int head, tail;    // the row's first vector and what follows its last one, in logits
    int first, mine;   // the slice's first logit and its number of vectors
    __device__ __forceinline__ Slice(const Logprobs &a, int64_t row, int rank, int log_size)
    {
        constexpr int N = Vec<T>::n;
        x = static_cast<const T *>(a.logits) + row * a.stride;
        const int odd = static_cast<int>((reinterpret_cast<uintptr_t>(x) & 15) / sizeof(T));
        head = min(a.vocab, odd ? N - odd : 0);
        const int nvec = (a.vocab - head) / N, share = (nvec + (1 << log_size) - 1) >> log_size, lo = min(nvec, rank * share);
        tail = head + nvec * N;
        mine = min(nvec, lo + share) - lo;
        first = head + lo * N;
        v = reinterpret_cast<const uint4 *>(x + head) + lo;
    }
    // The thread's vectors of the group that begins at vector `from`.
    __device__ __forceinline__ void fetch(uint4 (&d)[kUnroll], int from) const
    {
        const uint4 none = make_uint4(Vec<T>::kNone, Vec<T>::kNone, Vec<T>::kNone, Vec<T>::kNone);
        const uint4 *p = v + from + threadIdx.x;
        if (from + kUnroll * kThreads <= mine) {
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) d[u] = p[u * kThreads];
        } else {
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) d[u] = from + u * kThreads + static_cast<int>(threadIdx.x) < mine ? p[u * kThreads] : none;
        }
    }
};

// kTop: with alternatives
template <typename T, bool kTop>
__global__ void __launch_bounds__(kThreads, kCtas) logprobs_kernel(const Logprobs a, int log_size, int alone)
{
    extern __shared__ __align__(16) unsigned char raw[];
    Shared &sh = *reinterpret_cast<Shared *>(raw);
    constexpr int VN = Vec<T>::n, U = kUnroll;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int size = 1 << log_size, own = blockIdx.x & (size - 1), k = a.n_top;
    griddep_wait();
    griddep_launch_dependents();
    const uint4 none = make_uint4(Vec<T>::kNone, Vec<T>::kNone, Vec<T>::kNone, Vec<T>::kNone);
    // the CTA's i-th row: its own ones, then those of its cluster (there are less
    // than 2^31 rows, so that unsigned ones do not overflow)
    const unsigned rows = static_cast<unsigned>(a.rows), clusters = gridDim.x >> log_size;
    const unsigned shared = alone * gridDim.x + (blockIdx.x >> log_size) - alone * clusters;
    auto row_of = [&](int i) { return i < alone ? i * gridDim.x + blockIdx.x : shared + i * clusters; };
    auto slice_of = [&](int i) { return Slice<T>(a, row_of(i), i < alone ? 0 : own, i < alone ? 0 : log_size); };
    Slice<T> next = slice_of(0);
    uint4 v[2][U];
    next.fetch(v[0], 0);
    int i_row = 0, par = 0;
    for (unsigned row; (row = row_of(i_row)) < rows; ++i_row, par ^= 1) {
        const int C = i_row < alone ? 1 : size, rank = i_row < alone ? 0 : own, to_cta = i_row < alone ? own : 0;
        if (C > 1 && i_row == alone) tc::cluster_arrive();  // (rank 0's room is free of its own rows' results)
        const Slice<T> at_row = next;
        const T *x = at_row.x;
        const uint4 *xv = at_row.v;
        const int head = at_row.head, tail = at_row.tail, first = at_row.first, mine = at_row.mine;
        int token = -1;
        float token_logit = 0.f;
        if (rank == 0 && tid == 0 && a.logprob) {
            token = a.tokens[row];
            if (token >= 0 && token < a.vocab)
                token_logit = Vec<T>::one(x + token);
            else if (token != -1)
                record_status(a.status, kStatusBounds);
        }
        if (tid == 0) sh.n = sh.groups = 0;
        // ---- the pass: groups of vectors, the next group's loads ahead
        Run run{-INFINITY, kMasked, -INFINITY, -INFINITY, 0, 0, 0, 0};
        // the logits before the first vector (rank 0) and behind the last (the last rank)
        const bool has_head = rank == 0 && tid < head, has_tail = rank == C - 1 && tid < a.vocab - tail;
        const uint4 ends[2] = {has_head ? Vec<T>::lone(x + tid) : none, has_tail ? Vec<T>::lone(x + tail + tid) : none};
        for (int at = 0; at < mine; at += 2 * U * kThreads) {
            if (at + U * kThreads < mine) at_row.fetch(v[1], at + U * kThreads);
            take<T, kTop>(run, v[0], at);
            if (at + U * kThreads >= mine) break;
            if (at + 2 * U * kThreads < mine) at_row.fetch(v[0], at + 2 * U * kThreads);
            take<T, kTop>(run, v[1], at + U * kThreads);
        }
        const Run body = run;
        if (has_head || has_tail) take<T, false>(run, ends, 0);
        // the next row's first group is under way while this one's results are put together
        if (row_of(i_row + 1) < rows) {
            next = slice_of(i_row + 1);
            next.fetch(v[0], 0);
        }
        Stat r{run.m, run.b, 0.f, 0.f};
        {
            float y0, y1;
            upk(run.s, y0, y1);
            r.s = y0 + y1;
            upk(run.t, y0, y1);
            r.t = y0 + y1;
        }
        // ---- who has logits that reach far enough: each warp's ceil(k / 8) largest of
        // its lanes' maxima, the smallest of them all; at least k logits reach it
        float least = -INFINITY;
        if (kTop) {
            uint32_t rest = order_of(run.m), top = 0;
            for (int i = 0; i < (k + kWarps - 1) / kWarps; ++i) {
                top = __reduce_max_sync(0xffffffffu, rest);
                const unsigned who = __ballot_sync(0xffffffffu, rest == top);
                if (lane == __ffs(who) - 1) rest = 0;
            }
            if (lane == 0) sh.floor[warp] = top;
            __syncthreads();
            uint32_t f = sh.floor[0];
#pragma unroll
            for (int i = 1; i < kWarps; ++i) f = min(f, sh.floor[i]);
            least = f & 0x80000000u ? __uint_as_float(f & 0x7fffffffu) : __uint_as_float(~f);
            if (!(least > -INFINITY)) least = -INFINITY;  // (a lane without a logit)
            // (the third best too: all of the thread's)
            auto reaches = [&](float m) { return m >= least && m > kMasked; };
            if (reaches(body.m)) {
                const bool all = reaches(body.m2);
                const int n = all ? (mine + U * kThreads - 1) / (U * kThreads) : reaches(body.m1) ? 2 : 1;
                const int to = atomicAdd(&sh.groups, n);
                for (int i = 0; i < n && to + i < kGroups; ++i)
                    sh.reach[to + i] = tid + (all ? i * U * kThreads : i ? body.at1 : body.at0);
            }
        }
        // ---- the slice's statistics
        r = merged_lanes(r, 16);
        if (lane == 0) sh.warp_stats[warp] = r;
        __syncthreads();
        // (rank 0 has begun with the cluster's rows, and has read what it had of the one before last)
        if (C > 1 && (rank != 0 || i_row == alone)) tc::cluster_wait();
        if (warp == kWarps - 1) {
            const Stat q = merged_lanes(sh.warp_stats[lane & (kWarps - 1)], kWarps / 2);
            if (lane == 0) {
                const uint32_t to = map_rank(&sh.stats[par][rank], to_cta);
                st_cluster64(to, pk(q.m, q.b));
                st_cluster64(to + 8, pk(q.s, q.t));
            }
        }
        // ---- the slice's alternatives
        if (kTop) {
            auto put = [&](const uint4 &w, int at, int n) {
                for (int e = 0; e < n; ++e) {
                    const float y = Vec<T>::at(w, e);
                    if (y >= least && y > kMasked) {
                        const int i = atomicAdd(&sh.n, 1);
                        if (i < kKeys) sh.keys[i] = key_of(y, at + e);
                    }
                }
            };
            const int looks = sh.groups <= kGroups ? sh.groups * U : 0;
            for (int i = tid; i < looks && sh.n <= kKeys; i += kThreads) {
                const int at = sh.reach[i / U] + i % U * kThreads;
                if (at < mine) {
                    const uint4 w = xv[at];
                    const float wm = Vec<T>::max(w);
                    if (wm >= least && wm > kMasked) put(w, first + at * VN, VN);
                }
            }
            if (has_head) put(ends[0], tid, 1);
            if (has_tail) put(ends[1], tail + tid, 1);
            __syncthreads();
            const int n = sh.n;
            __syncthreads();
            if (n <= kRank && sh.groups <= kGroups) {
                rank_best(sh.keys, n, sh.best, k);
            } else if (n <= kKeys && sh.groups <= kGroups) {
                select_best(sh, n, k);
            } else {
                // piece by piece: what passes the worst of the best so far, merged into them
                if (tid < kMaxTop) sh.best[tid] = 0;
                __syncthreads();
                // (unsigned: the last piece of the longest rows ends past 2^31)
                const unsigned end = first + mine * VN + (rank == C - 1 ? a.vocab - tail : 0), from = rank == 0 ? 0 : first;
                for (unsigned p0 = from; p0 < end; p0 += kPiece) {
                    const uint64_t worst = sh.best[k - 1];
                    const bool had = tid < k && sh.best[tid] != 0;
                    if (had) sh.keys[tid] = sh.best[tid];
                    const int held = __syncthreads_count(had);
                    if (tid == 0) sh.n = held;
                    __syncthreads();
                    for (unsigned i = p0 + tid; i < min(end, p0 + kPiece); i += kThreads) {
                        const float y = Vec<T>::one(x + i);
                        const uint64_t key = key_of(y, static_cast<int>(i));
                        if (y > kMasked && key > worst) sh.keys[atomicAdd(&sh.n, 1)] = key;
                    }
                    __syncthreads();
                    const int now = sh.n;
                    __syncthreads();
                    if (now > held) select_best(sh, now, k);
                }
            }
            if (tid < k) st_cluster64(map_rank(&sh.all[par][rank * k + tid], to_cta), sh.best[tid]);
        }
        // Every slice's results reach rank 0, which reads them before it arrives at the next
        // row's barrier (the row after that writes this set again).  The others go on: they
        // wait for this barrier where they next write.
        if (C > 1) {
            tc::cluster_arrive();
            if (rank != 0) {
                __syncthreads();  // (sh.best and the keys are this row's no more)
                continue;
            }
            tc::cluster_wait();
        } else {
            __syncthreads();
        }
        if (kTop && C > 1) rank_best(sh.all[par], C * k, sh.best, k);
        if (warp == 0) {
            Stat q = sh.stats[par][0];
            for (int c = 1; c < C; ++c) q = merged(q, sh.stats[par][c]);
            const bool bad = !(q.s - q.s == 0.f), empty = !(q.m > kMasked) && !bad;
            if (!empty && !bad) rebase(q, q.m);
            const float z = bad ? NAN : empty ? 0.f : logf(q.s);
            if (lane == 0) {
                if (a.lse) a.lse[row] = empty ? -INFINITY : q.m + z;
                if (a.entropy) a.entropy[row] = empty ? 0.f : z - q.t / q.s;
                if (a.logprob && (token == -1 || (token >= 0 && token < a.vocab)))
                    a.logprob[row] = token == -1 ? 0.f
                                     : bad       ? NAN
                                     : token_logit > kMasked ? token_logit - q.m - z
                                                             : -INFINITY;
            }
            if (lane < k) {
                const uint64_t key = sh.best[lane];
                if (a.top_index) a.top_index[static_cast<size_t>(row) * k + lane] = key ? index_of(key) : -1;
                if (a.top_logprob) a.top_logprob[static_cast<size_t>(row) * k + lane] = bad ? NAN : key ? value_of(key) - q.m - z : -INFINITY;
            }
        }
        __syncthreads();  // (sh.best and the keys are this row's no more)
    }
    if (own != 0 && i_row > alone) tc::cluster_wait();
}

template <typename T, bool kTop>
cudaError_t launch(const Logprobs &p, cudaStream_t st)
{
    // Every CTA takes as many rows alone as fill whole waves; what is left goes to
    // clusters, of the size whose CTAs finish first: waves times a slice's vectors and
    // what a row costs besides (more where slices are joined).  Measured, in us: 0.13 a
    // vector of all threads, 0.34 once most CTAs are busy; besides 2 with alternatives
    // (4.6 and 5.2 in clusters of 2 and 4), 1 without (2.3, 2.9).  At 128256 bf16 logits
    // and 20 alternatives 64 rows take 14.7, 13.5 and 11.9 us in clusters of 1, 2, 4,
    // 200 rows 20.3, 16.4 and 23.2 us, 456 rows 25.9, 31.0 and 66 us.
    const int64_t slots = static_cast<int64_t>(p.sms) * kCtas / kMaxCluster * kMaxCluster;
    const double vectors = static_cast<double>(p.vocab) / Vec<T>::n / kThreads;
    int best = 1, alone = 0;
    double least = 0;
    for (int c = 1; c <= kMaxCluster; c *= 2) {
        const int own = c > 1 ? static_cast<int>(p.rows / slots) : 0;
        const int64_t rest = p.rows - own * slots, at_once = slots / c;
        const double busy = rest < at_once ? static_cast<double>(rest) / at_once : 1.;
        const double rate = fmin(0.13 + 0.3 * busy, 0.34), fixed = (c == 1 ? 2. : c == 2 ? 4.6 : 5.2) * (kTop ? 1 : 0.55);
        const double cost = own * (vectors * 0.34 + (kTop ? 2. : 1.)) + (rest + at_once - 1) / at_once * (vectors / c * rate + fixed);
        if (c == 1 || cost < least) {
            least = cost;
            best = c;
            alone = own;
        }
    }
    const int64_t rest = p.rows - alone * slots, clusters = alone || slots / best < rest ? slots / best : rest;
    cudaError_t e = allow_smem<logprobs_kernel<T, kTop>>(sizeof(Shared));
    if (e != cudaSuccess) return e;
    return launch_dependent(logprobs_kernel<T, kTop>, dim3(static_cast<unsigned>(clusters * best)), dim3(kThreads), sizeof(Shared), st,
                            best, p, best == 4 ? 2 : best - 1, alone);
}

}  // namespace

cudaError_t launch_logprobs(const Logprobs &p, int dtype, cudaStream_t st)
{
    if (p.n_top > 0) return dtype == 0 ? launch<float, true>(p, st) : launch<uint16_t, true>(p, st);
    return dtype == 0 ? launch<float, false>(p, st) : launch<uint16_t, false>(p, st);
}

}  // namespace gbmla
