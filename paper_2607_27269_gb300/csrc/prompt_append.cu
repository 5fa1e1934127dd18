// mla_gqa_prompt_append: keys and values of packed prompts into the caches of
// the original GQA layer, keys and queries rotated to their positions
// (Sec. 3.1, R_t; Eq. 1's projections as input).
//
// y = x cos(p theta_k) - x' sin(p theta_k) over head_dim / 2 pairs: three
// operations a value against four bytes moved, so memory is the bound: 67584 tokens
// of 32 + 2 x 8 heads of 64 into a paged cache, 830 MB, take 133 us, 6.2 TB/s.  A block
// takes up to eight tokens of all heads: the sine and cosine of a (token, pair)
// are evaluated once, into shared memory, and serve every head; so are the
// tokens' sequences, positions and pages.  Everything else moves in 16-byte
// vectors, a rotation's two vectors in one thread.
#include "common.cuh"
#include "internal.h"

namespace gbmla {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxTokens = kThreads / 32;  // a warp looks a token up

struct Args {
    PromptAppend p;
    RopeTurns turns;
};

__device__ __forceinline__ float lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack(float a, float b)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ uint4 ld16(const uint16_t *p) { return *reinterpret_cast<const uint4 *>(p); }
__device__ __forceinline__ void st16(uint16_t *p, const uint4 &v) { *reinterpret_cast<uint4 *>(p) = v; }

// A row's eight pairs number 8 c .. 8 c + 7, a and b their two vectors: of style
// 0 the first and second halves of the row, of style 1 two neighbours.
template <int STYLE>
__device__ __forceinline__ void rotate(uint4 &a, uint4 &b, const float2 *cs)
{
    uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (STYLE == 0) {
            const float2 c0 = cs[2 * i], c1 = cs[2 * i + 1];
            const float p0 = lo(x[i]), p1 = hi(x[i]), q0 = lo(y[i]), q1 = hi(y[i]);
            x[i] = pack(p0 * c0.x - q0 * c0.y, p1 * c1.x - q1 * c1.y);
            y[i] = pack(q0 * c0.x + p0 * c0.y, q1 * c1.x + p1 * c1.y);
        } else {
            const float2 c0 = cs[i], c1 = cs[4 + i];
            x[i] = pack(lo(x[i]) * c0.x - hi(x[i]) * c0.y, hi(x[i]) * c0.x + lo(x[i]) * c0.y);
            y[i] = pack(lo(y[i]) * c1.x - hi(y[i]) * c1.y, hi(y[i]) * c1.x + lo(y[i]) * c1.y);
        }
    }
    a = make_uint4(x[0], x[1], x[2], x[3]);
    b = make_uint4(y[0], y[1], y[2], y[3]);
}

// D: head width.  nt: tokens of a block.
template <int D, int STYLE>
__global__ void __launch_bounds__(kThreads) prompt_append_kernel(const __grid_constant__ Args a, int nt)
{
    constexpr int C = D / 16;  // groups of eight pairs a row
    __shared__ int32_t s_pos[kMaxTokens];                // position; kNone: no such token
    __shared__ int32_t s_seq[kMaxTokens];
    __shared__ __align__(16) float2 s_cs[kMaxTokens][D / 2];
    __shared__ int32_t s_blk[kMaxTokens][128];           // a token's block in each group's cache, -1: not cached
    constexpr int32_t kNone = INT32_MIN;
    const PromptAppend &p = a.p;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int t0 = blockIdx.x * nt, n = min(nt, p.total - t0);
    // (writes caches: no early trigger, see append.cu)
    griddep_wait();
    if (blockIdx.x == 0) {
        for (int b = tid; b < p.batch; b += kThreads)
            if (p.cu[b] < 0 || p.cu[b + 1] < p.cu[b] || p.cu[b + 1] > p.total) record_status(p.status, kStatusBounds);
    }
    if (warp < n) {
        // the first sequence that holds the token, if any does (others' offsets may fall)
        const int t = t0 + warp;
        int seq = INT32_MAX;
        for (int b = lane; b < p.batch; b += 32) {
            const int first = p.cu[b], end = p.cu[b + 1];
            if (first >= 0 && first <= t && t < end && end <= p.total) seq = min(seq, b);
        }
        seq = __reduce_min_sync(0xffffffffu, seq);
        if (lane == 0) {
            int pos = kNone;
            if (seq != INT32_MAX) {
                const int64_t at = static_cast<int64_t>(p.start[seq]) + (t - p.cu[seq]);
                if (at >= 0 && at < INT32_MAX)
                    pos = static_cast<int>(at);
                else
                    record_status(p.status, kStatusBounds);
            }
            s_pos[warp] = pos;
            s_seq[warp] = seq;
        }
    }
    __syncthreads();
    for (int i = tid; i < n * (D / 2); i += kThreads) {
        const int t = i / (D / 2), k = i - t * (D / 2);
        if (s_pos[t] != kNone) {
            float c, s;
            rope_cos_sin(s_pos[t], a.turns.f[k], &c, &s);
            s_cs[t][k] = make_float2(c, s);
        }
    }
    const CacheView &c = p.cache;
    for (int i = tid; i < n * p.groups; i += kThreads) {
        const int t = i / p.groups, g = i - t * p.groups;
        int blk = -1;
        if (s_pos[t] != kNone) {
            const int64_t u = static_cast<int64_t>(s_seq[t]) * p.groups + g;
            if (s_pos[t] < c.capacity) {
                blk = c.block_table ? c.block_table[u * c.bt_stride + s_pos[t] / c.page_size] : static_cast<int>(u);
                if (c.block_table && (blk < 0 || blk >= c.num_pages)) blk = -1;
            }
            if (blk < 0) record_status(p.status, kStatusBounds);
        }
        s_blk[t][g] = blk;
    }
    __syncthreads();
    const int rows = p.groups + (p.q ? p.heads : 0);  // rotated rows a token
    constexpr int kSecond = STYLE == 0 ? D / 2 : 8, kStep = STYLE == 0 ? 8 : 16;
    for (int i = tid; i < n * rows * C; i += kThreads) {
        const int t = i / (rows * C), rest = i - t * rows * C, h = rest / C, e = rest - h * C;
        if (s_pos[t] == kNone) continue;
        const int64_t tok = t0 + t;
        const uint16_t *src;
        uint16_t *dst;
        if (h < p.groups) {
            const int blk = s_blk[t][h];
            if (blk < 0) continue;
            const int slot = c.block_table ? s_pos[t] % c.page_size : s_pos[t];
            src = static_cast<const uint16_t *>(p.k) + tok * p.k_stride + h * D;
            dst = (uint16_t *)c.k_rope + blk * c.r_blk + slot * c.r_tok;
        } else {
            src = static_cast<const uint16_t *>(p.q) + tok * p.q_stride + (h - p.groups) * D;
            dst = static_cast<uint16_t *>(p.q_rot) + tok * p.q_rot_stride + (h - p.groups) * D;
        }
        uint4 x = ld16(src + e * kStep), y = ld16(src + e * kStep + kSecond);
        rotate<STYLE>(x, y, &s_cs[t][8 * e]);
        st16(dst + e * kStep, x);
        st16(dst + e * kStep + kSecond, y);
    }
    for (int i = tid; i < n * p.groups * (D / 8); i += kThreads) {
        const int t = i / (p.groups * (D / 8)), rest = i - t * p.groups * (D / 8), g = rest / (D / 8), e = rest % (D / 8);
        if (s_pos[t] == kNone || s_blk[t][g] < 0) continue;
        const int slot = c.block_table ? s_pos[t] % c.page_size : s_pos[t];
        st16((uint16_t *)c.c_kv + s_blk[t][g] * c.c_blk + slot * c.c_tok + e * 8,
             ld16(static_cast<const uint16_t *>(p.v) + (t0 + t) * p.v_stride + g * D + e * 8));
    }
}

}  // namespace

cudaError_t launch_prompt_append(const PromptAppend &p, cudaStream_t st)
{
    Args a{p, rope_turns(p.head_dim, p.rope_base)};
    // eight tokens a block, fewer where that leaves SMs without one
    int nt = kMaxTokens;
    while (nt > 1 && (p.total + nt - 1) / nt < 2 * p.sms) nt /= 2;
    const dim3 grid((p.total + nt - 1) / nt);
    const auto kernel = p.head_dim == 64 ? (p.rope_style == 0 ? prompt_append_kernel<64, 0> : prompt_append_kernel<64, 1>)
                                         : (p.rope_style == 0 ? prompt_append_kernel<128, 0> : prompt_append_kernel<128, 1>);
    return launch_dependent(kernel, grid, dim3(kThreads), 0, st, 1, a, nt);
}

}  // namespace gbmla
