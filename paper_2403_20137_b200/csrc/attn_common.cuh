// Row data of attn_rows and attn_umma, and the launch that prepares the latter.
#pragma once
#include <math.h>

#include <atomic>

#include "attn.cuh"
#include "ptx.cuh"

namespace kvbfp {
namespace {

// tanh as 1 - 2 / (1 + e^2x) is off by some 2e-7 whatever its value, which a cap multiplies: fine for caps up to this one
// (2e-5 of a score at most), while larger ones would lose the scores they are meant to leave alone.
constexpr float kCapFast = 64.f;
__device__ __forceinline__ float finite_factor(float x) { return fminf(x, 1e38f); }      // (0 times it, or three times it, has to stay 0)
// tanh to about 2e-6 of its value: the Taylor series x - x^3/3 + 2x^5/15 - 17x^7/315 + 62x^9/2835 below 1/4 (the next term is
// 9e-9 of the value there), the exponential above.
__device__ __forceinline__ float tanh_relative(float x) {
    const float s = x * x;
    const float small = x * fmaf(s, fmaf(s, fmaf(s, fmaf(s, 62.f / 2835.f, -17.f / 315.f), 2.f / 15.f), -1.f / 3.f), 1.f);
    return fabsf(x) < 0.25f ? small : 1.f - __fdividef(2.f, 1.f + ex2_approx(x * 2.8853900817779268f));
}

// Depth of drafted token i, and what a query row (draft-major, group-minor) needs of itself; rows behind R see no draft.
__device__ __forceinline__ int draft_depth(const AttnArgs& a, int b, int i) {
    return a.depth ? min(max(a.depth[(int64_t)b * a.n_draft + i], 0), a.n_draft - 1) : i;
}
__device__ __forceinline__ RowInfo row_info(const AttnArgs& a, int b, int hk, int row, int R) {
    const int i = row / a.group, ctx = min(max(a.ctx_lens[b], 0), a.fmt.max_seq);
    RowInfo x;
    x.pos = ctx - 1;
    x.slope = 0.f;
    x.m0 = x.m1 = 0u;
    if (row < R) {
        if (a.slopes) x.slope = a.slopes[hk * a.group + row - i * a.group];
        if (a.tree) {
            const uint64_t m = a.tree_mask ? a.tree_mask[(int64_t)b * a.n_draft + i] : (i == 63 ? ~0ull : (2ull << i) - 1ull);
            x.pos = ctx + draft_depth(a, b, i);
            x.m0 = (uint32_t)m;
            x.m1 = (uint32_t)(m >> 32);
        }
    }
    return x;
}

// Everything attn_umma reads besides the cache, per (sequence, kv head, row tile) of ROWS query rows: rows of q
// (stored-slot order through `sp`, zeros behind the last row) to shared memory, per-row data, and from the first
// block the tiles before each sequence.  128 threads; ends with a barrier.
template <int ROWS>
__device__ __forceinline__ void prep_common(const AttnArgs& a, float (&sq)[ROWS][kHeadDim + 4], int (&sp)[kHeadDim]) {
    constexpr int D = kHeadDim;
    __shared__ int scan[4];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int Hkv = a.fmt.n_kv_heads, B = a.fmt.batch, R = a.n_draft * a.group;
    const int x0 = blockIdx.x, rt = x0 % a.n_row_tiles, hk = x0 / a.n_row_tiles % Hkv, b = x0 / a.n_row_tiles / Hkv;
    pdl_wait();
    pdl_trigger();
    sp[tid] = a.perm_k ? (a.perm_k[hk * D + tid] & (D - 1)) : tid;
    // rows of q, 16 bytes a thread and step
#pragma unroll
    for (int x = tid; x < ROWS * D / 8; x += 128) {
        const int r = x / (D / 8), c = x % (D / 8) * 8, row = rt * ROWS + r;
        uint4 y = make_uint4(0u, 0u, 0u, 0u);
        if (row < R) {
            const int i = row / a.group, hq = hk * a.group + row - i * a.group;
            y = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.q) + (((int64_t)b * a.n_draft + i) * a.n_q_heads + hq) * D + c);
        }
        const uint32_t w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            sq[r][c + 2 * e] = __uint_as_float(w[e] << 16);
            sq[r][c + 2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
        }
    }
    if (tid < ROWS) a.rows[(int64_t)x0 * ROWS + tid] = row_info(a, b, hk, rt * ROWS + tid, R);
    if (hk == 0 && rt == 0) {
        const SeqView sv = seq_view(a, b);
        if (tid == 0) {
            a.views[b] = sv;
            if (sv.clamped) raise_flag(a.status, KVBFP_FLAG_POSITION);
        }
        if (tid < a.n_draft) a.dpos[b * kAttnMaxDraft + tid] = sv.ctx + draft_depth(a, b, tid);
    }
    if (x0 == 0) {      // tiles before each sequence
        const int per = (B + 127) / 128;
        int mine = 0;
        for (int i = 0; i < per; ++i)
            if (tid * per + i < B) mine += seq_view(a, tid * per + i).n;
        int x = mine;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, off);
            if (lane >= off) x += y;
        }
        if (lane == 31) scan[warp] = x;
        __syncthreads();
        int before = x - mine;
        for (int w = 0; w < warp; ++w) before += scan[w];
        for (int i = 0; i < per; ++i) {
            const int bb = tid * per + i;
            if (bb < B) {
                a.plan[bb] = before;
                before += seq_view(a, bb).n;
                if (bb == B - 1) a.plan[B] = before;
            }
        }
    }
    __syncthreads();
}

}  // namespace
}  // namespace kvbfp
