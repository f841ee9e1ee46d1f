// What the launches that prepare attn_rows and attn_umma share.
#pragma once
#include <math.h>

#include <atomic>

#include "attn.cuh"
#include "ptx.cuh"

namespace kvbfp {
namespace {

// Everything a call's main kernel reads besides the cache, per (sequence, kv head, row tile) of ROWS query rows: rows of
// q (stored-slot order through `sp`, zeros behind the last row) to shared memory, per-row data, and from the first
// block the tiles before each sequence.  128 threads; ends with a barrier.
template <int ROWS, bool F32>
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
    constexpr int PIECE = F32 ? 4 : 8;      // elements
#pragma unroll
    for (int x = tid; x < ROWS * D / PIECE; x += 128) {
        const int r = x / (D / PIECE), c = x % (D / PIECE) * PIECE, row = rt * ROWS + r;
        float v[PIECE];
#pragma unroll
        for (int e = 0; e < PIECE; ++e) v[e] = 0.f;
        if (row < R) {
            const int i = row / a.group, hq = hk * a.group + row - i * a.group;
            const int64_t at = (((int64_t)b * a.n_draft + i) * a.n_q_heads + hq) * D + c;
            if (F32) {
                const float4 y = *reinterpret_cast<const float4*>(static_cast<const float*>(a.q) + at);
                v[0] = y.x; v[1] = y.y; v[2] = y.z; v[3] = y.w;
            } else {
                const uint4 y = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.q) + at);
                const uint32_t w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[(2 * e) % PIECE] = __uint_as_float(w[e] << 16);
                    v[(2 * e + 1) % PIECE] = __uint_as_float(w[e] & 0xffff0000u);
                }
            }
        }
#pragma unroll
        for (int e = 0; e < PIECE; ++e) sq[r][c + e] = v[e];
    }
    if (tid < ROWS) {
        const int row = rt * ROWS + tid, i = row / a.group;
        const int ctx = min(max(a.ctx_lens[b], 0), a.fmt.max_seq);
        RowInfo x;
        x.pos = ctx - 1;
        x.slope = 0.f;
        x.m0 = x.m1 = 0u;
        if (row < R) {
            if (a.slopes) x.slope = a.slopes[hk * a.group + row - i * a.group];
            if (a.tree) {
                const int64_t at = (int64_t)b * a.n_draft + i;
                const int dep = a.depth ? min(max(a.depth[at], 0), a.n_draft - 1) : i;
                const uint64_t m = a.tree_mask ? a.tree_mask[at] : (i == 63 ? ~0ull : (2ull << i) - 1ull);
                x.pos = ctx + dep;
                x.m0 = (uint32_t)m;
                x.m1 = (uint32_t)(m >> 32);
            }
        }
        a.rows[(int64_t)x0 * ROWS + tid] = x;
    }
    if (hk == 0 && rt == 0) {
        const SeqView sv = seq_view(a, b);
        if (tid == 0) {
            a.views[b] = sv;
            if (sv.clamped) raise_flag(a.status, KVBFP_FLAG_POSITION);
        }
        if (a.tree && tid < a.n_draft)
            a.dpos[b * kAttnMaxDraft + tid] = sv.ctx + (a.depth ? min(max(a.depth[(int64_t)b * a.n_draft + tid], 0), a.n_draft - 1) : tid);
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
