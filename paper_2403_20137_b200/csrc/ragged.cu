// Attention of a ragged batch of new tokens over a contiguous or paged packed cache: entry point and merge of partial results.
#include <math.h>

#include "ragged.cuh"

namespace kvbfp {
namespace {

// out = sum_w 2^(m_w - m) o_w / sum_w 2^(m_w - m) l_w over the workers that share an entry.  The block of worker w serves the
// entry that ends in w's first run: with SPLIT a row (blockIdx.y) by four warps that take every fourth partial, else a row per
// warp.  Most blocks find that their worker has none.
template <bool SPLIT>
__global__ void __launch_bounds__(128) ragged_merge(const RaggedArgs a) {
    constexpr int D = kHeadDim;
    __shared__ float so[4][D];
    __shared__ float sml[4][2];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    pdl_wait();
    pdl_trigger();
    const int w1 = blockIdx.x;
    const int4 rec = a.rec[w1];
    if (rec.x < 0) return;
    const int b = rec.x, rt = rec.y, hk = rec.z, w0 = rec.w;
    const int r = SPLIT ? (int)blockIdx.y : (int)blockIdx.y * 4 + warp, row = rt * a.rows_tile + r;
    int4 slot = make_int4(4 * lane, 4 * lane + 1, 4 * lane + 2, 4 * lane + 3);
    if (a.inv_perm_v) slot = *reinterpret_cast<const int4*>(a.inv_perm_v + hk * D + 4 * lane);
    const RaggedSeq s = ragged_seq(a, b);
    const int i = row / a.group, hq = hk * a.group + row - i * a.group;
    if (r >= a.part_rows || i >= s.n || s.base + i < 0) return;           // (SPLIT: the whole block)
    auto part = [&](int w) { return a.partials + ((int64_t)(2 * w + (w == w0 ? 1 : 0)) * a.part_rows + r) * kAttnPart; };
    float m = -INFINITY, l = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    // a batch of 32 partials: a lane each for maximum and sum, the vectors eight at a time, the first of them on their way
    // before the maximum is known
    const int step = SPLIT ? 4 : 1;
    for (int base = w0 + (SPLIT ? warp : 0); base <= w1; base += 32 * step) {
        const int w = base + lane * step, cnt = min(32, (w1 - base) / step + 1);
        const bool have = w <= w1;
        const float* pk = part(have ? w : w0);
        const float mk = have ? pk[D] : -INFINITY;
        const float lk = have ? pk[D + 1] : 0.f;
        float4 v[8];
        auto load = [&](int j0) {
#pragma unroll
            for (int u = 0; u < 8; ++u)
                v[u] = (j0 + u < cnt) ? *reinterpret_cast<const float4*>(part(base + (j0 + u) * step) + 4 * lane)
                                      : make_float4(0.f, 0.f, 0.f, 0.f);
        };
        load(0);
        float mn = mk;
#pragma unroll
        for (int off = 16; off; off >>= 1) mn = fmaxf(mn, __shfl_xor_sync(0xffffffffu, mn, off));
        mn = fmaxf(mn, m);
        const float a1 = (m == -INFINITY) ? 0.f : exp2f(m - mn);
        const float ak = have ? exp2f(mk - mn) : 0.f;
        float ls = have ? ak * lk : 0.f;
#pragma unroll
        for (int off = 16; off; off >>= 1) ls += __shfl_xor_sync(0xffffffffu, ls, off);
        acc.x *= a1; acc.y *= a1; acc.z *= a1; acc.w *= a1;
        l = l * a1 + ls;
        m = mn;
        for (int j0 = 0; j0 < cnt; j0 += 8) {
            if (j0) load(j0);
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const float f = __shfl_sync(0xffffffffu, ak, (j0 + u) & 31);
                acc.x += f * v[u].x; acc.y += f * v[u].y; acc.z += f * v[u].z; acc.w += f * v[u].w;
            }
        }
    }
    *reinterpret_cast<float4*>(&so[warp][4 * lane]) = acc;
    if (SPLIT) {
        if (lane == 0) { sml[warp][0] = m; sml[warp][1] = l; }
        __syncthreads();
        if (warp != 0) return;
        m = fmaxf(fmaxf(sml[0][0], sml[1][0]), fmaxf(sml[2][0], sml[3][0]));
        acc = make_float4(0.f, 0.f, 0.f, 0.f);
        l = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = (sml[w][0] == -INFINITY) ? 0.f : exp2f(sml[w][0] - m);
            const float4 v = *reinterpret_cast<const float4*>(&so[w][4 * lane]);
            acc.x += f * v.x; acc.y += f * v.y; acc.z += f * v.z; acc.w += f * v.w;
            l += f * sml[w][1];
        }
        __syncwarp();
        *reinterpret_cast<float4*>(&so[0][4 * lane]) = acc;
    }
    __syncwarp();
    const float* src = so[SPLIT ? 0 : warp];
    const float inv = l != 0.f ? a.out_up / l : 0.f;
    const int sl[4] = {slot.x & (D - 1), slot.y & (D - 1), slot.z & (D - 1), slot.w & (D - 1)};
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = inv == 0.f ? 0.f : src[sl[e]] * inv;
    const int64_t at = ((int64_t)(s.start + i) * a.n_q_heads + hq) * D + 4 * lane;
    if (a.q_is_bf16)
        *reinterpret_cast<__nv_bfloat162*>(static_cast<__nv_bfloat16*>(a.out) + at) = __floats2bfloat162_rn(v[0], v[1]),
        *reinterpret_cast<__nv_bfloat162*>(static_cast<__nv_bfloat16*>(a.out) + at + 2) = __floats2bfloat162_rn(v[2], v[3]);
    else
        *reinterpret_cast<float4*>(static_cast<float*>(a.out) + at) = make_float4(v[0], v[1], v[2], v[3]);
}

inline size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
constexpr int kRowsWorkers = 3 * kAttnWarps * kAttnMaxSms;

// Workspace regions in order; returns the size and, with `a`, sets the pointers.
size_t lay_out(int64_t rows, RaggedArgs* a, uint8_t* base) {
    const int part_rows = (int)(rows < 8 ? rows : 8);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        uint8_t* p = base + at;
        at += up256(bytes);
        return p;
    };
    uint8_t* rec = take((size_t)kRowsWorkers * sizeof(int4));
    uint8_t* part = take((size_t)2 * kRowsWorkers * part_rows * kAttnPart * 4);
    if (a) {
        a->part_rows = part_rows;
        a->rec = reinterpret_cast<int4*>(rec);
        a->partials = reinterpret_cast<float*>(part);
    }
    return at;
}

}  // namespace
}  // namespace kvbfp

extern "C" size_t kvbfp_ragged_workspace_bytes(const kvbfp_format* fmt, int32_t batch, int32_t n_q_heads, int32_t n_tokens) {
    using namespace kvbfp;
    if (check_format(fmt) != KVBFP_OK || n_q_heads < 1 || n_q_heads % fmt->n_kv_heads != 0 || n_tokens < 0 || batch < 1) return 0;
    if (batch > kMaxPagedBatch || n_q_heads / fmt->n_kv_heads > 8) return 0;
    return lay_out((int64_t)n_tokens * (n_q_heads / fmt->n_kv_heads), nullptr, nullptr);
}

extern "C" kvbfp_status kvbfp_ragged_attn(const kvbfp_cache* cache, const kvbfp_pages* pages, const void* q, kvbfp_dtype dt,
                                          int32_t n_q_heads, int32_t n_tokens, int32_t batch, const int32_t* starts,
                                          const int32_t* seq_lens, int32_t max_new, int32_t window, int32_t n_sink,
                                          const int32_t* perm_k, const int32_t* inv_perm_v, float softmax_scale, void* out,
                                          void* workspace, size_t workspace_bytes, void* stream) {
    using namespace kvbfp;
    if (!cache) return KVBFP_ERR_INVALID_ARG;
    const kvbfp_format& f = cache->fmt;
    kvbfp_status st = check_format(&f);
    if (st == KVBFP_OK && pages) st = check_pool(f, pages);
    if (st != KVBFP_OK) return st;
    if (!cache->k_mant || !cache->k_exp || !cache->v_mant || !cache->v_exp || !q || !starts || !seq_lens || !out) return KVBFP_ERR_INVALID_ARG;
    if (dt != KVBFP_F32 && dt != KVBFP_BF16) return KVBFP_ERR_INVALID_ARG;
    if (n_q_heads < 1 || n_q_heads % f.n_kv_heads != 0 || n_tokens < 0 || max_new < 0 || window < 0 || n_sink < 0) return KVBFP_ERR_INVALID_ARG;
    if (batch != (pages ? pages->batch : f.batch)) return KVBFP_ERR_INVALID_ARG;
    const int group = n_q_heads / f.n_kv_heads;
    if (group > 8 || batch > kMaxPagedBatch || n_tokens > 1 << 26) return KVBFP_ERR_UNSUPPORTED;
    if (!(softmax_scale >= 0.f) || isinf(softmax_scale)) return KVBFP_ERR_INVALID_ARG;
    const void* ptrs[] = {cache->k_mant, cache->k_exp, cache->v_mant, cache->v_exp, q, out, workspace, perm_k, inv_perm_v};
    for (const void* p : ptrs)
        if (p && !aligned16(p)) return KVBFP_ERR_ALIGNMENT;
    if (!workspace || workspace_bytes < kvbfp_ragged_workspace_bytes(&f, batch, n_q_heads, n_tokens)) return KVBFP_ERR_WORKSPACE;
    if (n_tokens == 0) return KVBFP_OK;

    RaggedArgs a = {};
    a.fmt = f;
    a.map = token_map(f, pages);
    a.k_mant = cache->k_mant; a.k_exp = cache->k_exp; a.v_mant = cache->v_mant; a.v_exp = cache->v_exp;
    a.q = q; a.q_is_bf16 = dt == KVBFP_BF16; a.n_q_heads = n_q_heads; a.group = group; a.batch = batch; a.n_tokens = n_tokens;
    a.starts = starts; a.lens = seq_lens; a.perm_k = perm_k; a.inv_perm_v = inv_perm_v;
    a.scale = softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)f.head_dim);
    a.window = window; a.n_sink = window > 0 ? n_sink : 0;
    a.out = out;
    const int64_t rows = (int64_t)n_tokens * group;
    (void)lay_out(rows, &a, static_cast<uint8_t*>(workspace));
    st = status_word(&a.status);
    if (st != KVBFP_OK) return st;
    int n_sm = 0;
    st = sm_count(&n_sm);
    if (st != KVBFP_OK) return st;
    a.few_lo = 0;
    a.few_hi = 0x7fffffff;
    a.rows_tile = 8;
    a.out_up = 256.f;
    const int tile = attn_rows_tile(f.mant_bits);
    // items are counted in 32 bits
    const int64_t most = (rows / 8 + batch) * f.n_kv_heads * (a.map.cap / tile + 2);
    if (most >= (int64_t)1 << 31) return KVBFP_ERR_UNSUPPORTED;
    int64_t grid = (int64_t)n_sm * attn_rows_blocks(a.q_is_bf16);
    if (grid * kAttnWarps > kRowsWorkers) grid = kRowsWorkers / kAttnWarps;
    if (grid > most) grid = most;
    a.workers = (int)grid * kAttnWarps;

    cudaStream_t s = (cudaStream_t)stream;
    st = f.mant_bits == 4 ? launch_ragged_rows4(a, (int)grid, s) : f.mant_bits == 6 ? launch_ragged_rows6(a, (int)grid, s) : launch_ragged_rows8(a, (int)grid, s);
    if (st != KVBFP_OK) return st;
    // a block per row where an entry has one or two, a warp per row otherwise
    if (a.part_rows <= 2) KVBFP_CUDA(launch_pdl(ragged_merge<true>, dim3(a.workers, a.part_rows), dim3(128), 0, s, a));
    else KVBFP_CUDA(launch_pdl(ragged_merge<false>, dim3(a.workers, (a.part_rows + 3) / 4), dim3(128), 0, s, a));
    KVBFP_LAUNCH_CHECK("ragged_merge");
    return KVBFP_OK;
}
