// Attention of a ragged batch of new tokens over a contiguous or paged packed cache: entry point and merge of partial results.
#include <math.h>

#include "ragged.cuh"

namespace kvbfp {
namespace {

// Tokens at negative positions see nothing: zeros, by all threads of the grid.
__device__ __noinline__ void ragged_zeros(const RaggedArgs& a) {
    const int lane = threadIdx.x & 31, row = a.n_q_heads * kHeadDim * (a.q_is_bf16 ? 2 : 4) / 16;
    const int64_t me = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * blockDim.x + threadIdx.x, step = (int64_t)gridDim.x * gridDim.y * blockDim.x;
    for (int b0 = 0; b0 < a.batch; b0 += 32) {
        RaggedSeq s = {};
        if (b0 + lane < a.batch) s = ragged_seq(a, b0 + lane);
        const int mine = ragged_row_tiles(a, s, a.rows_tile) > 0 ? min(s.n, max(-s.base, 0)) : 0;
        for (uint32_t some = __ballot_sync(0xffffffffu, mine > 0); some; some &= some - 1) {
            const int l = __ffs(some) - 1;
            uint4* to = static_cast<uint4*>(a.out) + (int64_t)__shfl_sync(0xffffffffu, s.start, l) * row;
            const int64_t pieces = (int64_t)__shfl_sync(0xffffffffu, mine, l) * row;
            for (int64_t i = me; i < pieces; i += step) to[i] = make_uint4(0u, 0u, 0u, 0u);
        }
    }
}

// out = sum_w 2^(m_w - m) o_w / sum_w 2^(m_w - m) l_w over the workers that share an entry.  The block of worker w serves the
// entry that ends in w's first run: with SPLIT a row (blockIdx.y) by four warps that take every fourth partial, else a row per
// warp.  Most blocks find that their worker has none.
template <bool SPLIT>
__global__ void __launch_bounds__(128) ragged_merge(const __grid_constant__ RaggedArgs a) {
    constexpr int D = kHeadDim;
    __shared__ float so[4][D];
    __shared__ float sml[4][2];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    pdl_wait();
    pdl_trigger();
    const int w1 = blockIdx.x;
    const int4 rec = a.rec[w1];
    if (*a.edge) ragged_zeros(a);
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

// Sequences of up to kFewRows bf16 query rows per kv head go to ragged_rows (every eight rows read the cache anew), longer ones
// to ragged_umma (256 rows a pass).  us of both, 8 kv heads, 4 bits (8 bits), rows per kv head:
//                                9 to 16             24               32
//   16 x 8192 tokens      96 | 172 (139 | 192)  131 | 173 (195 | 193)  168 | 175 (256 | 195)
//   1 x 32768             44 | 50  (55 | 54)    52 | 51   (69 | 54)    58 | 51   (80 | 55)
//   64 x 512              39 | 88  (51 | 96)    50 | 89   (67 | 95)    61 | 90   (84 | 98)
constexpr int kFewRows = 16, kRowsTile = 8;
// What beginning and ending an entry costs ragged_umma, in tiles: 14 000 cycles (pi(Q), the first scores, the results) against
// 4700 a tile.
constexpr int kEntryTiles = 3;
struct Kernel {
    int rows_tile, tile, max_workers;
};
inline Kernel kernel_of(bool umma, int mant_bits, int few_tile = kRowsTile) {
    return umma ? Kernel{256, 128, kAttnMaxSms} : Kernel{few_tile, attn_rows_tile(mant_bits), 3 * kAttnWarps * kAttnMaxSms};
}

// Workspace of one of the two from `base` on; returns the size and, with `a`, sets the pointers.
size_t lay_out(const Kernel& k, int64_t rows, RaggedArgs* a, uint8_t* base) {
    const int part_rows = (int)(rows < k.rows_tile ? rows : k.rows_tile);
    const size_t rec = up256((size_t)k.max_workers * sizeof(int4)) + 256;
    if (a) {
        a->rows_tile = k.rows_tile;
        a->part_rows = part_rows;
        a->rec = reinterpret_cast<int4*>(base);
        a->edge = reinterpret_cast<int*>(base + rec - 256);
        a->partials = reinterpret_cast<float*>(base + rec);
    }
    return rec + up256((size_t)2 * k.max_workers * part_rows * kAttnPart * 4);
}

kvbfp_status launch_kernel(RaggedArgs a, bool umma, const Kernel& k, int64_t rows, uint8_t* workspace, int n_sm, cudaStream_t s) {
    const int bits = a.fmt.mant_bits;
    (void)lay_out(k, rows, &a, workspace);
    const int64_t most = (rows / k.rows_tile + a.batch) * a.fmt.n_kv_heads * (a.map.cap / k.tile + 2 + kEntryTiles);
    const int per_block = umma ? 1 : kAttnWarps;
    int64_t grid = (int64_t)n_sm * (umma ? 1 : attn_rows_blocks(a.q_is_bf16));
    if (grid * per_block > k.max_workers) grid = k.max_workers / per_block;
    if (grid > most) grid = most;
    a.workers = (int)grid * per_block;
    a.extra = umma ? kEntryTiles : 0;
    a.out_up = umma ? 65536.f : 256.f;
    kvbfp_status st;
    if (umma) st = bits == 4 ? launch_ragged_umma4(a, (int)grid, s) : bits == 6 ? launch_ragged_umma6(a, (int)grid, s) : launch_ragged_umma8(a, (int)grid, s);
    else st = bits == 4 ? launch_ragged_rows4(a, (int)grid, s) : bits == 6 ? launch_ragged_rows6(a, (int)grid, s) : launch_ragged_rows8(a, (int)grid, s);
    if (st != KVBFP_OK) return st;
    // a block per row where an entry has one or two, a warp per row otherwise
    if (a.part_rows <= 2) KVBFP_CUDA(launch_pdl(ragged_merge<true>, dim3(a.workers, a.part_rows), dim3(128), 0, s, a));
    else KVBFP_CUDA(launch_pdl(ragged_merge<false>, dim3(a.workers, (a.part_rows + 3) / 4), dim3(128), 0, s, a));
    KVBFP_LAUNCH_CHECK("ragged_merge");
    return KVBFP_OK;
}

}  // namespace
}  // namespace kvbfp

extern "C" size_t kvbfp_ragged_workspace_bytes(const kvbfp_format* fmt, int32_t batch, int32_t n_q_heads, int32_t n_tokens) {
    using namespace kvbfp;
    if (check_format(fmt) != KVBFP_OK || n_q_heads < 1 || n_q_heads % fmt->n_kv_heads != 0 || n_tokens < 0 || batch < 1) return 0;
    if (batch > kMaxPagedBatch || n_q_heads / fmt->n_kv_heads > 8) return 0;
    const int64_t rows = (int64_t)n_tokens * (n_q_heads / fmt->n_kv_heads);
    const size_t few = lay_out(kernel_of(false, fmt->mant_bits), rows, nullptr, nullptr);
    return rows > kFewRows ? few + lay_out(kernel_of(true, fmt->mant_bits), rows, nullptr, nullptr) : few;
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
    if (!cache->k_mant || !cache->k_exp || !cache->v_mant || !cache->v_exp || !starts || !seq_lens) return KVBFP_ERR_INVALID_ARG;
    if (n_tokens != 0 && (!q || !out)) return KVBFP_ERR_INVALID_ARG;          // (arrays of no tokens may well have no address)
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
    a.window = window < a.map.cap ? window : 0;          // (a window of the whole cache hides nothing)
    a.n_sink = a.window == 0 ? 0 : n_sink < a.map.cap ? n_sink : a.map.cap;
    a.out = out;
    const int64_t rows = (int64_t)n_tokens * group;
    st = status_word(&a.status);
    if (st != KVBFP_OK) return st;
    int n_sm = 0;
    st = sm_count(&n_sm);
    if (st != KVBFP_OK) return st;
    cudaStream_t s = (cudaStream_t)stream;
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    const bool bf16 = dt == KVBFP_BF16;
    const size_t few_bytes = lay_out(kernel_of(false, f.mant_bits), rows, nullptr, nullptr);
    // The hint says whether any sequence may have many rows; where it says that none has, all go to ragged_rows, whatever they
    // have.  Where some may, single tokens between them still do.  Items are counted in 32 bits.
    const auto countable = [&](const Kernel& k, int64_t row_tiles) {
        return row_tiles * f.n_kv_heads * (a.map.cap / k.tile + 2 + kEntryTiles) < (int64_t)1 << 31;
    };
    // ragged_rows: four bf16 rows an item where more are not expected (single tokens, or single tokens between longer sequences),
    // whose second term of the weights costs 1 %; eight, which read the cache once for all of them (second term: 4.5 to 12 %), otherwise.
    // (16 x 8192, 8 heads: four rows 50 us in fours, 55 in eights; eight rows 83, 59.)  In fours, only up to eight rows of a sequence
    // stay with ragged_rows (8 bits, us of both: 8 rows 130 | 188, 16 rows 245 | 193).
    const int64_t hint = (int64_t)max_new * group;
    const bool four = bf16 && (hint <= 4 || (hint > kFewRows && group <= 4)) && countable(kernel_of(false, f.mant_bits, 4), rows / 4 + batch);
    const Kernel k_few = kernel_of(false, f.mant_bits, four ? 4 : kRowsTile), k_many = kernel_of(true, f.mant_bits);
    const bool all_few = countable(k_few, rows / k_few.rows_tile + batch);
    const bool many = bf16 && rows > kFewRows && (hint > kFewRows || !all_few);
    if (many ? !countable(k_few, batch) || !countable(k_many, rows / k_many.rows_tile + batch) : !all_few) return KVBFP_ERR_UNSUPPORTED;
    const int few = four ? 8 : kFewRows;
    a.few_lo = 0;
    a.few_hi = many ? few : 0x7fffffff;
    st = !many || batch > 1 ? launch_kernel(a, false, k_few, rows, ws, n_sm, s) : KVBFP_OK;
    if (st != KVBFP_OK || !many) return st;
    a.few_lo = batch > 1 ? few : 0;
    a.few_hi = 0x7fffffff;
    return launch_kernel(a, true, k_many, rows, ws + few_bytes, n_sm, s);
}
