// Attention over the packed cache beyond one plain token: drafted trees, capped / biased / masked scores, attention
// weights gathered per cached token.  Entry points, merge of partial results, and the weight pass.
#include <math.h>

#include "attn.cuh"

namespace kvbfp {
namespace {

// One warp (SPLIT: one block of four) per query row: out = sum_w 2^(m_w - m) o_w / sum_w 2^(m_w - m) l_w over the
// partials of the workers that share the row's tiles.  Rows whose tiles one worker had are written already; rows that
// see no tile are zeros.
template <bool SPLIT>
__global__ void __launch_bounds__(128) attn_merge(const AttnArgs a, int64_t n_rows) {
    constexpr int D = kHeadDim;
    __shared__ float so[4][D];
    __shared__ float sml[4][2];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t x = SPLIT ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * 4 + warp;       // ((b, hk), row): rows of a pair together
    pdl_wait();
    pdl_trigger();
    if (x >= n_rows) return;
    const int R = a.n_draft * a.group, Hkv = a.fmt.n_kv_heads, B = a.fmt.batch;
    const int row = (int)(x % R), hk = (int)(x / R % Hkv), b = (int)(x / R / Hkv);
    const int i = row / a.group, hq = hk * a.group + row % a.group;
    // (all that does not depend on the split first: what bounds this kernel is the chain of loads)
    const int c0 = a.plan[b], n = a.plan[b + 1] - c0;
    const int nd = a.tree ? a.views[b].nd : a.n_draft;
    int4 slot = make_int4(4 * lane, 4 * lane + 1, 4 * lane + 2, 4 * lane + 3);
    if (a.inv_perm_v) slot = *reinterpret_cast<const int4*>(a.inv_perm_v + hk * D + 4 * lane);
    const int HR = Hkv * a.n_row_tiles, n_items = a.plan[B] * HR;
    const int rt = row / a.rows_tile, r = row - rt * a.rows_tile;
    int w0 = 0, w1 = -1;
    if (n > 0) {
        const int first = c0 * HR + (hk * a.n_row_tiles + rt) * n;
        const int workers = min(a.workers, n_items);
        w0 = worker_of(first, n_items, workers);
        w1 = worker_of(first + n - 1, n_items, workers);
        if (w0 == w1) return;
    }
    auto part = [&](int w) {
        return a.partials + ((int64_t)(2 * w + (w == w0 ? 1 : 0)) * a.part_rows + r) * kAttnPart;
    };
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
    const bool live = n > 0 && i < nd;
    const float inv = (live && l != 0.f) ? a.out_up / l : 0.f;
    const int sl[4] = {slot.x & (D - 1), slot.y & (D - 1), slot.z & (D - 1), slot.w & (D - 1)};
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = inv == 0.f ? 0.f : src[sl[e]] * inv;
    const int64_t at = (((int64_t)b * a.n_draft + i) * a.n_q_heads + hq) * D + 4 * lane;
    if (a.q_is_bf16)
        *reinterpret_cast<__nv_bfloat162*>(static_cast<__nv_bfloat16*>(a.out) + at) = __floats2bfloat162_rn(v[0], v[1]),
        *reinterpret_cast<__nv_bfloat162*>(static_cast<__nv_bfloat16*>(a.out) + at + 2) = __floats2bfloat162_rn(v[2], v[3]);
    else
        *reinterpret_cast<float4*>(static_cast<float*>(a.out) + at) = make_float4(v[0], v[1], v[2], v[3]);
    if (a.lse && lane == 0) a.lse[(int64_t)b * a.n_q_heads + hq] = l > 0.f ? m + log2f(l) : (l == 0.f ? INFINITY : l);
}

// mass[b, h, t] += sum over the group's query heads of 2^(score - lse).  tile / 4 lanes per tile, four tokens a lane;
// the tiles are those the scores were written for.  Hidden tokens are skipped, not added as zeros: the sum of a query that
// is not finite is NaN.  Memory-bound: 4 G + 8 bytes a token.
__global__ void __launch_bounds__(128) attn_mass(const AttnArgs a) {
    pdl_wait();
    pdl_trigger();
    const int B = a.fmt.batch, Hkv = a.fmt.n_kv_heads, max_seq = a.fmt.max_seq;
    const int lanes = a.tile / 4, teams = gridDim.x * (128 / lanes), me = (blockIdx.x * 128 + threadIdx.x) / lanes;
    const int n_items = a.plan[B] * Hkv;
    if (n_items == 0) return;
    const int i0 = worker_start(me, n_items, teams), i1 = worker_start(me + 1, n_items, teams);
    if (i0 >= i1) return;
    int lo = 0, hi = B - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.plan[mid] * Hkv <= i0) lo = mid; else hi = mid - 1;
    }
    int b = lo, n = a.plan[lo + 1] - a.plan[lo];
    int h = (i0 - a.plan[lo] * Hkv) / n, k = i0 - a.plan[lo] * Hkv - h * n;
    SeqView sv = a.views[b];
    for (int item = i0; item < i1; ++item) {
        const int tok = tile_token(sv, k, a.tile) + 4 * (threadIdx.x % lanes);
        if (tok < sv.ctx) {
            float4* to = reinterpret_cast<float4*>(a.mass + ((int64_t)b * Hkv + h) * max_seq + tok);
            float4 acc = *to;
            const float* y = a.scores + ((int64_t)b * a.n_q_heads + h * a.group) * max_seq + tok;
            const float* ls = a.lse + (int64_t)b * a.n_q_heads + h * a.group;
            const int from = max(sv.first, a.window > 0 ? sv.ctx - a.window : 0);
            bool see[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) see[e] = tok + e < sv.ctx && (tok + e >= from || tok + e < sv.pf);
            for (int q = 0; q < a.group; ++q) {
                const float4 s = *reinterpret_cast<const float4*>(y + (int64_t)q * max_seq);
                const float z = ls[q];
                if (see[0]) acc.x += exp2f(s.x - z);
                if (see[1]) acc.y += exp2f(s.y - z);
                if (see[2]) acc.z += exp2f(s.z - z);
                if (see[3]) acc.w += exp2f(s.w - z);
            }
            *to = acc;
        }
        if (++k == n) {
            k = 0;
            if (++h == Hkv) {
                h = 0;
                do { ++b; } while (b < B && a.plan[b + 1] == a.plan[b]);
                if (b < B) {
                    n = a.plan[b + 1] - a.plan[b];
                    sv = a.views[b];
                }
            }
        }
    }
}

// Query rows per work item.  Eight rows are the narrow side of a warp-level product (attn_rows); up to 64 bf16 rows of a
// kv head share the tiles that attn_umma converts once, in its three widths.  Both sides at 16 x 32 x 8192 4-bit rows: eight
// bf16 rows 160 us with attn_rows, 181 with attn_umma (with the weights); 16 rows 128 us with attn_umma, 150 with a
// warp-level kernel of that width.  fp32 rows stay with attn_rows: their three bf16 terms fill its registers at eight.
inline int rows_tile_for(int rows, bool bf16) { return !bf16 || rows <= 8 ? 8 : rows <= 16 ? 16 : rows <= 32 ? 32 : 64; }
inline int max_workers(int rows_tile) { return (rows_tile == 8 ? 3 * kAttnWarps : 3) * kAttnMaxSms; }

inline size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

// Workspace regions in order; returns the size and, with `a`, sets the pointers.
size_t lay_out(const kvbfp_format& f, int n_q_heads, int n_draft, bool bf16, bool with_mass, AttnArgs* a, uint8_t* base) {
    const int rows = n_draft * (n_q_heads / f.n_kv_heads), tile = rows_tile_for(rows, bf16);
    const size_t items = (size_t)f.batch * f.n_kv_heads * ((rows + tile - 1) / tile);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        uint8_t* p = base + at;
        at += up256(bytes);
        return p;
    };
    uint8_t* plan = take((size_t)(f.batch + 1) * sizeof(int));
    uint8_t* views = take((size_t)f.batch * sizeof(SeqView));
    uint8_t *dpos = nullptr, *info = nullptr, *frag = nullptr;
    if (tile != 8) {          // attn_umma's
        dpos = take((size_t)f.batch * kAttnMaxDraft * sizeof(int));
        info = take(items * tile * sizeof(RowInfo));
        frag = take(items * tile * kHeadDim * 2);
    }
    uint8_t *lse = nullptr, *scores = nullptr;
    if (with_mass) {
        lse = take((size_t)f.batch * n_q_heads * 4);
        scores = take((size_t)f.batch * n_q_heads * f.max_seq * 4);
    }
    uint8_t* part = take((size_t)2 * max_workers(tile) * (rows < tile ? rows : tile) * kAttnPart * 4);
    if (a) {
        a->plan = reinterpret_cast<int*>(plan);
        a->views = reinterpret_cast<SeqView*>(views);
        a->dpos = reinterpret_cast<int*>(dpos);
        a->rows = reinterpret_cast<RowInfo*>(info);
        a->qfrag = reinterpret_cast<uint4*>(frag);
        a->lse = reinterpret_cast<float*>(lse);
        a->scores = reinterpret_cast<float*>(scores);
        a->partials = reinterpret_cast<float*>(part);
    }
    return at;
}

struct AttnCall {
    const kvbfp_cache* cache;
    const void* q;
    kvbfp_dtype dt;
    int n_q_heads, n_draft, tree;
    const int32_t *ctx_lens, *draft_lens;
    const uint64_t* tree_mask;
    const int32_t* depth;
    const int32_t *perm_k, *inv_perm_v;
    float softmax_scale;
    const kvbfp_score_mod* mod;
    float* mass;
    bool with_mass;
    void* out;
    void* workspace;
    size_t workspace_bytes;
    void* stream;
};

kvbfp_status attn_common(const AttnCall& c) {
    if (!c.cache) return KVBFP_ERR_INVALID_ARG;
    const kvbfp_format& f = c.cache->fmt;
    kvbfp_status st = check_format(&f);
    if (st != KVBFP_OK) return st;
    if (!c.cache->k_mant || !c.cache->k_exp || !c.cache->v_mant || !c.cache->v_exp || !c.q || !c.ctx_lens || !c.out ||
        (c.with_mass && !c.mass))
        return KVBFP_ERR_INVALID_ARG;
    if (c.dt != KVBFP_F32 && c.dt != KVBFP_BF16) return KVBFP_ERR_INVALID_ARG;
    if (c.n_q_heads < 1 || c.n_q_heads % f.n_kv_heads != 0 || c.n_draft < 1) return KVBFP_ERR_INVALID_ARG;
    const int group = c.n_q_heads / f.n_kv_heads;
    if (group > 8 || c.n_draft > kAttnMaxDraft || f.batch > kAttnMaxBatch) return KVBFP_ERR_UNSUPPORTED;
    if (!(c.softmax_scale >= 0.f) || isinf(c.softmax_scale)) return KVBFP_ERR_INVALID_ARG;
    if (c.mod && (!(c.mod->softcap >= 0.f) || isinf(c.mod->softcap) || c.mod->window < 0)) return KVBFP_ERR_INVALID_ARG;
    if (c.mod && c.mod->softcap != 0.f && c.mod->softcap < 1e-20f) return KVBFP_ERR_INVALID_ARG;       // (its inverse has to stay in range)
    const void* ptrs[] = {c.cache->k_mant, c.cache->k_exp, c.cache->v_mant, c.cache->v_exp, c.q, c.out, c.workspace,
                          c.perm_k, c.inv_perm_v, c.mass, c.tree_mask};
    for (const void* p : ptrs)
        if (p && !aligned16(p)) return KVBFP_ERR_ALIGNMENT;
    const int rows = c.n_draft * group;
    const int rows_tile = rows_tile_for(rows, c.dt == KVBFP_BF16), n_row_tiles = (rows + rows_tile - 1) / rows_tile;
    const int64_t n_rows = (int64_t)f.batch * f.n_kv_heads * rows;
    // tile numbers and row numbers are 32-bit
    if ((int64_t)f.batch * f.n_kv_heads * n_row_tiles * (f.max_seq / 32 + 2) >= (int64_t)1 << 31 || n_rows >= (int64_t)1 << 31)
        return KVBFP_ERR_UNSUPPORTED;
    const size_t need = kvbfp_attn_workspace_bytes(&f, c.n_q_heads, c.n_draft, c.with_mass);
    if (!c.workspace || c.workspace_bytes < need) return KVBFP_ERR_WORKSPACE;

    AttnArgs a = {};
    a.fmt = f;
    a.k_mant = c.cache->k_mant; a.k_exp = c.cache->k_exp; a.v_mant = c.cache->v_mant; a.v_exp = c.cache->v_exp;
    a.q = c.q; a.q_is_bf16 = c.dt == KVBFP_BF16; a.n_q_heads = c.n_q_heads; a.group = group; a.n_draft = c.n_draft;
    a.tree = c.tree;
    a.rows_tile = rows_tile; a.n_row_tiles = n_row_tiles; a.part_rows = rows < rows_tile ? rows : rows_tile;
    a.ctx_lens = c.ctx_lens; a.draft_lens = c.draft_lens; a.tree_mask = c.tree_mask; a.depth = c.depth;
    a.perm_k = c.perm_k; a.inv_perm_v = c.inv_perm_v;
    a.scale = c.softmax_scale > 0.f ? c.softmax_scale : 1.0f / sqrtf((float)f.head_dim);
    if (c.mod) {
        // (2^126: so that neither its inverse nor its multiples leave the fp32 range; scores that it would cap are near the end of that range themselves)
        a.softcap = fminf(c.mod->softcap, 0x1p126f); a.window = c.mod->window; a.slopes = c.mod->slopes;
        a.first = c.mod->first; a.prefix = c.mod->prefix;
    }
    a.out = c.out;
    a.mass = c.mass;
    (void)lay_out(f, c.n_q_heads, c.n_draft, c.dt == KVBFP_BF16, c.with_mass, &a, static_cast<uint8_t*>(c.workspace));
    st = status_word(&a.status);
    if (st != KVBFP_OK) return st;
    int n_sm = 0;
    st = sm_count(&n_sm);
    if (st != KVBFP_OK) return st;
    const bool bf16 = c.dt == KVBFP_BF16;
    const bool few = rows_tile == 8;          // attn_rows, else attn_umma
    a.tile = few ? attn_rows_tile(f.mant_bits) : 128;
    a.out_up = few ? 256.f : (float)(1 << (19 - f.mant_bits));      // 2^8 | 2^(17 - (p - 2))
    const int64_t most = (int64_t)f.batch * f.n_kv_heads * n_row_tiles * (f.max_seq / a.tile + 2);    // tiles at the longest
    int64_t grid = (int64_t)n_sm * (few ? attn_rows_blocks(bf16) : 1);
    const int per_block = few ? kAttnWarps : attn_teams(f.mant_bits, rows_tile);      // warps or teams
    if (grid * per_block > max_workers(rows_tile)) grid = max_workers(rows_tile) / per_block;
    if (grid > most) grid = most;
    a.workers = (int)grid * per_block;

    cudaStream_t s = (cudaStream_t)c.stream;
    if (!few) st = f.mant_bits == 4 ? launch_attn_umma4(a, (int)grid, s) : f.mant_bits == 6 ? launch_attn_umma6(a, (int)grid, s) : launch_attn_umma8(a, (int)grid, s);
    else st = f.mant_bits == 4 ? launch_attn_rows4(a, (int)grid, s) : f.mant_bits == 6 ? launch_attn_rows6(a, (int)grid, s) : launch_attn_rows8(a, (int)grid, s);
    if (st != KVBFP_OK) return st;
    // Partials of a row, about: a block per row where they are many (32 heads x 4104 tokens, 55 of them: 19.8 us against 22.7
    // with a warp per row), a warp per row otherwise (16 x 32 x 8192, 16 tokens: 128 us against 140).
    const bool split = a.workers / ((int64_t)f.batch * f.n_kv_heads * n_row_tiles) >= 8;
    if (split) KVBFP_CUDA(launch_pdl(attn_merge<true>, dim3((unsigned)n_rows), dim3(128), 0, s, a, n_rows));
    else KVBFP_CUDA(launch_pdl(attn_merge<false>, dim3((unsigned)((n_rows + 3) / 4)), dim3(128), 0, s, a, n_rows));
    KVBFP_LAUNCH_CHECK("attn_merge");
    if (c.with_mass) {
        const int64_t blocks = (most + 3) / 4;
        KVBFP_CUDA(launch_pdl(attn_mass, dim3((unsigned)(blocks < n_sm * 8 ? blocks : n_sm * 8)), dim3(128), 0, s, a));
        KVBFP_LAUNCH_CHECK("attn_mass");
    }
    return KVBFP_OK;
}

}  // namespace
}  // namespace kvbfp

extern "C" size_t kvbfp_attn_workspace_bytes(const kvbfp_format* fmt, int32_t n_q_heads, int32_t n_draft,
                                             int32_t with_mass) {
    using namespace kvbfp;
    if (check_format(fmt) != KVBFP_OK || n_q_heads < 1 || n_q_heads % fmt->n_kv_heads != 0 || n_draft < 1) return 0;
    if (n_draft > kAttnMaxDraft || n_q_heads / fmt->n_kv_heads > 8) return 0;
    const size_t x = lay_out(*fmt, n_q_heads, n_draft, true, with_mass != 0, nullptr, nullptr);
    const size_t y = lay_out(*fmt, n_q_heads, n_draft, false, with_mass != 0, nullptr, nullptr);
    return x > y ? x : y;
}

extern "C" kvbfp_status kvbfp_tree_attn(const kvbfp_cache* cache, const void* q, kvbfp_dtype dt, int32_t n_q_heads,
                                        int32_t n_draft, const int32_t* ctx_lens, const int32_t* draft_lens,
                                        const uint64_t* tree_mask, const int32_t* depth, const int32_t* perm_k,
                                        const int32_t* inv_perm_v, float softmax_scale, const kvbfp_score_mod* mod,
                                        void* out, void* workspace, size_t workspace_bytes, void* stream) {
    return kvbfp::attn_common({cache, q, dt, n_q_heads, n_draft, 1, ctx_lens, draft_lens, tree_mask, depth, perm_k,
                               inv_perm_v, softmax_scale, mod, nullptr, false, out, workspace, workspace_bytes, stream});
}

extern "C" kvbfp_status kvbfp_decode_attn_mod(const kvbfp_cache* cache, const void* q, kvbfp_dtype dt, int32_t n_q_heads,
                                              const int32_t* seq_lens, const int32_t* perm_k, const int32_t* inv_perm_v,
                                              float softmax_scale, const kvbfp_score_mod* mod, void* out,
                                              void* workspace, size_t workspace_bytes, void* stream) {
    return kvbfp::attn_common({cache, q, dt, n_q_heads, 1, 0, seq_lens, nullptr, nullptr, nullptr, perm_k, inv_perm_v,
                               softmax_scale, mod, nullptr, false, out, workspace, workspace_bytes, stream});
}

extern "C" kvbfp_status kvbfp_decode_attn_mass(const kvbfp_cache* cache, const void* q, kvbfp_dtype dt,
                                               int32_t n_q_heads, const int32_t* seq_lens, const int32_t* perm_k,
                                               const int32_t* inv_perm_v, float softmax_scale,
                                               const kvbfp_score_mod* mod, float* mass, void* out, void* workspace,
                                               size_t workspace_bytes, void* stream) {
    return kvbfp::attn_common({cache, q, dt, n_q_heads, 1, 0, seq_lens, nullptr, nullptr, nullptr, perm_k, inv_perm_v,
                               softmax_scale, mod, mass, true, out, workspace, workspace_bytes, stream});
}
