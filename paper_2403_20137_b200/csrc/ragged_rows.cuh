// Attention of a ragged batch over the packed cache, few query rows per kv head (single tokens, short chunks), and all fp32
// rows: the fragments, conversion and products of attn_rows (attn_rows.cuh: rows as the narrow side of warp-level bf16
// matrix instructions, two groups of 16 tokens at a time), with the split of ragged.cuh, pages, and the causal mask, window
// and first tokens in the place of trees, caps and biases.
//
// Pages.  A tile is copied in pieces of a page (or of the tile where pages are longer), a lane per piece; the piece's page
// number was asked for one tile earlier, so that the copy does not wait for the table.  Pieces that no row sees are not copied:
// what lies there in shared memory is converted all the same (any byte converts to a finite number) and masked.
//
// Weights.  bf16 queries: P in two bf16 terms, hi = P rounded, lo = (P - hi) rounded (2^-16 relative at most, as many bits as
// kvbfp_decode_attn keeps).  Items of up to four rows (TWICE) need no more products for it: the rows stand in the matrix
// instruction's eight columns twice, and the second time P is lo; the columns' results are added at the end.  Items of eight
// rows take a second product.  (One term: 146 and 65 us of the times below, 148 and 66 with TWICE, 164 and 72 with a second product; eight
// 6-bit rows 129, 135.)  fp32 queries: three terms of q and P.
//
// What bounds it: instructions, 357 per warp and 16 tokens, most of them the conversion of fields (integer pipe 56 % busy, issue slots
// 61 %, three warps a scheduler).  16 tokens, 32 heads x 8192, 4 bits, pages of 64: 148 us, 3.8 TB/s; 8 tokens, 8 heads x up to
// 32768, four query heads each, pages of 32: 66 us; one token under a window of 1000: 11.3 us with the merge.  V's words loaded
// before the softmax: no gain (a microsecond off the first, three on top of the second at 8 bits).
#pragma once
#include "attn_rows.cuh"
#include "ragged.cuh"
#include "umma.cuh"

namespace kvbfp {
namespace {

template <int P, bool N16, bool F32, bool TWICE>
__global__ void __launch_bounds__(kAttnWarps * 32, attn_rows_blocks(!F32)) ragged_rows(const RaggedArgs a, const __grid_constant__ CUtensorMap k_map,
                                                                                         const __grid_constant__ CUtensorMap v_map) {
    using G_ = AGeo<P>;
    constexpr int D = kHeadDim, ROW_M = G_::ROW_M, STAGES = G_::STAGES, TILE = G_::TILE, ROWS = TWICE ? 4 : kRows;
    constexpr int SPLIT = F32 ? 3 : 1, TERMS = F32 ? 3 : TWICE ? 1 : 2;      // bf16 terms of q, of P in products of their own
    constexpr int GROUP = 16 * ROW_M;
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ int s_scan[2][kAttnWarps];
    int* s_items = reinterpret_cast<int*>(smem);      // (until the copies begin)
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int row_e = D / a.fmt.block, exp_half = TILE * row_e;
    // mantissa tiles of all warps and stages first (whole swizzle periods), then the exponent bytes, then the rest
    uint8_t* my_m = smem + warp * STAGES * G_::KE_OFF;
    uint8_t* my_e = smem + kAttnWarps * STAGES * G_::KE_OFF + warp * STAGES * 2 * exp_half;
    uint8_t* small = smem + kAttnWarps * STAGES * (G_::KE_OFF + 2 * exp_half) + warp * G_::WARP_SMALL;
    float* orow = reinterpret_cast<float*>(small);
    const uint32_t bar = smem_u32(small + kHeadDim * 4);

    if (lane == 0) {
        for (int s = 0; s < STAGES; ++s) mbar_init(bar + 8 * s, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    pdl_wait();
    ragged_count<kAttnWarps * 32>(a, s_items, s_items + kMaxPagedBatch + 1, s_scan, ROWS, TILE);
    const int H = a.fmt.n_kv_heads, n_items = s_items[a.batch];
    const int workers = min(a.workers, n_items), me = blockIdx.x + gridDim.x * warp;      // neighbouring ranges on different SMs
    const int i0 = me < workers ? worker_start(me, n_items, workers) : 0;
    const int i1 = me < workers ? worker_start(me + 1, n_items, workers) : 0;
    const int n_mine = i1 - i0;
    const int b_first = ragged_find(a, s_items, i0), at_first = i0 - s_items[b_first];
    __syncthreads();
    fence_async_shared();
    if (n_mine <= 0) {
        if (lane == 0 && me < a.workers) a.rec[me] = make_int4(-1, 0, 0, 0);
        pdl_trigger();
        return;
    }
    RaggedCursor cc;
    {
        int before;
        (void)ragged_seek(a, cc, b_first, at_first, ROWS, TILE, before);
    }

    // ---- copies: the same items, STAGES ahead (every lane keeps the cursor; a lane per piece of a tile issues)
    RaggedCursor pc = cc;
    const int sub = a.map.table ? min(TILE, 1 << a.map.shift) : TILE;      // tokens of a piece
    const int pieces = TILE / sub;
    int issued = 0, page = -1;
    auto look_up = [&]() {            // page of the lane's piece of the next tile to copy, -1: not to be copied
        page = -1;
        const int at = ragged_token(pc.v, pc.k, TILE) + lane * sub;
        if (lane < pieces && at <= pc.v.p1 && (a.window == 0 || at + sub > pc.v.p0 - a.window + 1 || at < a.n_sink)) {
            page = token_page(a.map, pc.b, at);
            if (page < 0) raise_flag(a.status, KVBFP_FLAG_POSITION);
        }
    };
    auto issue = [&]() {
        const int s = issued % STAGES;
        const uint32_t br = bar + 8 * s;
        const int at = ragged_token(pc.v, pc.k, TILE) + lane * sub, in = token_row(a.map, at);
        const int rows = min(sub, a.fmt.max_seq - in);              // a multiple of 16
        const uint32_t mant = (P == 6 ? rows : sub) * ROW_M;        // a tiled copy always brings its whole box
        const bool go = page >= 0;
        const uint32_t pieces_here = __popc(__ballot_sync(0xffffffffu, go));
        if (lane == 0) mbar_expect_tx(br, pieces_here * (2 * mant + 2 * rows * row_e));
        __syncwarp();
        if (go) {
            const int64_t row0 = ((int64_t)page * H + pc.hk) * a.fmt.max_seq + in;
            const uint32_t dst = smem_u32(my_m) + s * G_::KE_OFF + lane * sub * ROW_M, de = smem_u32(my_e) + s * 2 * exp_half + lane * sub * row_e;
            if (P == 6) {
                bulk_g2s(dst, a.k_mant + row0 * ROW_M, mant, br);
                bulk_g2s(dst + G_::VM_OFF, a.v_mant + row0 * ROW_M, mant, br);
            } else {
                const int y = (int)(P == 4 ? row0 >> 1 : row0);
                tensor_g2s_2d(dst, &k_map, 0, y, br);
                tensor_g2s_2d(dst + G_::VM_OFF, &v_map, 0, y, br);
            }
            bulk_g2s(de, a.k_exp + row0 * row_e, rows * row_e, br);
            bulk_g2s(de + exp_half, a.v_exp + row0 * row_e, rows * row_e, br);
        }
        ++issued;
        if (++pc.k == pc.v.n) ragged_next(a, pc, ROWS, TILE);
        if (issued < n_mine) look_up();
    };
    look_up();
    for (int s = 0; s < STAGES && issued < n_mine; ++s) issue();

    const float mul = finite_factor(a.scale * kValueUp * 1.4426950408889634f);        // scores to log2 units
    // lane offsets inside a 16-token group: K rows of column g in both score tiles, V rows of the lane's four k positions
    int ko[2], ke[2], vo[4], ve[4];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int row = tok_of<P>(g >> 1, g & 1, j);
        ko[j] = P == 4 ? tile_at<P>(row, 16 * t) : (P == 8 ? row * 128 : tile_at<P>(row, 24 * t));
        ke[j] = row * row_e + (N16 ? 2 * t : (32 * t) / a.fmt.block);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int row = tok_of<P>(t, e & 1, e >> 1);
        vo[e] = G_::VM_OFF + tile_at<P>(row, 2 * P * g);
        ve[e] = exp_half + row * row_e + (16 * g) / a.fmt.block;
    }
    const int kx = (tok_of<P>(g >> 1, g & 1, 0) & 7) << 4;       // 8-bit rows: swizzle of the lane's K rows (both tiles alike)
    int tk[2];            // the lane's tokens of a group: rows g, g + 8 of the scores
#pragma unroll
    for (int j = 0; j < 2; ++j) tk[j] = tok_of<P>(g >> 1, g & 1, j);

    const float rest = !TWICE || t >= 2 ? -1.f : 0.f;         // is the next term what the one before left

    bool dead = false;            // a copy did not arrive: no more waits, no more work, the flag is up
    int it = 0;
    int4 rec = make_int4(-1, 0, 0, 0);
    while (it < n_mine) {
        // ================================================================ a run: tiles [k0, k1) of one entry
        const int b = cc.b, hk = cc.hk, rt = cc.rt, R = cc.s.n * a.group;
        const RaggedView sv = cc.v;
        const int k0 = cc.k, k1 = min(sv.n, k0 + n_mine - it);
        uint4 qr[SPLIT][4];           // k steps 2 i, 2 i + 1
        {
            const int row = rt * ROWS + (TWICE ? g & 3 : g), i = row / a.group;
            const int64_t at = ((int64_t)(cc.s.start + i) * a.n_q_heads + hk * a.group + row - i * a.group) * D;
            const void* q = F32 ? (const void*)(static_cast<const float*>(a.q) + at) : (const void*)(static_cast<const __nv_bfloat16*>(a.q) + at);
            load_q<P, F32>(a, row < R ? q : nullptr, hk, t, qr);
        }
        int pos[2];                   // of rows 2 t, 2 t + 1
#pragma unroll
        for (int e = 0; e < 2; ++e) pos[e] = cc.s.base + min(rt * ROWS + 2 * (TWICE ? t & 1 : t) + e, R - 1) / a.group;

        float o[8][4];                // slots 16 g + 2 i (+ 1: upper pair) of rows 2 t, 2 t + 1
        float m_run[2], l_run[2];     // of rows 2 t, 2 t + 1
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) o[i][k] = 0.f;
        m_run[0] = m_run[1] = -3.4028235e38f;
        l_run[0] = l_run[1] = 0.f;

        for (int k = k0; k < k1; ++k, ++it) {
            const int stage = it % STAGES;
            if (!dead && !mbar_wait_bounded(bar + 8 * stage, (uint32_t)(it / STAGES) & 1u)) dead = true;
            dead = __any_sync(0xffffffffu, dead);
            if (dead) continue;
            const int tt = ragged_token(sv, k, TILE);
            const uint8_t* stm = my_m + stage * G_::KE_OFF;
            const uint8_t* ste = my_e + stage * 2 * exp_half;
#pragma unroll 1
            for (int u = 0; u < TILE / 32; ++u, stm += 2 * GROUP, ste += 32 * row_e) {        // 32 tokens: two groups of 16
                const int tok0 = tt + 32 * u;
                if (tok0 > sv.p1) break;
                // ---- scores: sc[g][0..1] = the lane's first token of group g, rows 2 t, 2 t + 1; sc[g][2..3] = its second
                float sc[2][4];
#pragma unroll
                for (int gr = 0; gr < 2; ++gr) {
                    const uint8_t *gm = stm + gr * GROUP, *ge = ste + gr * 16 * row_e;
                    uint32_t kw[2][P];
                    AW kg[2][N16 ? 2 : 1];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        if (P == 6) {
#pragma unroll
                            for (int i = 0; i < 3; ++i) {
                                const uint2 x = *reinterpret_cast<const uint2*>(gm + ko[j] + 8 * i);
                                kw[j][2 * i] = x.x; kw[j][2 * i + 1] = x.y;
                            }
                        } else {
#pragma unroll
                            for (int i = 0; i < P / 4; ++i) {
                                const uint4 x = *reinterpret_cast<const uint4*>(gm + ko[j] + (P == 8 ? ((32 * t + 16 * i) ^ kx) : 0));
                                kw[j][4 * i] = x.x; kw[j][4 * i + 1] = x.y; kw[j][4 * i + 2] = x.z; kw[j][4 * i + 3] = x.w;
                            }
                        }
#pragma unroll
                        for (int i = 0; i < (N16 ? 2 : 1); ++i) kg[j][i] = aw_make<P>(ge[ke[j] + i] * 0x00010001u);
                    }
                    float s2[4];        // odd k steps: two chains of MMAs
#pragma unroll
                    for (int e = 0; e < 4; ++e) sc[gr][e] = s2[e] = 0.f;
#pragma unroll
                    for (int ks = 0; ks < 8; ks += 2) {
                        uint32_t r[2][4];
#pragma unroll
                        for (int j = 0; j < 2; ++j) attn_k<P>(kw[j], ks, kg[j][N16 ? ks >> 2 : 0], r[j]);
#pragma unroll
                        for (int s = 0; s < SPLIT; ++s) {
                            const uint4 q = qr[s][ks >> 1];
                            mma_bf16(sc[gr], r[0][0], r[1][0], r[0][1], r[1][1], q.x, q.y);
                            mma_bf16(s2, r[0][2], r[1][2], r[0][3], r[1][3], q.z, q.w);
                        }
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) sc[gr][e] += s2[e];
                }
                // ---- masks; mul * sc is the score in log2 units
                const bool clear = tok0 + 31 <= sv.p0 && (a.window == 0 || tok0 > sv.p1 - a.window || tok0 + 32 <= a.n_sink);
                if (!clear) {
#pragma unroll
                    for (int x = 0; x < 8; ++x) {
                        const int tok = tok0 + 16 * (x >> 2) + tk[(x >> 1) & 1], dist = pos[x & 1] - tok;
                        const bool see = dist >= 0 && (a.window == 0 || dist < a.window || tok < a.n_sink);
                        if (!see) sc[x >> 2][x & 3] = -INFINITY;
                    }
                }
                // ---- running softmax: the reference moves only when a score passes it by 8 (2^8 keeps P in range)
                float top[2];
                bool grow = false;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    top[e] = mul * fmaxf(fmaxf(sc[0][e], sc[0][2 + e]), fmaxf(sc[1][e], sc[1][2 + e]));
                    grow |= top[e] > m_run[e] + 8.f;
                }
                if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float x = top[e];
                        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
                        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
                        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
                        x = fmaxf(x, m_run[e]);
                        const float al = ex2_approx(m_run[e] - x);
                        m_run[e] = x;
                        l_run[e] *= al;
#pragma unroll
                        for (int i = 0; i < 8; ++i) { o[i][e] *= al; o[i][2 + e] *= al; }
                    }
                }
#pragma unroll
                for (int gr = 0; gr < 2; ++gr) {
                    const uint8_t *gm = stm + gr * GROUP, *ge = ste + gr * 16 * row_e;
                    // P as B fragments: a token's pair of rows, transposed, in its terms
                    uint32_t pb[TERMS][2];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        float p0 = ex2_approx(fmaf(sc[gr][2 * j], mul, -m_run[0]));
                        float p1 = ex2_approx(fmaf(sc[gr][2 * j + 1], mul, -m_run[1]));
                        l_run[0] += p0;
                        l_run[1] += p1;
#pragma unroll
                        for (int s = 0; s < TERMS; ++s) {
                            uint32_t x = pack_bf16x2_rn(p0, p1);
                            p0 = fmaf(rest, __uint_as_float(x << 16), p0);
                            p1 = fmaf(rest, __uint_as_float(x & 0xffff0000u), p1);
                            if (TWICE) x = pack_bf16x2_rn(p0, p1);
                            pb[s][j] = transpose8(x);
                        }
                    }
                    // ---- V^T . P^T
                    uint32_t vw[4][P / 2], ve8[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {       // k = 2t, 2t+1, 2t+8, 2t+9
                        if (P == 4) {
                            const uint2 x = *reinterpret_cast<const uint2*>(gm + vo[e]);
                            vw[e][0] = x.x; vw[e][1] = x.y;
                        } else if (P == 6) {
#pragma unroll
                            for (int i = 0; i < 3; ++i) vw[e][i] = *reinterpret_cast<const uint32_t*>(gm + vo[e] + 4 * i);
                        } else {
                            const uint4 x = *reinterpret_cast<const uint4*>(gm + vo[e]);
                            vw[e][0] = x.x; vw[e][1] = x.y; vw[e][P / 2 - 2] = x.z; vw[e][P / 2 - 1] = x.w;
                        }
                        ve8[e] = ge[ve[e]];
                    }
                    const AW ga = aw_make<P>(ve8[0] + (ve8[1] << 16)), gb = aw_make<P>(ve8[2] + (ve8[3] << 16));
#pragma unroll
                    for (int r = 0; r < 8; r += 2) {
                        uint32_t xa[4], xb[4];
                        attn_v<P>(vw[0], vw[1], r, ga, xa);
                        attn_v<P>(vw[2], vw[3], r, gb, xb);
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            float (&acc)[4] = o[r + h];          // slots 16 g + 2 (r + h), + 1
                            if (F32) {
                                float d[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                                for (int c = TERMS - 1; c >= 0; --c) mma_bf16(d, xa[2 * h], xa[2 * h + 1], xb[2 * h], xb[2 * h + 1], pb[c][0], pb[c][1]);
                                acc[0] += d[0]; acc[1] += d[1]; acc[2] += d[2]; acc[3] += d[3];
                            } else {
#pragma unroll
                                for (int c = TERMS - 1; c >= 0; --c) mma_bf16(acc, xa[2 * h], xa[2 * h + 1], xb[2 * h], xb[2 * h + 1], pb[c][0], pb[c][1]);
                            }
                        }
                    }
                }
            }
            __syncwarp();                      // every lane has read the stage
            if (issued < n_mine) issue();
        }

        // ---- the run's result: a lane holds slots [16 g, 16 g + 16) of rows 2 t and 2 t + 1 (TWICE: t < 2)
        if (TWICE) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) o[i][k] += __shfl_xor_sync(0xffffffffu, o[i][k], 2);
        }
        const bool whole = k0 == 0 && k1 == sv.n;
        if (k0 > 0 && k1 == sv.n) rec = make_int4(b, rt, hk, worker_of(i0 + it - sv.n, n_items, workers));
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float l = l_run[e];
            l += __shfl_xor_sync(0xffffffffu, l, 4);
            l += __shfl_xor_sync(0xffffffffu, l, 8);
            l += __shfl_xor_sync(0xffffffffu, l, 16);
            const int r = 2 * t + e, row = r < ROWS ? rt * ROWS + r : R;      // (R: none)
            const int i = row / a.group, hq = hk * a.group + row - i * a.group;
            if (!whole) {
                if (row < R) {
                    float* dst = a.partials + ((int64_t)(2 * me + (k0 == 0 ? 1 : 0)) * a.part_rows + r) * kAttnPart;
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        reinterpret_cast<float4*>(dst + 16 * g)[c] = make_float4(o[2 * c][e], o[2 * c][2 + e], o[2 * c + 1][e], o[2 * c + 1][2 + e]);
                    if (g == 0) { dst[D] = m_run[e]; dst[D + 1] = l; }
                }
                continue;
            }
            const bool wanted = row < R && pos[e] >= 0;            // (rows before the first position: zeros, by the merge)
            const float inv = l != 0.f ? kValueUp / l : 0.f;
            float v[16];
#pragma unroll
            for (int s = 0; s < 16; ++s) v[s] = l != 0.f ? o[s >> 1][2 * (s & 1) + e] * inv : 0.f;
            const int64_t at = ((int64_t)(cc.s.start + i) * a.n_q_heads + hq) * D;
            if (!a.inv_perm_v) {
                if (wanted) {
                    if (F32) {
                        float4* to = reinterpret_cast<float4*>(static_cast<float*>(a.out) + at + 16 * g);
#pragma unroll
                        for (int c = 0; c < 4; ++c) to[c] = make_float4(v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]);
                    } else {
                        uint4* to = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.out) + at + 16 * g);
#pragma unroll
                        for (int c = 0; c < 2; ++c)
                            to[c] = make_uint4(pack_bf16x2_rn(v[8 * c], v[8 * c + 1]), pack_bf16x2_rn(v[8 * c + 2], v[8 * c + 3]),
                                               pack_bf16x2_rn(v[8 * c + 4], v[8 * c + 5]), pack_bf16x2_rn(v[8 * c + 6], v[8 * c + 7]));
                    }
                }
            } else {          // channels in their own order: one row at a time through shared memory
                const int32_t* ip = a.inv_perm_v + hk * D;
                int sl[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) sl[c] = ip[4 * lane + c] & (D - 1);
                for (int tt = 0; tt < ROWS / 2; ++tt) {
                    if (rt * ROWS + 2 * tt + e >= R) break;
                    __syncwarp();
                    if (t == tt) {
#pragma unroll
                        for (int s = 0; s < 16; ++s) orow[16 * g + s] = v[s];
                    }
                    __syncwarp();
                    const int64_t to = __shfl_sync(0xffffffffu, at, tt) + 4 * lane;
                    if (!__shfl_sync(0xffffffffu, (int)wanted, tt)) continue;
                    const float y0 = orow[sl[0]], y1 = orow[sl[1]], y2 = orow[sl[2]], y3 = orow[sl[3]];
                    if (F32) *reinterpret_cast<float4*>(static_cast<float*>(a.out) + to) = make_float4(y0, y1, y2, y3);
                    else *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.out) + to) = make_uint2(pack_bf16x2_rn(y0, y1), pack_bf16x2_rn(y2, y3));
                }
                __syncwarp();
            }
        }
        cc.k = k1;
        if (k1 == sv.n) ragged_next(a, cc, ROWS, TILE);
    }
    if (lane == 0) a.rec[me] = rec;
    if (dead) {
        // give the copies still in flight a bounded chance to land before the shared memory is released
        if (lane == 0) raise_flag(a.status, KVBFP_FLAG_WAIT_TIMEOUT);
        for (int s = 0; s < STAGES; ++s) {
            (void)mbar_wait_bounded(bar + 8 * s, 0);
            (void)mbar_wait_bounded(bar + 8 * s, 1);
        }
    }
    pdl_trigger();
}

template <int P, bool N16, bool F32, bool TWICE>
kvbfp_status launch_ragged(const RaggedArgs& a, int grid, cudaStream_t s) {
    auto kernel = ragged_rows<P, N16, F32, TWICE>;
    static std::atomic<bool> attr_set[64];      // per device; setting the attribute twice is harmless
    int dev = 0;
    KVBFP_CUDA(cudaGetDevice(&dev));
    if (dev < 0 || dev >= 64) return KVBFP_ERR_UNSUPPORTED;
    if (!attr_set[dev].load(std::memory_order_acquire)) {
        KVBFP_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, AGeo<P>::smem_bytes(8)));
        attr_set[dev].store(true, std::memory_order_release);
    }
    CUtensorMap k_map = {}, v_map = {};
    if (P != 6) {
        const uint64_t rows = (uint64_t)a.fmt.batch * a.fmt.n_kv_heads * a.fmt.max_seq * P / 8;     // lines of 128 bytes
        const int tile = AGeo<P>::TILE, sub = a.map.table && a.fmt.max_seq < tile ? a.fmt.max_seq : tile;
        kvbfp_status st = make_row_map(&k_map, a.k_mant, rows, 128, sub * P / 8);
        if (st == KVBFP_OK) st = make_row_map(&v_map, a.v_mant, rows, 128, sub * P / 8);
        if (st != KVBFP_OK) return st;
    }
    KVBFP_CUDA(launch_pdl(kernel, dim3(grid), dim3(kAttnWarps * 32), AGeo<P>::smem_bytes(kHeadDim / a.fmt.block), s, a, k_map, v_map));
    KVBFP_LAUNCH_CHECK("ragged_rows");
    return KVBFP_OK;
}

template <int P>
kvbfp_status launch_ragged_p(const RaggedArgs& a, int grid, cudaStream_t s) {
    const bool n16 = a.fmt.block == 16;
    if (!a.q_is_bf16) return n16 ? launch_ragged<P, true, true, false>(a, grid, s) : launch_ragged<P, false, true, false>(a, grid, s);
    if (a.rows_tile == 4) return n16 ? launch_ragged<P, true, false, true>(a, grid, s) : launch_ragged<P, false, false, true>(a, grid, s);
    return n16 ? launch_ragged<P, true, false, false>(a, grid, s) : launch_ragged<P, false, false, false>(a, grid, s);
}

}  // namespace
}  // namespace kvbfp
