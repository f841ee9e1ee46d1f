// Attention of fp32 query rows over the packed cache with warp-level bf16 MMAs, 16 rows of a (batch, kv head) at a time.
//
//   S[rows x tokens] = pi(Q) . K^T ;  y = log2(e) * (cap * tanh(scale * S / cap) - slope * distance) ;  P = 2^(y - m)
//   O[rows x slots] += P . V ;  l += rowsum(P)
//
// Work split.  attn_prep writes, per (sequence, kv head, row tile), pi(q) in fragment order, and the tiles each sequence
// has to read (counted from the real lengths and windows, so ragged batches and windows stay balanced).  attn_rows is
// persistent: all tiles are cut into one contiguous range per warp; a warp walks its range as runs (the tiles of one
// (sequence, head, row tile)), shares nothing with other warps and meets no barrier.  A run that covers all tiles
// writes the result itself, others leave a partial for attn_merge.  The tiles come through a per-warp ring of
// shared-memory stages filled by asynchronous copies that run ahead across run boundaries.
//
// Fragments.  Query rows are the M rows of m16n8k16, so the scores' accumulators are the A fragment of P . V as they
// stand (no shuffles).  K and V are converted in registers: the stored field (an unsigned offset) or-ed under the bits
// of 128.0 is an exact bf16 number, one bf16x2 fma removes the offset and applies the block's power of two (a mantissa
// has at most 7 bits + sign: exact).  The contraction order is free, so a lane's 32-slot chunk of a K row and 16-slot
// chunk of a V row are used in the order they unpack in; the 16 tokens of a tile are dealt to columns so that both the
// K and the V loads touch every bank once (tok_of).
//
// Types.  bf16 queries are exact operands, P is rounded to bf16 (half a step, 2^-9 relative, at random: the output is
// rounded to bf16 too).  fp32 queries are three bf16 terms (24 bits) and P two (16 bits, 2^-17); their O is summed
// outside the MMAs because the tensor cores cut, not round, the running sum.  m, l, O and scores are fp32.
#pragma once
#include "attn_common.cuh"

namespace kvbfp {
namespace {

constexpr int kRows = 16;       // query rows of a work item
constexpr int kSplit = 3;       // bf16 terms of an fp32 operand

// Cached values are carried times 2^-8, so that no exponent byte leaves the bf16 range with the conversion's offset;
// undone on scores and outputs.
constexpr float kValueUp = 256.f;

// Stored fields to bf16 pairs.
template <int P> struct AFmt;
template <> struct AFmt<4> { static constexpr uint32_t mask = 0x000F000Fu, magic = 0x43004300u, bias = 0xC308C308u; };  // -136
template <> struct AFmt<6> { static constexpr uint32_t mask = 0x003F003Fu, magic = 0x43004300u, bias = 0xC320C320u; };  // -160
template <> struct AFmt<8> { static constexpr uint32_t mask = 0x000F000Fu, magic = 0x43004300u, bias = 0xC510C510u; };  // -2304

// bf16 bits of 2^(e8 - 127 - (P-2) - 8); 0 below the smallest subnormal.
template <int P>
__device__ __forceinline__ uint32_t attn_weight(int e8) {
    const int f = e8 - (P - 2) - 8;
    return f >= 1 ? ((uint32_t)f << 7) : (f > -7 ? (0x40u >> (-f)) : 0u);
}

struct AW {
    uint32_t s, c, s16;      // weight pair, -offset * weight, 16 * weight (8-bit fields)
};
template <int P>
__device__ __forceinline__ AW aw_make(uint32_t s, uint32_t c) {
    AW w;
    w.s = s;
    w.c = c;
    w.s16 = (P == 8) ? mul_bf16x2(s, 0x41804180u) : 0u;
    return w;
}
template <int P>
__device__ __forceinline__ uint32_t acvt(uint32_t x, const AW& w) {
    if (P == 8) {
        const uint32_t lo = lop3<0xEA>(x, 0x000F000Fu, 0x43004300u);
        const uint32_t hi = lop3<0xEA>(x >> 4, 0x000F000Fu, 0x43004300u);
        return fma_bf16x2(lo, w.s, fma_bf16x2(hi, w.s16, w.c));
    }
    return fma_bf16x2(lop3<0xEA>(x, AFmt<P>::mask, AFmt<P>::magic), w.s, w.c);
}

// Slot that k position kk (0..3 = k 2t, 2t+1, 2t+8, 2t+9) of k-step ks holds in lane column t.
template <int P>
__device__ __forceinline__ int attn_k_slot(int ks, int t, int kk) {
    if (P == 4) return 32 * t + 8 * (ks >> 1) + 2 * (ks & 1) + (kk >> 1) + 4 * (kk & 1);
    if (P == 8) return 32 * t + 4 * ks + 2 * (kk & 1) + (kk >> 1);
    return 32 * t + 4 * ks + kk;
}
// The four operand registers of k-steps ks, ks + 1 (ks even) from a lane's 32 slots of one K row.
template <int P>
__device__ __forceinline__ void attn_k(const uint32_t (&w)[P], int ks, const AW& wg, uint32_t (&r)[4]) {
    if (P == 4) {
        const uint32_t x = w[ks >> 1];
        r[0] = acvt<4>(x, wg);
        r[1] = acvt<4>(x >> 4, wg);
        r[2] = acvt<4>(x >> 8, wg);
        r[3] = acvt<4>(x >> 12, wg);
    } else if (P == 8) {
        r[0] = acvt<8>(w[ks], wg);
        r[1] = acvt<8>(w[ks] >> 8, wg);
        r[2] = acvt<8>(w[ks + 1], wg);
        r[3] = acvt<8>(w[ks + 1] >> 8, wg);
    } else {
        uint32_t f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int bit = 6 * (4 * ks + j), word = bit >> 5, s = bit & 31;
            f[j] = (s + 6 > 32) ? __funnelshift_r(w[word], w[(word + 1) % P], s) : (w[word] >> s);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) r[j] = acvt<6>(prmt(f[2 * j], f[2 * j + 1], 0x5410u), wg);
    }
}
// Slots 2r .. 2r+3 (r even) of a lane's 16-slot chunks of two V rows: (slot, row a | row b) pairs.
template <int P>
__device__ __forceinline__ void attn_v(const uint32_t* wa, const uint32_t* wb, int r, const AW& wg, uint32_t (&o)[4]) {
    if (P == 4) {
        const uint32_t x = prmt(wa[r >> 2], wb[r >> 2], ((r >> 1) & 1) ? 0x7632u : 0x5410u);
        o[0] = acvt<4>(x, wg);
        o[1] = acvt<4>(x >> 4, wg);
        o[2] = acvt<4>(x >> 8, wg);
        o[3] = acvt<4>(x >> 12, wg);
    } else if (P == 8) {
        const uint32_t xl = prmt(wa[r >> 1], wb[r >> 1], 0x5410u), xh = prmt(wa[r >> 1], wb[r >> 1], 0x7632u);
        o[0] = acvt<8>(xl, wg);
        o[1] = acvt<8>(xl >> 8, wg);
        o[2] = acvt<8>(xh, wg);
        o[3] = acvt<8>(xh >> 8, wg);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int bit = 6 * (2 * r + j), word = bit >> 5, s = bit & 31;
            const uint32_t fa = (s + 6 > 32) ? __funnelshift_r(wa[word], wa[(word + 1) % 3], s) : (wa[word] >> s);
            const uint32_t fb = (s + 6 > 32) ? __funnelshift_r(wb[word], wb[(word + 1) % 3], s) : (wb[word] >> s);
            o[j] = acvt<6>(prmt(fa, fb, 0x5410u), wg);
        }
    }
}

// Token (0..15 of a 16-token group) in column 2t + e of the j-th 8-column score tile.  Chosen per row size so that a
// lane's K row (column g) and V rows (columns of lane t) are read without bank conflicts: rows of 64 bytes lie two to a
// swizzled 128-byte line, rows of 128 bytes one, rows of 96 bytes follow each other unswizzled.
template <int P>
__device__ __forceinline__ int tok_of(int t, int e, int j) {
    if (P == 4) return (t & 1) + 4 * (t >> 1) + 8 * e + 2 * j;
    if (P == 6) return ((t + 2 * e) & 3) + 4 * (e + 2 * j);
    return 2 * t + e + 8 * j;
}
// Byte offset of the piece at byte `x` of row `row` (0..15) of a 16-row group; groups follow each other 16 rows on.
template <int P>
__device__ __forceinline__ int tile_at(int row, int x) {
    if (P == 4) {
        const int line = row >> 1, p = ((row & 1) << 6) + x;
        return line * 128 + (p ^ ((line & 7) << 4));
    }
    if (P == 8) return row * 128 + (x ^ ((row & 7) << 4));
    return row * 96 + x;
}

// Query fragments of one (sequence, kv head, row tile) per block.
template <int P>
__global__ void __launch_bounds__(128) attn_prep(const AttnArgs a) {
    __shared__ float sq[kRows][kHeadDim + 4];
    __shared__ int sp[kHeadDim];
    prep_common<kRows, true>(a, sq, sp);
    const int tid = threadIdx.x, x0 = blockIdx.x;
    uint4* to = a.qfrag + (int64_t)x0 * (kSplit * 8 * 32);
#pragma unroll
    for (int x = tid; x < 8 * 32; x += 128) {
        const int ln = x & 31, ks = x >> 5, g = ln >> 2, t = ln & 3;
        uint32_t reg[kSplit][4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {       // row g | g + 8, k positions 0, 1 | 2, 3
            const float* row = sq[g + 8 * (k & 1)];
            float v0 = row[sp[attn_k_slot<P>(ks, t, (k & 2))]], v1 = row[sp[attn_k_slot<P>(ks, t, (k & 2) + 1)]];
#pragma unroll
            for (int s = 0; s < kSplit; ++s) {
                reg[s][k] = pack_bf16x2_rn(v0, v1);
                v0 -= __uint_as_float(reg[s][k] << 16);
                v1 -= __uint_as_float(reg[s][k] & 0xffff0000u);
            }
        }
#pragma unroll
        for (int s = 0; s < kSplit; ++s) to[s * 256 + x] = make_uint4(reg[s][0], reg[s][1], reg[s][2], reg[s][3]);
    }
}

template <int P>
struct AGeo {
    static constexpr int ROW_M = kHeadDim * P / 8;
    static constexpr int TILE = attn_rows_tile(P);       // tokens per stage
    static constexpr int STAGES = 2;
    static constexpr int VM_OFF = TILE * ROW_M, KE_OFF = 2 * VM_OFF;
    // exponent bytes of a stage: 2 * TILE * row_e, the stage rounded up to the swizzle's 1024 bytes for the tiled copies
    __host__ __device__ static int exp_bytes(int row_e) { return 2 * TILE * row_e; }
    static constexpr int LUT_BYTES = 256 * 8;
    static constexpr int WARP_SMALL = STAGES * 8 + 32 * 16 + kAttnMaxDraft * 4;    // barriers, rows (one output row at the end of a run), positions
    __host__ __device__ static int smem_bytes(int row_e) {
        return kAttnWarps * STAGES * (KE_OFF + exp_bytes(row_e)) + LUT_BYTES + kAttnWarps * WARP_SMALL;
    }
};

template <int P, bool N16>
__global__ void __launch_bounds__(kAttnWarps * 32, 2) attn_rows(const AttnArgs a, const __grid_constant__ CUtensorMap k_map,
                                                                   const __grid_constant__ CUtensorMap v_map) {
    using G_ = AGeo<P>;
    constexpr int D = kHeadDim, ROW_M = G_::ROW_M, STAGES = G_::STAGES, TILE = G_::TILE, ROWS = kRows;
    constexpr int GROUP = 16 * ROW_M;
    extern __shared__ __align__(1024) uint8_t smem[];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int row_e = D / a.fmt.block, exp_half = TILE * row_e;
    // mantissa tiles of all warps and stages first (whole swizzle periods), then the exponent bytes, then the rest
    uint8_t* my_m = smem + warp * STAGES * G_::KE_OFF;
    uint8_t* my_e = smem + kAttnWarps * STAGES * G_::KE_OFF + warp * STAGES * 2 * exp_half;
    uint8_t* rest = smem + kAttnWarps * STAGES * (G_::KE_OFF + 2 * exp_half);
    uint2* lut = reinterpret_cast<uint2*>(rest);
    uint8_t* small = rest + G_::LUT_BYTES + warp * G_::WARP_SMALL;
    RowInfo* ri = reinterpret_cast<RowInfo*>(small);
    float* orow = reinterpret_cast<float*>(small);
    int* dpos = reinterpret_cast<int*>(small + 32 * 16);
    const uint32_t bar = smem_u32(small + 32 * 16 + kAttnMaxDraft * 4);

    for (int e = tid; e < 256; e += kAttnWarps * 32) {
        const uint32_t s2 = attn_weight<P>(e) * 0x00010001u;
        lut[e] = make_uint2(s2, mul_bf16x2(s2, AFmt<P>::bias));
    }
    if (lane == 0) {
        for (int s = 0; s < STAGES; ++s) mbar_init(bar + 8 * s, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncthreads();
    pdl_wait();       // what attn_prep wrote is read by plain loads below: read-only ones could be moved above this line

    const int B = a.fmt.batch, Hkv = a.fmt.n_kv_heads, HR = Hkv * a.n_row_tiles, max_seq = a.fmt.max_seq;
    const int n_items = a.plan[B] * HR;
    const int workers = min(a.workers, n_items), me = blockIdx.x + gridDim.x * warp;      // neighbouring ranges on different SMs
    const int i0 = me < workers ? worker_start(me, n_items, workers) : 0;
    const int i1 = me < workers ? worker_start(me + 1, n_items, workers) : 0;
    const int n_mine = i1 - i0;
    if (n_mine <= 0) {
        pdl_trigger();
        return;
    }
    struct Cursor {      // an item: sequence, kv head and row tile (hr), tile k of n
        int b, hr, k, n;
    };
    Cursor cc;
    {
        // last sequence that begins at or before the item and has tiles: 32 looked at per step
        int last = 0;
        for (int b0 = 0; b0 < B; b0 += 32) {
            const bool in = b0 + lane < B && a.plan[b0 + lane] * HR <= i0;
            const uint32_t v = __ballot_sync(0xffffffffu, in);
            if (v) last = b0 + 31 - __clz(v);
            if (v != 0xffffffffu) break;
        }
        const int c0 = a.plan[last];
        cc.b = last;
        cc.n = a.plan[last + 1] - c0;
        const int in = i0 - c0 * HR;
        cc.hr = in / cc.n;
        cc.k = in - cc.hr * cc.n;
    }
    auto next_pair = [&](Cursor& c) {           // to the first tile of the next (sequence, head, row tile)
        c.k = 0;
        if (++c.hr == HR) {
            c.hr = 0;
            c.n = 0;
            while (c.n == 0 && ++c.b < B) c.n = a.plan[c.b + 1] - a.plan[c.b];
        }
    };
    auto view = [&](int b) {
        const int4 x = reinterpret_cast<const int4*>(a.views + b)[0], y = reinterpret_cast<const int4*>(a.views + b)[1];
        SeqView s;
        s.ctx = x.x; s.nd = x.y; s.first = x.z; s.pf = x.w; s.lo = y.x; s.np = y.y; s.n = y.z; s.clamped = y.w;
        return s;
    };

    // ---- copies: the same items, STAGES ahead (every lane keeps the cursor, lane 0 issues)
    Cursor pc = cc;
    SeqView psv = view(pc.b);
    int issued = 0;
    auto issue = [&]() {
        const int s = issued % STAGES;
        if (lane == 0) {
            const int tt = tile_token(psv, pc.k, TILE);
            const int64_t row0 = ((int64_t)pc.b * Hkv + pc.hr / a.n_row_tiles) * max_seq + tt;
            const int rows = min(TILE, max_seq - tt);           // a multiple of 16
            const uint32_t dst = smem_u32(my_m) + s * G_::KE_OFF, de = smem_u32(my_e) + s * 2 * exp_half, br = bar + 8 * s;
            const uint32_t mant = (P == 6 ? rows : TILE) * ROW_M;       // a tiled copy always brings its whole box
            mbar_expect_tx(br, 2 * mant + 2 * rows * row_e);
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
        if (++pc.k == pc.n) {
            const int b = pc.b;
            next_pair(pc);
            if (pc.b != b && pc.b < B) psv = view(pc.b);
        }
    };
    for (int s = 0; s < STAGES && issued < n_mine; ++s) issue();

    const int R = a.n_draft * a.group;
    const float up = a.scale * kValueUp, to_log2 = 1.4426950408889634f, plain = up * to_log2;
    const float cap_in = a.softcap > 0.f ? up / a.softcap : 0.f;
    const bool reshape = a.softcap > 0.f || a.slopes != nullptr;
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

    bool dead = false;            // a copy did not arrive: no more waits, no more work, the flag is up
    int it = 0;
    while (it < n_mine) {
        // ================================================================ a run: tiles [k0, k1) of one (b, head, row tile)
        const int b = cc.b, hk = cc.hr / a.n_row_tiles, rt = cc.hr - hk * a.n_row_tiles;
        const int k0 = cc.k, k1 = min(cc.n, k0 + n_mine - it);
        const SeqView sv = view(b);
        const int64_t item = (int64_t)b * HR + cc.hr;
        uint4 qr[kSplit][8];
        {
            const uint4* src = a.qfrag + item * (kSplit * 256) + lane;
#pragma unroll
            for (int s = 0; s < kSplit; ++s)
#pragma unroll
                for (int ks = 0; ks < 8; ++ks) qr[s][ks] = src[(s * 8 + ks) * 32];
        }
        __syncwarp();
        if (lane < ROWS) reinterpret_cast<uint4*>(ri)[lane] = reinterpret_cast<const uint4*>(a.rows)[item * ROWS + lane];
        if (a.tree) {
            dpos[lane] = a.dpos[b * kAttnMaxDraft + lane];
            dpos[lane + 32] = a.dpos[b * kAttnMaxDraft + lane + 32];
        }
        __syncwarp();

        float o[16][4];
        float m_run[2], l_run[2];
        {
#pragma unroll
            for (int s = 0; s < 16; ++s)
#pragma unroll
                for (int k = 0; k < 4; ++k) o[s][k] = 0.f;
            m_run[0] = m_run[1] = -3.4028235e38f;
            l_run[0] = l_run[1] = 0.f;
        }
        // tokens [clear_lo, ctx) and [0, pf) are visible to every row
        int clear_lo = sv.first;
        if (a.window > 0) clear_lo = max(clear_lo, sv.ctx + (a.tree ? a.n_draft - 1 : -1) - a.window + 1);
        const int end = sv.ctx + sv.nd;

        for (int k = k0; k < k1; ++k, ++it) {
            const int stage = it % STAGES;
            if (!dead && !mbar_wait_bounded(bar + 8 * stage, (uint32_t)(it / STAGES) & 1u)) dead = true;
            dead = __any_sync(0xffffffffu, dead);
            if (dead) continue;
            const int tt = tile_token(sv, k, TILE);
            const uint8_t* stm = my_m + stage * G_::KE_OFF;
            const uint8_t* ste = my_e + stage * 2 * exp_half;
#pragma unroll 1
            for (int u = 0; u < TILE / 16; ++u, stm += GROUP, ste += 16 * row_e) {
                const int tok0 = tt + 16 * u;
                if (tok0 >= end) break;
                // ---- scores of 16 tokens: sc[m tile][column tile][...]
                float sc[2][4];
                {
                    float s2[2][4];        // odd k steps: two chains of MMAs per column tile
                    uint32_t kw[2][P];
                    AW kg[2][N16 ? 2 : 1];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        if (P == 6) {
#pragma unroll
                            for (int i = 0; i < 3; ++i) {
                                const uint2 x = *reinterpret_cast<const uint2*>(stm + ko[j] + 8 * i);
                                kw[j][2 * i] = x.x; kw[j][2 * i + 1] = x.y;
                            }
                        } else {
#pragma unroll
                            for (int i = 0; i < P / 4; ++i) {
                                const uint4 x = *reinterpret_cast<const uint4*>(stm + ko[j] + (P == 8 ? ((32 * t + 16 * i) ^ kx) : 0));
                                kw[j][4 * i] = x.x; kw[j][4 * i + 1] = x.y; kw[j][4 * i + 2] = x.z; kw[j][4 * i + 3] = x.w;
                            }
                        }
#pragma unroll
                        for (int i = 0; i < (N16 ? 2 : 1); ++i) {
                            const uint2 l = lut[ste[ke[j] + i]];
                            kg[j][i] = aw_make<P>(l.x, l.y);
                        }
                    }
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) sc[j][e] = s2[j][e] = 0.f;
#pragma unroll
                    for (int ks = 0; ks < 8; ks += 2) {
                        uint32_t r[2][4];
#pragma unroll
                        for (int j = 0; j < 2; ++j) attn_k<P>(kw[j], ks, kg[j][N16 ? ks >> 2 : 0], r[j]);
#pragma unroll
                        for (int s = 0; s < kSplit; ++s)
                            {
                                const uint4 q0 = qr[s][ks], q1 = qr[s][ks + 1];
#pragma unroll
                                for (int j = 0; j < 2; ++j) mma_bf16(sc[j], q0.x, q0.y, q0.z, q0.w, r[j][0], r[j][1]);
#pragma unroll
                                for (int j = 0; j < 2; ++j) mma_bf16(s2[j], q1.x, q1.y, q1.z, q1.w, r[j][2], r[j][3]);
                            }
                    }
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) sc[j][e] += s2[j][e];
                }
                // ---- cap, bias, masks: y = mul * sc in log2 units; tiles that every row sees whole need only the factor
                float mul = plain;
                if (reshape || !(tok0 + 16 <= sv.ctx && (tok0 >= clear_lo || tok0 + 16 <= sv.pf))) {
                    mul = 1.f;
#pragma unroll
                    for (int hh = 0; hh < 2; ++hh) {
                        const RowInfo x = ri[g + 8 * hh];
#pragma unroll
                        for (int j = 0; j < 2; ++j)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                float y = sc[j][2 * hh + e];
                                if (a.softcap > 0.f) {
                                    y *= cap_in;
                                    y = a.softcap * tanhf(y);
                                } else {
                                    y *= up;
                                }
                                const int tok = tok0 + tok_of<P>(t, e, j);
                                bool see;
                                int dist;
                                if (tok < sv.ctx) {
                                    dist = x.pos - tok;
                                    see = (tok >= sv.first && (a.window == 0 || dist < a.window)) || tok < sv.pf;
                                } else {
                                    const int jd = tok - sv.ctx;
                                    const bool in = jd < sv.nd;
                                    dist = x.pos - dpos[in ? jd : 0];
                                    see = in && (((jd < 32 ? x.m0 >> (jd & 31) : x.m1 >> (jd & 31)) & 1u) != 0u) &&
                                    (a.window == 0 || dist < a.window);
                                }
                                y = (y - x.slope * (float)dist) * to_log2;
                                sc[j][2 * hh + e] = see ? y : -INFINITY;
                            }
                    }
                }
                if (a.scores) {
#pragma unroll
                    for (int hh = 0; hh < 2; ++hh) {
                        const int row = rt * ROWS + g + 8 * hh;
                        if (row < R) {
                            float* to = a.scores + ((int64_t)b * a.n_q_heads + hk * a.group + row) * max_seq + tok0;
#pragma unroll
                            for (int j = 0; j < 2; ++j)
#pragma unroll
                                for (int e = 0; e < 2; ++e) to[tok_of<P>(t, e, j)] = sc[j][2 * hh + e] * mul;
                        }
                    }
                }
                // ---- running softmax: the reference moves only when a score passes it by 8 (2^8 keeps P in range)
                float top[2];
                bool grow = false;
#pragma unroll
                for (int hh = 0; hh < 2; ++hh) {
                    const float x = mul * fmaxf(fmaxf(sc[0][2 * hh], sc[0][2 * hh + 1]),
                                                fmaxf(sc[1][2 * hh], sc[1][2 * hh + 1]));
                    top[hh] = x;
                    grow |= x > m_run[hh] + 8.f;
                }
                if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
                    for (int hh = 0; hh < 2; ++hh) {
                        float x = top[hh];
                        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
                        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
                        x = fmaxf(x, m_run[hh]);
                        const float al = ex2_approx(m_run[hh] - x);
                        m_run[hh] = x;
                        l_run[hh] *= al;
#pragma unroll
                        for (int s = 0; s < 16; ++s) { o[s][2 * hh] *= al; o[s][2 * hh + 1] *= al; }
                    }
                }
                // P as A fragments: (row g, tile 0), (row g+8, tile 0), (row g, tile 1), (row g+8, tile 1); fp32: three terms
                uint32_t pa[kSplit][4];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int hh = x & 1, j = x >> 1;
                    float p0 = ex2_approx(fmaf(sc[j][2 * hh], mul, -m_run[hh]));
                    float p1 = ex2_approx(fmaf(sc[j][2 * hh + 1], mul, -m_run[hh]));
                    l_run[hh] += p0 + p1;
#pragma unroll
                    for (int s = 0; s < kSplit; ++s) {
                        pa[s][x] = pack_bf16x2_rn(p0, p1);
                        p0 -= __uint_as_float(pa[s][x] << 16);
                        p1 -= __uint_as_float(pa[s][x] & 0xffff0000u);
                    }
                }
                // ---- P . V
                uint32_t vw[4][P / 2];
                uint2 lv[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {       // k = 2t, 2t+1, 2t+8, 2t+9
                    if (P == 4) {
                        const uint2 x = *reinterpret_cast<const uint2*>(stm + vo[e]);
                        vw[e][0] = x.x; vw[e][1] = x.y;
                    } else if (P == 6) {
#pragma unroll
                        for (int i = 0; i < 3; ++i) vw[e][i] = *reinterpret_cast<const uint32_t*>(stm + vo[e] + 4 * i);
                    } else {
                        const uint4 x = *reinterpret_cast<const uint4*>(stm + vo[e]);
                        vw[e][0] = x.x; vw[e][1] = x.y; vw[e][P / 2 - 2] = x.z; vw[e][P / 2 - 1] = x.w;
                    }
                    lv[e] = lut[ste[ve[e]]];
                }
                const AW ga = aw_make<P>(prmt(lv[0].x, lv[1].x, 0x7610u), prmt(lv[0].y, lv[1].y, 0x7610u));
                const AW gb = aw_make<P>(prmt(lv[2].x, lv[3].x, 0x7610u), prmt(lv[2].y, lv[3].y, 0x7610u));
#pragma unroll
                for (int r = 0; r < 8; r += 2) {
                    uint32_t xa[4], xb[4];
                    attn_v<P>(vw[0], vw[1], r, ga, xa);
                    attn_v<P>(vw[2], vw[3], r, gb, xb);
#pragma unroll
                    for (int s = 0; s < 4; ++s) {
                        float (&acc)[4] = o[2 * r + s];
                        float d[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int c = 2; c >= 0; --c) {
                            const uint32_t (&p)[4] = pa[c];
                            mma_bf16(d, p[0], p[1], p[2], p[3], xa[s], xb[s]);
                        }
                        acc[0] += d[0]; acc[1] += d[1]; acc[2] += d[2]; acc[3] += d[3];
                    }
                }
            }
            __syncwarp();                      // every lane has read the stage
            if (issued < n_mine) issue();
        }

        // ---- the run's result: a lane holds slots [32t, 32t + 32) of rows g and g + 8 of each m tile
        const bool whole = k0 == 0 && k1 == cc.n;
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
            float l = l_run[hh];
            l += __shfl_xor_sync(0xffffffffu, l, 1);
            l += __shfl_xor_sync(0xffffffffu, l, 2);
            const int r = g + 8 * hh, row = rt * ROWS + r;
            const int i = row / a.group, hq = hk * a.group + row - i * a.group;
            const float m = m_run[hh];
            if (!whole) {
                if (row < R) {
                    float* dst = a.partials + ((int64_t)(2 * me + (k0 == 0 ? 1 : 0)) * a.part_rows + r) * kAttnPart;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        reinterpret_cast<float4*>(dst + 32 * t)[c] = make_float4(o[4 * c][2 * hh], o[4 * c + 1][2 * hh], o[4 * c + 2][2 * hh], o[4 * c + 3][2 * hh]);
                        reinterpret_cast<float4*>(dst + 32 * t + 16)[c] = make_float4(o[4 * c][2 * hh + 1], o[4 * c + 1][2 * hh + 1], o[4 * c + 2][2 * hh + 1], o[4 * c + 3][2 * hh + 1]);
                    }
                    if (t == 0) { dst[D] = m; dst[D + 1] = l; }
                }
                continue;
            }
            const bool live = row < R && (!a.tree || i < sv.nd) && l != 0.f;
            const float inv = live ? kValueUp / l : 0.f;
            float v[2][16];
#pragma unroll
            for (int s = 0; s < 16; ++s)
#pragma unroll
                for (int e = 0; e < 2; ++e) v[e][s] = live ? o[s][2 * hh + e] * inv : 0.f;
            const int64_t at = (((int64_t)b * a.n_draft + i) * a.n_q_heads + hq) * D;
            if (a.lse && row < R && t == 0) a.lse[(int64_t)b * a.n_q_heads + hq] = l > 0.f ? m + log2f(l) : (l == 0.f ? INFINITY : l);
            if (!a.inv_perm_v) {
                if (row < R) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float4* to = reinterpret_cast<float4*>(static_cast<float*>(a.out) + at + 32 * t + 16 * e);
#pragma unroll
                        for (int c = 0; c < 4; ++c) to[c] = make_float4(v[e][4 * c], v[e][4 * c + 1], v[e][4 * c + 2], v[e][4 * c + 3]);
                    }
                }
            } else {          // channels in their own order: one row at a time through shared memory
                const int32_t* ip = a.inv_perm_v + hk * D;
                int sl[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) sl[e] = ip[4 * lane + e] & (D - 1);
                for (int gg = 0; gg < 8; ++gg) {
                    if (rt * ROWS + gg + 8 * hh >= R) break;
                    __syncwarp();
                    if (g == gg) {
#pragma unroll
                        for (int s = 0; s < 16; ++s) { orow[32 * t + s] = v[0][s]; orow[32 * t + 16 + s] = v[1][s]; }
                    }
                    __syncwarp();
                    const int64_t to = __shfl_sync(0xffffffffu, at, gg * 4) + 4 * lane;
                    const float y0 = orow[sl[0]], y1 = orow[sl[1]], y2 = orow[sl[2]], y3 = orow[sl[3]];
                    *reinterpret_cast<float4*>(static_cast<float*>(a.out) + to) = make_float4(y0, y1, y2, y3);
                }
            }
        }
        cc.k = k1;
        if (k1 == cc.n) next_pair(cc);
    }
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

template <int P, bool N16>
kvbfp_status launch_attn(const AttnArgs& a, int grid, cudaStream_t s) {
    auto kernel = attn_rows<P, N16>;
    static std::atomic<bool> attr_set[64];      // per device; setting the attribute twice is harmless
    int dev = 0;
    KVBFP_CUDA(cudaGetDevice(&dev));
    if (dev < 0 || dev >= 64) return KVBFP_ERR_UNSUPPORTED;
    if (!attr_set[dev].load(std::memory_order_acquire)) {
        KVBFP_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, AGeo<P>::smem_bytes(8)));
        attr_set[dev].store(true, std::memory_order_release);
    }
    CUtensorMap k_map, v_map;
    if (P != 6) {
        const uint64_t rows = (uint64_t)a.fmt.batch * a.fmt.n_kv_heads * a.fmt.max_seq * P / 8;     // lines of 128 bytes
        kvbfp_status st = make_row_map(&k_map, a.k_mant, rows, 128, AGeo<P>::TILE * P / 8);
        if (st == KVBFP_OK) st = make_row_map(&v_map, a.v_mant, rows, 128, AGeo<P>::TILE * P / 8);
        if (st != KVBFP_OK) return st;
    }
    KVBFP_CUDA(launch_pdl(attn_prep<P>, dim3(a.fmt.batch * a.fmt.n_kv_heads * a.n_row_tiles), dim3(128), 0, s, a));
    KVBFP_LAUNCH_CHECK("attn_prep");
    KVBFP_CUDA(launch_pdl(kernel, dim3(grid), dim3(kAttnWarps * 32), AGeo<P>::smem_bytes(kHeadDim / a.fmt.block), s, a, k_map, v_map));
    KVBFP_LAUNCH_CHECK("attn_rows");
    return KVBFP_OK;
}

template <int P>
kvbfp_status launch_attn_p(const AttnArgs& a, int grid, cudaStream_t s) {
    return a.fmt.block == 16 ? launch_attn<P, true>(a, grid, s) : launch_attn<P, false>(a, grid, s);
}

}  // namespace
}  // namespace kvbfp
