// Attention of up to 64 query rows per (batch, kv head) over the packed cache with warp-level bf16 MMAs.
//
//   S[rows x tokens] = pi(Q) . K^T ;  y = log2(e) * (cap * tanh(scale * S / cap) - slope * distance) ;  P = 2^(y - m)
//   O[rows x slots] += P . V ;  l += rowsum(P)
//
// Work split.  Persistent thread blocks; all 128-token tiles of all (sequence, kv head, row tile) are cut into one
// contiguous range per block, counted on the device from the real lengths and windows, so ragged batches and windows
// stay balanced.  A block walks its range as runs (the tiles of one (sequence, head, row tile)); a run that covers all
// tiles writes the result itself, others leave a partial for attn_merge.  The tiles come through a ring of
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
#include <math.h>

#include <atomic>

#include "attn.cuh"
#include "ptx.cuh"

namespace kvbfp {
namespace {

constexpr int kAW = 4;      // warps per thread block

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
// Byte offset of 16-byte-or-smaller piece at byte `x` of row `row` in a staged tile.
template <int P>
__device__ __forceinline__ int tile_at(int row, int x) {
    if (P == 4) {
        const int line = row >> 1, p = ((row & 1) << 6) + x;
        return line * 128 + (p ^ ((line & 7) << 4));
    }
    if (P == 8) return row * 128 + (x ^ ((row & 7) << 4));
    return row * 96 + x;
}

struct RowInfo {
    int pos;           // position of the query row's token
    float slope;
    uint32_t m0, m1;   // drafted tokens it sees (all clear for rows that do not exist)
};

template <int P, int MT, int RG, bool F32>
struct AGeo {
    static constexpr int ROW_M = kHeadDim * P / 8;
    static constexpr int STAGES = (P == 8) ? 2 : 3;
    static constexpr int VM_OFF = kAttnTile * ROW_M;
    static constexpr int KE_OFF = 2 * kAttnTile * ROW_M;
    static constexpr int VE_OFF = KE_OFF + kAttnTile * 8;
    static constexpr int STAGE_BYTES = VE_OFF + kAttnTile * 8;       // a multiple of 1024
    static constexpr int ROWS = 16 * MT * RG;
    static constexpr int QSPLIT = F32 ? 3 : 1;
    static constexpr int OSTRIDE = kHeadDim + 8;
    static constexpr int QF_OFF = STAGES * STAGE_BYTES;
    static constexpr int O_OFF = QF_OFF + QSPLIT * MT * RG * 8 * 512;
    static constexpr int ML_OFF = O_OFF + ROWS * OSTRIDE * 4;        // per (token group, row): max, sum
    static constexpr int RI_OFF = ML_OFF + (kAW / RG) * ROWS * 8;
    static constexpr int DP_OFF = RI_OFF + ROWS * 16;                // positions of the drafted rows
    static constexpr int LUT_OFF = DP_OFF + kAttnMaxDraft * 4;
    static constexpr int BAR_OFF = LUT_OFF + 256 * 8;
    static constexpr int SCAN_OFF = BAR_OFF + 2 * STAGES * 8;
    static constexpr int CUM_OFF = SCAN_OFF + kAW * 32 * 4;
    static int smem_bytes(int batch) { return CUM_OFF + (batch + 1) * 4 + 1024; }    // + alignment of the base
};

template <int P, int MT, int RG, bool F32>
__global__ void __launch_bounds__(kAW * 32, 2) attn_rows(const AttnArgs a, const __grid_constant__ CUtensorMap k_map,
                                                         const __grid_constant__ CUtensorMap v_map) {
    using G_ = AGeo<P, MT, RG, F32>;
    constexpr int D = kHeadDim, ROW_M = G_::ROW_M, STAGES = G_::STAGES, TG = kAW / RG, ROWS = G_::ROWS;
    constexpr bool Q_REGS = MT == 1 && !F32;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int rg = warp % RG, tg = warp / RG;

    uint4* qf = reinterpret_cast<uint4*>(smem + G_::QF_OFF);
    float* ob = reinterpret_cast<float*>(smem + G_::O_OFF);
    float2* ml = reinterpret_cast<float2*>(smem + G_::ML_OFF);
    RowInfo* ri = reinterpret_cast<RowInfo*>(smem + G_::RI_OFF);
    int* dpos = reinterpret_cast<int*>(smem + G_::DP_OFF);
    uint2* lut = reinterpret_cast<uint2*>(smem + G_::LUT_OFF);
    int* scan = reinterpret_cast<int*>(smem + G_::SCAN_OFF);
    int* cum = reinterpret_cast<int*>(smem + G_::CUM_OFF);
    const uint32_t bar_full = smem_u32(smem + G_::BAR_OFF), bar_empty = bar_full + 8 * STAGES;

    for (int e = tid; e < 256; e += kAW * 32) {
        const uint32_t s2 = attn_weight<P>(e) * 0x00010001u;
        lut[e] = make_uint2(s2, mul_bf16x2(s2, AFmt<P>::bias));
    }
    if (tid == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(bar_full + 8 * s, 1);
            mbar_init(bar_empty + 8 * s, kAW);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    pdl_wait();

    // ---- tiles per sequence, summed over the batch
    const int B = a.fmt.batch, Hkv = a.fmt.n_kv_heads, HR = Hkv * a.n_row_tiles, max_seq = a.fmt.max_seq;
    {
        const int per = (B + kAW * 32 - 1) / (kAW * 32);
        int mine = 0;
        for (int i = 0; i < per; ++i) {
            const int b = tid * per + i;
            if (b < B) mine += seq_view(a, b).n;
        }
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
            const int b = tid * per + i;
            if (b < B) {
                cum[b] = before;
                const SeqView sv = seq_view(a, b);
                before += sv.n;
                if (b == B - 1) cum[B] = before;
                if (sv.clamped && blockIdx.x == 0) raise_flag(a.status, KVBFP_FLAG_POSITION);
            }
        }
        __syncthreads();
        if (blockIdx.x == 0)
            for (int b = tid; b <= B; b += kAW * 32) a.plan[b] = cum[b];
    }
    const int n_items = cum[B] * HR;
    const int workers = min(a.workers, n_items);
    const int i0 = (int)blockIdx.x < workers ? worker_start(blockIdx.x, n_items, workers) : 0;
    const int i1 = (int)blockIdx.x < workers ? worker_start(blockIdx.x + 1, n_items, workers) : 0;
    const int n_mine = i1 - i0;
    if (n_mine <= 0) {
        pdl_trigger();
        return;
    }
    struct Cursor {      // an item: sequence, kv head and row tile (hr), tile of n
        int b, hr, k, n;
    };
    auto seek = [&](int item) {
        int lo = 0, hi = B - 1;                 // last sequence whose first item is not behind `item` and that has tiles
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (cum[mid] * HR <= item) lo = mid; else hi = mid - 1;
        }
        Cursor c;
        c.b = lo;
        c.n = cum[lo + 1] - cum[lo];
        const int in = item - cum[lo] * HR;
        c.hr = in / c.n;
        c.k = in - c.hr * c.n;
        return c;
    };
    auto next_pair = [&](Cursor& c) {           // to the first tile of the next (sequence, head, row tile)
        c.k = 0;
        if (++c.hr == HR) {
            c.hr = 0;
            do { ++c.b; } while (c.b < B && cum[c.b + 1] == cum[c.b]);
            c.n = c.b < B ? cum[c.b + 1] - cum[c.b] : 0;
        }
    };

    // ---- copies: warp 0, lane 0 walks the same items STAGES ahead
    const int row_e = D / a.fmt.block;
    Cursor pc = seek(i0);
    SeqView psv = seq_view(a, pc.b);
    int issued = 0;
    auto issue = [&]() {
        const int s = issued % STAGES;
        const int tt = psv.tile_token(pc.k);
        const int64_t row0 = ((int64_t)pc.b * Hkv + pc.hr / a.n_row_tiles) * max_seq + tt;
        const int rows = min(kAttnTile, max_seq - tt);           // a multiple of 16
        const uint32_t dst = smem_u32(smem) + s * G_::STAGE_BYTES, bar = bar_full + 8 * s;
        const uint32_t mant = (P == 6 ? rows : kAttnTile) * ROW_M;       // a tiled copy always brings its whole box
        mbar_expect_tx(bar, 2 * mant + 2 * rows * row_e);
        if (P == 6) {
            bulk_g2s(dst, a.k_mant + row0 * ROW_M, mant, bar);
            bulk_g2s(dst + G_::VM_OFF, a.v_mant + row0 * ROW_M, mant, bar);
        } else {
            const int y = (int)(P == 4 ? row0 >> 1 : row0);
            tensor_g2s_2d(dst, &k_map, 0, y, bar);
            tensor_g2s_2d(dst + G_::VM_OFF, &v_map, 0, y, bar);
        }
        bulk_g2s(dst + G_::KE_OFF, a.k_exp + row0 * row_e, rows * row_e, bar);
        bulk_g2s(dst + G_::VE_OFF, a.v_exp + row0 * row_e, rows * row_e, bar);
        ++issued;
        if (++pc.k == pc.n) {
            const int b = pc.b;
            next_pair(pc);
            if (pc.b != b && pc.b < B) psv = seq_view(a, pc.b);
        }
    };
    if (tid == 0)
        for (int s = 0; s < STAGES && issued < n_mine; ++s) issue();

    Cursor cc = seek(i0);
    const int R = a.n_draft * a.group;
    const float up = a.scale * kValueUp;
    const float to_log2 = 1.4426950408889634f;
    const float cap_in = a.softcap > 0.f ? up / a.softcap : 0.f;
    const int ke_lane = (a.fmt.block == 16) ? 2 * t : (32 * t) / a.fmt.block;
    const int ve_lane = (16 * g) / a.fmt.block;
    const bool n16 = a.fmt.block == 16;
    bool dead = false;            // a copy did not arrive: no more waits, no more work, the flag is up
    int it = 0;
    while (it < n_mine) {
        // ================================================================ a run: tiles [k0, k1) of one (b, head, row tile)
        const int b = cc.b, hk = cc.hr / a.n_row_tiles, rt = cc.hr - hk * a.n_row_tiles;
        const int k0 = cc.k, k1 = min(cc.n, k0 + n_mine - it);
        const SeqView sv = seq_view(a, b);
        __syncthreads();
        for (int r = tid; r < ROWS; r += kAW * 32) {
            const int row = rt * ROWS + r, i = row / a.group;
            RowInfo x;
            x.pos = sv.ctx - 1;
            x.slope = 0.f;
            x.m0 = x.m1 = 0u;
            if (row < R) {
                if (a.slopes) x.slope = a.slopes[hk * a.group + row - i * a.group];
                if (a.tree) {
                    const int64_t at = (int64_t)b * a.n_draft + i;
                    const int dep = a.depth ? min(max(a.depth[at], 0), a.n_draft - 1) : i;
                    const uint64_t m = a.tree_mask ? a.tree_mask[at] : (i == 63 ? ~0ull : (2ull << i) - 1ull);
                    x.pos = sv.ctx + dep;
                    x.m0 = (uint32_t)m;
                    x.m1 = (uint32_t)(m >> 32);
                }
            }
            ri[r] = x;
        }
        if (a.tree)
            for (int j = tid; j < a.n_draft; j += kAW * 32)
                dpos[j] = sv.ctx + (a.depth ? min(max(a.depth[(int64_t)b * a.n_draft + j], 0), a.n_draft - 1) : j);
        // pi(q) as A fragments: [split][m tile][k step][lane] of four registers
#pragma unroll 4
        for (int x = tid; x < MT * RG * 8 * 32 * 4; x += kAW * 32) {
            const int reg = x & 3, ln = (x >> 2) & 31, ks = (x >> 7) & 7, mt = x >> 10;
            const int r = mt * 16 + (ln >> 2) + 8 * (reg & 1), row = rt * ROWS + r;
            const int i = row / a.group, hq = hk * a.group + row - i * a.group;
            float v[2] = {0.f, 0.f};
            if (row < R) {
                const int64_t base = (((int64_t)b * a.n_draft + i) * a.n_q_heads + hq) * D;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int slot = attn_k_slot<P>(ks, ln & 3, (reg & 2) + e);
                    const int ch = a.perm_k ? (a.perm_k[hk * D + slot] & (D - 1)) : slot;
                    v[e] = F32 ? static_cast<const float*>(a.q)[base + ch]
                               : __bfloat162float(static_cast<const __nv_bfloat16*>(a.q)[base + ch]);
                }
            }
            uint32_t* to = reinterpret_cast<uint32_t*>(qf) + x;
#pragma unroll
            for (int sp = 0; sp < G_::QSPLIT; ++sp) {
                const uint32_t p = pack_bf16x2_rn(v[0], v[1]);
                to[sp * MT * RG * 8 * 32 * 4] = p;
                if (F32) {
                    v[0] -= __uint_as_float(p << 16);
                    v[1] -= __uint_as_float(p & 0xffff0000u);
                }
            }
        }
        __syncthreads();
        uint4 qr[Q_REGS ? 8 : 1];
        if (Q_REGS) {
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) qr[Q_REGS ? ks : 0] = qf[(rg * 8 + ks) * 32 + lane];
        }

        float o[MT][16][4];
        float m_run[MT][2], l_run[MT][2];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
            for (int s = 0; s < 16; ++s)
#pragma unroll
                for (int k = 0; k < 4; ++k) o[mt][s][k] = 0.f;
            m_run[mt][0] = m_run[mt][1] = -3.4028235e38f;
            l_run[mt][0] = l_run[mt][1] = 0.f;
        }
        // tokens [clear_lo, ctx) and [0, pf) are visible to every row
        int clear_lo = sv.first;
        if (a.window > 0) clear_lo = max(clear_lo, sv.ctx + (a.tree ? a.n_draft - 1 : -1) - a.window + 1);

        for (int k = k0; k < k1; ++k, ++it) {
            const int stage = it % STAGES;
            const uint32_t phase = (uint32_t)(it / STAGES) & 1u;
            if (warp == 0 && it > 0 && issued < n_mine) {      // refill the stage used one tile ago (lane 0 counts `issued`)
                if (lane == 0 && !dead) {
                    const int pi = it - 1;
                    if (mbar_wait_bounded(bar_empty + 8 * (pi % STAGES), (uint32_t)(pi / STAGES) & 1u)) issue();
                    else dead = true;
                }
            }
            __syncwarp();
            dead = __any_sync(0xffffffffu, dead);
            if (!dead && !mbar_wait_bounded(bar_full + 8 * stage, phase)) dead = true;
            dead = __any_sync(0xffffffffu, dead);
            if (!dead) {
                const uint8_t* st = smem + stage * G_::STAGE_BYTES;
                const int tt = sv.tile_token(k);
                const int end = sv.ctx + sv.nd;
#pragma unroll 1
                for (int u = tg; u < kAttnTile / 32; u += TG) {          // 32 tokens at a time
                    const int u0 = u * 32, tok0 = tt + u0;
                    if (tok0 >= end) break;
                    // ---- scores: sc[m tile][16-token group * 2 + column tile][...]
                    float sc[MT][4][4];
                    {
                        uint32_t kw[4][P];
                        AW kg[4][2];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int row = u0 + 16 * (j >> 1) + tok_of<P>(g >> 1, g & 1, j & 1);
                            if (P == 6) {
#pragma unroll
                                for (int i = 0; i < 3; ++i) {
                                    const uint2 x = *reinterpret_cast<const uint2*>(st + tile_at<P>(row, 24 * t + 8 * i));
                                    kw[j][2 * i] = x.x; kw[j][2 * i + 1] = x.y;
                                }
                            } else {
#pragma unroll
                                for (int i = 0; i < P / 4; ++i) {
                                    const uint4 x = *reinterpret_cast<const uint4*>(st + tile_at<P>(row, 4 * P * t + 16 * i));
                                    kw[j][4 * i] = x.x; kw[j][4 * i + 1] = x.y; kw[j][4 * i + 2] = x.z; kw[j][4 * i + 3] = x.w;
                                }
                            }
                            const uint8_t* pe = st + G_::KE_OFF + row * row_e + ke_lane;
                            const uint2 l0 = lut[pe[0]];
                            kg[j][0] = aw_make<P>(l0.x, l0.y);
                            kg[j][1] = kg[j][0];
                            if (n16) {
                                const uint2 l1 = lut[pe[1]];
                                kg[j][1] = aw_make<P>(l1.x, l1.y);
                            }
                        }
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                            for (int j = 0; j < 4; ++j) sc[mt][j][0] = sc[mt][j][1] = sc[mt][j][2] = sc[mt][j][3] = 0.f;
#pragma unroll
                        for (int ks = 0; ks < 8; ks += 2) {
                            uint32_t r[4][4];
#pragma unroll
                            for (int j = 0; j < 4; ++j) attn_k<P>(kw[j], ks, kg[j][ks >> 2], r[j]);
#pragma unroll
                            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                                for (int sp = 0; sp < G_::QSPLIT; ++sp) {
                                    const uint4* qp = qf + ((sp * MT * RG + rg * MT + mt) * 8 + ks) * 32 + lane;
                                    const uint4 q0 = Q_REGS ? qr[Q_REGS ? ks : 0] : qp[0];
                                    const uint4 q1 = Q_REGS ? qr[Q_REGS ? ks + 1 : 0] : qp[32];
#pragma unroll
                                    for (int j = 0; j < 4; ++j) {
                                        mma_bf16(sc[mt][j], q0.x, q0.y, q0.z, q0.w, r[j][0], r[j][1]);
                                        mma_bf16(sc[mt][j], q1.x, q1.y, q1.z, q1.w, r[j][2], r[j][3]);
                                    }
                                }
                        }
                    }
                    // ---- cap, bias, masks; log2 units
                    const bool clear = tok0 + 32 <= sv.ctx && (tok0 >= clear_lo || tok0 + 32 <= sv.pf);
                    const bool bias = a.slopes != nullptr;
                    if (a.softcap > 0.f) {
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                            for (int j = 0; j < 4; ++j)
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    const float x = sc[mt][j][e] * cap_in;
                                    float th;
                                    if (F32) {
                                        th = tanhf(x);
                                    } else {                       // 1 - 2 / (1 + e^2x): about 2e-7 absolute
                                        th = 1.f - __fdividef(2.f, 1.f + ex2_approx(x * 2.8853900817779268f));
                                    }
                                    sc[mt][j][e] = th * a.softcap;
                                }
                    } else {
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                            for (int j = 0; j < 4; ++j)
#pragma unroll
                                for (int e = 0; e < 4; ++e) sc[mt][j][e] *= up;
                    }
                    if (bias || !clear) {
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                            for (int hh = 0; hh < 2; ++hh) {
                                const RowInfo x = ri[(rg * MT + mt) * 16 + g + 8 * hh];
#pragma unroll
                                for (int j = 0; j < 4; ++j)
#pragma unroll
                                    for (int e = 0; e < 2; ++e) {
                                        const int tok = tok0 + 16 * (j >> 1) + tok_of<P>(t, e, j & 1);
                                        float& y = sc[mt][j][2 * hh + e];
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
                                        y -= x.slope * (float)dist;
                                        if (!see) y = -INFINITY;
                                    }
                            }
                    }
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
#pragma unroll
                            for (int e = 0; e < 4; ++e) sc[mt][j][e] *= to_log2;
                    if (a.scores) {
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                            for (int hh = 0; hh < 2; ++hh) {
                                const int row = rt * ROWS + (rg * MT + mt) * 16 + g + 8 * hh;
                                if (row < R) {
                                    float* to = a.scores + ((int64_t)b * a.n_q_heads + hk * a.group + row) * max_seq;
#pragma unroll
                                    for (int j = 0; j < 4; ++j)
#pragma unroll
                                        for (int e = 0; e < 2; ++e) {
                                            const int tok = tok0 + 16 * (j >> 1) + tok_of<P>(t, e, j & 1);
                                            if (tok < max_seq) to[tok] = sc[mt][j][2 * hh + e];
                                        }
                                }
                            }
                    }
                    // ---- running softmax: the reference moves only when a score passes it by 8 (2^8 keeps P in range)
                    float top[MT][2];
                    bool grow = false;
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                        for (int hh = 0; hh < 2; ++hh) {
                            float x = -INFINITY;
#pragma unroll
                            for (int j = 0; j < 4; ++j) x = fmaxf(x, fmaxf(sc[mt][j][2 * hh], sc[mt][j][2 * hh + 1]));
                            top[mt][hh] = x;
                            grow |= x > m_run[mt][hh] + 8.f;
                        }
                    if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                            for (int hh = 0; hh < 2; ++hh) {
                                float x = top[mt][hh];
                                x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
                                x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
                                x = fmaxf(x, m_run[mt][hh]);
                                const float al = ex2_approx(m_run[mt][hh] - x);
                                m_run[mt][hh] = x;
                                l_run[mt][hh] *= al;
#pragma unroll
                                for (int s = 0; s < 16; ++s) { o[mt][s][2 * hh] *= al; o[mt][s][2 * hh + 1] *= al; }
                            }
                    }
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const float p = ex2_approx(sc[mt][j][e] - m_run[mt][e >> 1]);
                                sc[mt][j][e] = p;
                                l_run[mt][e >> 1] += p;
                            }
                    // ---- P . V, 16 tokens at a time
#pragma unroll
                    for (int h16 = 0; h16 < 2; ++h16) {
                        if (tok0 + 16 * h16 >= end) break;
                        uint32_t vw[4][P / 2];
                        uint2 lv[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {       // k = 2t, 2t+1, 2t+8, 2t+9
                            const int row = u0 + 16 * h16 + tok_of<P>(t, e & 1, e >> 1);
                            if (P == 4) {
                                const uint2 x = *reinterpret_cast<const uint2*>(st + G_::VM_OFF + tile_at<P>(row, 8 * g));
                                vw[e][0] = x.x; vw[e][1] = x.y;
                            } else if (P == 6) {
#pragma unroll
                                for (int i = 0; i < 3; ++i)
                                    vw[e][i] = *reinterpret_cast<const uint32_t*>(st + G_::VM_OFF + tile_at<P>(row, 12 * g + 4 * i));
                            } else {
                                const uint4 x = *reinterpret_cast<const uint4*>(st + G_::VM_OFF + tile_at<P>(row, 16 * g));
                                vw[e][0] = x.x; vw[e][1] = x.y; vw[e][P / 2 - 2] = x.z; vw[e][P / 2 - 1] = x.w;
                            }
                            lv[e] = lut[st[G_::VE_OFF + row * row_e + ve_lane]];
                        }
                        const AW ga = aw_make<P>(prmt(lv[0].x, lv[1].x, 0x7610u), prmt(lv[0].y, lv[1].y, 0x7610u));
                        const AW gb = aw_make<P>(prmt(lv[2].x, lv[3].x, 0x7610u), prmt(lv[2].y, lv[3].y, 0x7610u));
                        uint32_t pa[MT][4], pl[F32 ? MT : 1][4];
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                            for (int x = 0; x < 4; ++x) {      // (row g, tile 0), (row g+8, tile 0), (row g, tile 1), (row g+8, tile 1)
                                const float p0 = sc[mt][2 * h16 + (x >> 1)][2 * (x & 1)], p1 = sc[mt][2 * h16 + (x >> 1)][2 * (x & 1) + 1];
                                pa[mt][x] = pack_bf16x2_rn(p0, p1);
                                if (F32)
                                    pl[F32 ? mt : 0][x] = pack_bf16x2_rn(p0 - __uint_as_float(pa[mt][x] << 16),
                                                                         p1 - __uint_as_float(pa[mt][x] & 0xffff0000u));
                            }
#pragma unroll
                        for (int r = 0; r < 8; r += 2) {
                            uint32_t xa[4], xb[4];
                            attn_v<P>(vw[0], vw[1], r, ga, xa);
                            attn_v<P>(vw[2], vw[3], r, gb, xb);
#pragma unroll
                            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                                for (int s = 0; s < 4; ++s) {
                                    float (&acc)[4] = o[mt][2 * r + s];
                                    if (F32) {
                                        float d[4] = {0.f, 0.f, 0.f, 0.f};
                                        mma_bf16(d, pl[F32 ? mt : 0][0], pl[F32 ? mt : 0][1], pl[F32 ? mt : 0][2], pl[F32 ? mt : 0][3], xa[s], xb[s]);
                                        mma_bf16(d, pa[mt][0], pa[mt][1], pa[mt][2], pa[mt][3], xa[s], xb[s]);
                                        acc[0] += d[0]; acc[1] += d[1]; acc[2] += d[2]; acc[3] += d[3];
                                    } else {
                                        mma_bf16(acc, pa[mt][0], pa[mt][1], pa[mt][2], pa[mt][3], xa[s], xb[s]);
                                    }
                                }
                        }
                    }
                }
            }
            __syncwarp();
            if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar_empty + 8 * stage) : "memory");
        }

        // ---- the token groups' results into one: o, max, sum per row
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) {
                float l = l_run[mt][hh];
                l += __shfl_xor_sync(0xffffffffu, l, 1);
                l += __shfl_xor_sync(0xffffffffu, l, 2);
                l_run[mt][hh] = l;
                if (t == 0) ml[tg * ROWS + (rg * MT + mt) * 16 + g + 8 * hh] = make_float2(m_run[mt][hh], l);
            }
        __syncthreads();
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) {
                const int r = (rg * MT + mt) * 16 + g + 8 * hh;
                float m = -INFINITY;
#pragma unroll
                for (int w = 0; w < TG; ++w) m = fmaxf(m, ml[w * ROWS + r].x);
                const float al = ex2_approx(m_run[mt][hh] - m);
#pragma unroll
                for (int s = 0; s < 16; ++s) { o[mt][s][2 * hh] *= al; o[mt][s][2 * hh + 1] *= al; }
            }
#pragma unroll 1
        for (int w = 0; w < TG; ++w) {
            if (tg == w) {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int s = 0; s < 16; ++s)
#pragma unroll
                        for (int hh = 0; hh < 2; ++hh) {
                            float2* p = reinterpret_cast<float2*>(ob + ((rg * MT + mt) * 16 + g + 8 * hh) * G_::OSTRIDE + 8 * s + 2 * t);
                            float2 v = make_float2(o[mt][s][2 * hh], o[mt][s][2 * hh + 1]);
                            if (w > 0) { const float2 y = *p; v.x += y.x; v.y += y.y; }
                            *p = v;
                        }
            }
            __syncthreads();
        }
        const bool whole = k0 == 0 && k1 == cc.n;
        for (int r = warp; r < ROWS; r += kAW) {
            const int row = rt * ROWS + r;
            if (row >= R) break;
            float m = -INFINITY, l = 0.f;
#pragma unroll
            for (int w = 0; w < TG; ++w) m = fmaxf(m, ml[w * ROWS + r].x);
#pragma unroll
            for (int w = 0; w < TG; ++w) { const float2 x = ml[w * ROWS + r]; l += x.y * ex2_approx(x.x - m); }
            const float* src = ob + r * G_::OSTRIDE;
            if (whole) {
                const int i = row / a.group, hq = hk * a.group + row - i * a.group;
                const bool live = !a.tree || i < sv.nd;
                const float inv = (live && l != 0.f) ? kValueUp / l : 0.f;
                const int64_t at = (((int64_t)b * a.n_draft + i) * a.n_q_heads + hq) * D + 4 * lane;
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int c = 4 * lane + e;
                    const int slot = a.inv_perm_v ? (a.inv_perm_v[hk * D + c] & (D - 1)) : c;
                    v[e] = inv == 0.f ? 0.f : src[part_pos(slot)] * inv;
                }
                if (F32) *reinterpret_cast<float4*>(static_cast<float*>(a.out) + at) = make_float4(v[0], v[1], v[2], v[3]);
                else *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.out) + at) =
                         make_uint2(pack_bf16x2_rn(v[0], v[1]), pack_bf16x2_rn(v[2], v[3]));
                if (a.lse && lane == 0) a.lse[(int64_t)b * a.n_q_heads + hq] = l > 0.f ? m + log2f(l) : (l == 0.f ? INFINITY : l);
            } else {
                float* dst = a.partials + ((int64_t)(2 * blockIdx.x + (k0 == 0 ? 1 : 0)) * ROWS + r) * kAttnPart;
                reinterpret_cast<float4*>(dst)[lane] = *reinterpret_cast<const float4*>(src + 4 * lane);
                if (lane == 0) { dst[D] = m; dst[D + 1] = l; }
            }
        }
        cc.k = k1;
        if (k1 == cc.n) next_pair(cc);
    }
    if (dead) {
        // give the copies still in flight a bounded chance to land before the shared memory is released
        if (lane == 0) raise_flag(a.status, KVBFP_FLAG_WAIT_TIMEOUT);
        for (int s = 0; s < STAGES; ++s) {
            (void)mbar_wait_bounded(bar_full + 8 * s, 0);
            (void)mbar_wait_bounded(bar_full + 8 * s, 1);
        }
    }
    pdl_trigger();
}

template <int P, int MT, int RG, bool F32>
kvbfp_status launch_attn(const AttnArgs& a, cudaStream_t s) {
    using G_ = AGeo<P, MT, RG, F32>;
    static std::atomic<bool> attr_set[64];      // per device; setting the attribute twice is harmless
    int dev = 0;
    KVBFP_CUDA(cudaGetDevice(&dev));
    const int smem = G_::smem_bytes(a.fmt.batch);
    if (dev < 0 || dev >= 64) return KVBFP_ERR_UNSUPPORTED;
    if (!attr_set[dev].load(std::memory_order_acquire)) {
        KVBFP_CUDA(cudaFuncSetAttribute(attn_rows<P, MT, RG, F32>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                        G_::smem_bytes(kAttnMaxBatch)));
        attr_set[dev].store(true, std::memory_order_release);
    }
    CUtensorMap k_map, v_map;
    if (P != 6) {
        const uint64_t rows = (uint64_t)a.fmt.batch * a.fmt.n_kv_heads * a.fmt.max_seq * P / 8;     // lines of 128 bytes
        kvbfp_status st = make_row_map(&k_map, a.k_mant, rows, 128, kAttnTile * P / 8);
        if (st == KVBFP_OK) st = make_row_map(&v_map, a.v_mant, rows, 128, kAttnTile * P / 8);
        if (st != KVBFP_OK) return st;
    }
    KVBFP_CUDA(launch_pdl(attn_rows<P, MT, RG, F32>, dim3(a.workers), dim3(kAW * 32), smem, s, a, k_map, v_map));
    KVBFP_LAUNCH_CHECK("attn_rows");
    return KVBFP_OK;
}

template <int P>
kvbfp_status launch_attn_p(const AttnArgs& a, cudaStream_t s) {
    if (!a.q_is_bf16) return a.rows_tile == 16 ? launch_attn<P, 1, 1, true>(a, s) : KVBFP_ERR_UNSUPPORTED;
    if (a.rows_tile == 16) return launch_attn<P, 1, 1, false>(a, s);
    if (a.rows_tile == 32) return launch_attn<P, 2, 1, false>(a, s);
    return launch_attn<P, 2, 2, false>(a, s);
}

}  // namespace
}  // namespace kvbfp
