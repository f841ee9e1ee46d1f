// Attention of up to eight bf16 query rows of a (batch, kv head), or of fp32 rows in items of eight, over the packed cache
// with warp-level bf16 MMAs.
//
//   S^T[tokens x rows] = K . pi(Q)^T ;  y = log2(e) * (cap * tanh(scale * S / cap) - slope * distance) ;  P = 2^(y - m)
//   O^T[slots x rows] += V^T . P^T ;  l += sum of P over tokens
//
// Work split.  Every block counts the tiles each sequence has to read (from the real lengths and windows, so ragged batches
// and windows stay balanced): that takes about a microsecond, a launch of its own before took three.  The kernel is
// persistent: all tiles are cut into one contiguous range per warp; a warp walks its range as runs (the tiles of one
// (sequence, head, row tile)), shares nothing with other warps and meets no barrier.  A run that covers all tiles
// writes the result itself, others leave a partial for attn_merge.  The tiles come through a per-warp ring of
// shared-memory stages filled by asynchronous copies that run ahead across run boundaries.  (Rows of q are read where a run
// begins, through the permutation, while the first copies are on their way.)
//
// Fragments.  The query rows are the narrow side (N = 8 of m16n8k16) of both products, so that few rows waste nothing: with
// the rows as the wide side (16) a token costs twice the matrix instructions and the accumulators twice the registers
// (16 x 32 x 8192 rows, one token each: 252 us for the weights' call then, 160 us now).  P comes out token by token and is
// turned by an 8 x 8 transposition.  K and V are converted in registers: the stored field (an unsigned offset) or-ed under
// the bits of 128.0 is an exact bf16 number, one bf16x2 fma removes the offset and applies the block's power of two (a
// mantissa has at most 7 bits + sign: exact).  The contraction order is free, so a lane's 32-slot chunk of a K row and
// 16-slot chunk of a V row are used in the order they unpack in; the 16 tokens of a group are dealt to rows so that both the
// K and the V loads touch every bank once (tok_of).  Two groups are scored before either is weighed, for more independent
// instructions.
//
// What bounds it: integer instructions (166 of the 357 a warp issues per 16 tokens, at half rate; 120 of them cut the 4-bit
// fields) and the latency between dependent ones: 0.55 instructions a cycle with the three blocks that registers allow.
// 16 x 32 heads of 8192 4-bit rows, 570 MB, one bf16 query each: 140 us, 4.1 TB/s.
//
// Types.  bf16 queries are exact operands, P is rounded to bf16 (half a step, 2^-9 relative, at random: the output is
// rounded to bf16 too).  fp32 queries and P are three bf16 terms each (24 bits); their O is summed outside the MMAs because
// the tensor cores cut, not round, the running sum.  m, l, O and scores are fp32.
#pragma once
#include "attn_common.cuh"

namespace kvbfp {
namespace {

constexpr int kRows = 8;        // query rows of a work item

// Cached values are carried times 2^-8, so that no exponent byte leaves the bf16 range with the conversion's offset;
// undone on scores and outputs.
constexpr float kValueUp = 256.f;

// Stored fields to bf16 pairs.
template <int P> struct AFmt;
template <> struct AFmt<4> { static constexpr uint32_t mask = 0x000F000Fu, magic = 0x43004300u, bias = 0xC308C308u; };  // -136
template <> struct AFmt<6> { static constexpr uint32_t mask = 0x003F003Fu, magic = 0x43004300u, bias = 0xC320C320u; };  // -160
template <> struct AFmt<8> { static constexpr uint32_t mask = 0x000F000Fu, magic = 0x43004300u, bias = 0xC510C510u; };  // -2304

struct AW {
    uint32_t s, c, s16;      // weight pair, -offset * weight, 16 * weight (8-bit fields)
};
// Weights of two exponent bytes (in 16-bit halves): 2^(e - 127 - (P - 2) - 8) as bf16, zero where that has no normal number.
template <int P>
__device__ __forceinline__ AW aw_make(uint32_t e2) {
    AW w;
    asm("max.s16x2 %0, %1, %2;" : "=r"(w.s) : "r"(e2), "r"((P + 6) * 0x00010001u));
    w.s = w.s * 0x80u - (P + 6) * 0x00800080u;
    w.c = mul_bf16x2(w.s, AFmt<P>::bias);
    w.s16 = (P == 8) ? mul_bf16x2(w.s, 0x41804180u) : 0u;
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

// An 8 x 8 matrix of 16-bit numbers, a row's pair per lane (row lane / 4), transposed.
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// pi(q) of one query row (`q`; NULL: zeros) at a lane's k positions as B operand: [term][k step / 2].
template <int P, bool F32, class Args>
__device__ __forceinline__ void load_q(const Args& a, const void* q, int hk, int t, uint4 (&qr)[F32 ? 3 : 1][4]) {
    int at[32];           // channels of the lane's 32 slots
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        int4 x = make_int4(32 * t + 4 * i, 32 * t + 4 * i + 1, 32 * t + 4 * i + 2, 32 * t + 4 * i + 3);
        if (a.perm_k) x = *reinterpret_cast<const int4*>(a.perm_k + hk * kHeadDim + 32 * t + 4 * i);
        at[4 * i] = x.x & (kHeadDim - 1); at[4 * i + 1] = x.y & (kHeadDim - 1);
        at[4 * i + 2] = x.z & (kHeadDim - 1); at[4 * i + 3] = x.w & (kHeadDim - 1);
    }
    float v[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        v[i] = 0.f;
        if (q) v[i] = F32 ? static_cast<const float*>(q)[at[i]] : __bfloat162float(static_cast<const __nv_bfloat16*>(q)[at[i]]);
    }
#pragma unroll
    for (int ks = 0; ks < 8; ks += 2) {
        uint32_t reg[F32 ? 3 : 1][4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {       // k step, positions 0, 1 | 2, 3
            float v0 = v[attn_k_slot<P>(ks + (k >> 1), 0, 2 * (k & 1))], v1 = v[attn_k_slot<P>(ks + (k >> 1), 0, 2 * (k & 1) + 1)];
#pragma unroll
            for (int c = 0; c < (F32 ? 3 : 1); ++c) {
                reg[c][k] = pack_bf16x2_rn(v0, v1);
                v0 -= __uint_as_float(reg[c][k] << 16);
                v1 -= __uint_as_float(reg[c][k] & 0xffff0000u);
            }
        }
#pragma unroll
        for (int c = 0; c < (F32 ? 3 : 1); ++c) qr[c][ks >> 1] = make_uint4(reg[c][0], reg[c][1], reg[c][2], reg[c][3]);
    }
}

template <int P>
struct AGeo {
    static constexpr int ROW_M = kHeadDim * P / 8;
    static constexpr int TILE = attn_rows_tile(P);       // tokens per stage
    static constexpr int STAGES = attn_rows_stages(P);
    static constexpr int VM_OFF = TILE * ROW_M, KE_OFF = 2 * VM_OFF;
    __host__ __device__ static int exp_bytes(int row_e) { return 2 * TILE * row_e; }       // of a stage
    static constexpr int WARP_SMALL = kHeadDim * 4 + (STAGES * 8 + 15) / 16 * 16;    // rows and positions (one output row at the end of a run), barriers
    static_assert(kRows * 16 + kAttnMaxDraft * 4 <= kHeadDim * 4, "in an output row's place");
    __host__ __device__ static int smem_bytes(int row_e) {
        return kAttnWarps * STAGES * (KE_OFF + exp_bytes(row_e)) + kAttnWarps * (WARP_SMALL + 16);
    }
};

// (A call: as code of the loop it slowed small capped calls down, whose instructions come from memory: one token over 32 x
// 1000 rows 14.5 us, 14.1 this way.)
__device__ __noinline__ float tanh_call(float x) { return tanh_relative(x); }

template <int P, bool N16, bool F32>
__global__ void __launch_bounds__(kAttnWarps * 32, attn_rows_blocks(!F32)) attn_rows(const AttnArgs a, const __grid_constant__ CUtensorMap k_map,
                                                                                       const __grid_constant__ CUtensorMap v_map) {
    using G_ = AGeo<P>;
    static_assert(G_::WARP_SMALL % 16 == 0 && (P == 6 || G_::VM_OFF % 1024 == 0), "vector accesses; whole swizzle periods");
    constexpr int D = kHeadDim, ROW_M = G_::ROW_M, STAGES = G_::STAGES, TILE = G_::TILE, ROWS = kRows, SPLIT = F32 ? 3 : 1;
    constexpr int GROUP = 16 * ROW_M;
    extern __shared__ __align__(1024) uint8_t smem[];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int row_e = D / a.fmt.block, exp_half = TILE * row_e;
    // mantissa tiles of all warps and stages first (whole swizzle periods), then the exponent bytes, then the rest
    uint8_t* my_m = smem + warp * STAGES * G_::KE_OFF;
    uint8_t* my_e = smem + kAttnWarps * STAGES * G_::KE_OFF + warp * STAGES * 2 * exp_half;
    uint8_t* rest = smem + kAttnWarps * STAGES * (G_::KE_OFF + 2 * exp_half);
    uint8_t* small = rest + warp * G_::WARP_SMALL;
    RowInfo* ri = reinterpret_cast<RowInfo*>(small);
    float* orow = reinterpret_cast<float*>(small);
    int* dpos = reinterpret_cast<int*>(small + kRows * 16);
    const uint32_t bar = smem_u32(small + kHeadDim * 4);

    if (lane == 0) {
        for (int s = 0; s < STAGES; ++s) mbar_init(bar + 8 * s, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncthreads();
    pdl_wait();

    const int B = a.fmt.batch, Hkv = a.fmt.n_kv_heads, HR = Hkv * a.n_row_tiles, max_seq = a.fmt.max_seq;
    // ---- the tiles of all sequences, and where this block's warps begin (block 0 leaves the counts for the merge)
    int *s_scan = reinterpret_cast<int*>(rest + kAttnWarps * G_::WARP_SMALL), *s_b = s_scan + kAttnWarps, *s_c0 = s_b + kAttnWarps, *s_n = s_c0 + kAttnWarps;
    const int per = (B + kAttnWarps * 32 - 1) / (kAttnWarps * 32);
    int mine = 0;
    for (int i = 0; i < per; ++i)
        if (tid * per + i < B) mine += seq_view(a, tid * per + i).n;
    int before = mine;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, before, off);
        if (lane >= off) before += y;
    }
    if (lane == 31) s_scan[warp] = before;
    __syncthreads();
    before -= mine;
    int total = 0;
#pragma unroll
    for (int w = 0; w < kAttnWarps; ++w) {
        if (w < warp) before += s_scan[w];
        total += s_scan[w];
    }
    const int n_items = total * HR;
    const int workers = min(a.workers, n_items), me = blockIdx.x + gridDim.x * warp;      // neighbouring ranges on different SMs
    for (int i = 0; i < per; ++i) {
        const int bb = tid * per + i;
        if (bb >= B) break;
        const SeqView sv = seq_view(a, bb);
#pragma unroll
        for (int w = 0; w < kAttnWarps; ++w) {
            const int m = blockIdx.x + gridDim.x * w, at = m < workers ? worker_start(m, n_items, workers) : -1;
            if (at >= before * HR && at < (before + sv.n) * HR) { s_b[w] = bb; s_c0[w] = before; s_n[w] = sv.n; }
        }
        if (blockIdx.x == 0) {
            a.plan[bb] = before;
            a.views[bb] = sv;
            if (bb == B - 1) a.plan[B] = total;
            if (sv.clamped) raise_flag(a.status, KVBFP_FLAG_POSITION);
        }
        before += sv.n;
    }
    __syncthreads();
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
    cc.b = s_b[warp];
    cc.n = s_n[warp];
    cc.hr = (i0 - s_c0[warp] * HR) / cc.n;
    cc.k = i0 - s_c0[warp] * HR - cc.hr * cc.n;
    auto next_pair = [&](Cursor& c) {           // to the first tile of the next (sequence, head, row tile)
        c.k = 0;
        if (++c.hr == HR) {
            c.hr = 0;
            c.n = 0;
            while (c.n == 0 && ++c.b < B) c.n = seq_view(a, c.b).n;
        }
    };

    // ---- copies: the same items, STAGES ahead (every lane keeps the cursor, lane 0 issues)
    Cursor pc = cc;
    SeqView psv = seq_view(a, pc.b);
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
            if (pc.b != b && pc.b < B) psv = seq_view(a, pc.b);
        }
    };
    for (int s = 0; s < STAGES && issued < n_mine; ++s) issue();

    const int R = a.n_draft * a.group;
    const float up = a.scale * kValueUp, to_log2 = 1.4426950408889634f, plain = finite_factor(up * to_log2);
    const float cap_in = a.softcap > 0.f ? finite_factor(up / a.softcap) : 0.f;
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
    const float tkf[2] = {(float)tk[0], (float)tk[1]};

    bool dead = false;            // a copy did not arrive: no more waits, no more work, the flag is up
    int it = 0;
    while (it < n_mine) {
        // ================================================================ a run: tiles [k0, k1) of one (b, head, row tile)
        const int b = cc.b, hk = cc.hr / a.n_row_tiles, rt = cc.hr - hk * a.n_row_tiles;
        const int k0 = cc.k, k1 = min(cc.n, k0 + n_mine - it);
        const SeqView sv = seq_view(a, b);
        uint4 qr[SPLIT][4];           // k steps 2 i, 2 i + 1
        {
            const int row = rt * ROWS + g, i = row / a.group;
            const int64_t at = (((int64_t)b * a.n_draft + i) * a.n_q_heads + hk * a.group + row - i * a.group) * D;
            const void* q = F32 ? (const void*)(static_cast<const float*>(a.q) + at) : (const void*)(static_cast<const __nv_bfloat16*>(a.q) + at);
            load_q<P, F32>(a, row < R ? q : nullptr, hk, t, qr);
        }
        __syncwarp();
        if (lane < ROWS) ri[lane] = row_info(a, b, hk, rt * ROWS + lane, R);
        if (a.tree) {
#pragma unroll
            for (int i = 0; i < kAttnMaxDraft; i += 32)
                if (i + lane < a.n_draft) dpos[i + lane] = sv.ctx + draft_depth(a, b, i + lane);
        }
        __syncwarp();

        float o[8][4];                // slots 16 g + 2 i (+ 1: upper pair) of rows 2 t, 2 t + 1
        float m_run[2], l_run[2];     // of rows 2 t, 2 t + 1
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) o[i][k] = 0.f;
        m_run[0] = m_run[1] = -3.4028235e38f;
        l_run[0] = l_run[1] = 0.f;
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
            for (int u = 0; u < TILE / 32; ++u, stm += 2 * GROUP, ste += 32 * row_e) {        // 32 tokens: two groups of 16
                const int tok0 = tt + 32 * u;
                if (tok0 >= end) break;
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
                // ---- cap, bias, masks: mul * sc is the score in log2 units; tokens that every row sees have no masks
                float mul = plain;
                if (a.softcap > 0.f) {
                    mul = a.softcap * to_log2;
                    if (!F32 && a.softcap > kCapFast) {
#pragma unroll
                        for (int x = 0; x < 8; ++x) sc[x >> 2][x & 3] = tanh_call(sc[x >> 2][x & 3] * cap_in);
                    } else
#pragma unroll
                    for (int x = 0; x < 8; ++x) {
                        float& y = sc[x >> 2][x & 3];
                        if (F32) y = tanhf(y * cap_in);
                        else y = 1.f - __fdividef(2.f, 1.f + ex2_approx(y * (cap_in * 2.8853900817779268f)));    // 1 - 2 / (1 + e^2y): about 2e-7 absolute
                    }
                }
                const bool clear = tok0 + 32 <= sv.ctx && (tok0 >= clear_lo || tok0 + 32 <= sv.pf);
                if (!clear || a.slopes) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const RowInfo x = ri[2 * t + e];
                        const float bias = x.slope * to_log2;
                        if (clear) {
                            const float far = (float)(x.pos - tok0);
#pragma unroll
                            for (int gj = 0; gj < 4; ++gj) {
                                float& y = sc[gj >> 1][2 * (gj & 1) + e];
                                y = fmaf(y, mul, -bias * (far - (tkf[gj & 1] + 16.f * (gj >> 1))));
                            }
                        } else {
#pragma unroll
                            for (int gj = 0; gj < 4; ++gj) {
                                float& y = sc[gj >> 1][2 * (gj & 1) + e];
                                const int tok = tok0 + 16 * (gj >> 1) + tk[gj & 1];
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
                                y = see ? fmaf(y, mul, -bias * (float)dist) : -INFINITY;
                            }
                        }
                    }
                    mul = 1.f;
                }
                if (a.scores) {
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        if (2 * t + e < R) {                  // (one token: one row tile)
                            float* to = a.scores + ((int64_t)b * a.n_q_heads + hk * a.group + 2 * t + e) * max_seq + tok0;
#pragma unroll
                            for (int gj = 0; gj < 4; ++gj)
                                if (gj < 2 || tok0 + 16 < max_seq) to[16 * (gj >> 1) + tk[gj & 1]] = sc[gj >> 1][2 * (gj & 1) + e] * mul;
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
                    // P as B fragments: a token's pair of rows, transposed; fp32: three terms
                    uint32_t pb[SPLIT][2];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        float p0 = ex2_approx(fmaf(sc[gr][2 * j], mul, -m_run[0]));
                        float p1 = ex2_approx(fmaf(sc[gr][2 * j + 1], mul, -m_run[1]));
                        l_run[0] += p0;
                        l_run[1] += p1;
#pragma unroll
                        for (int s = 0; s < SPLIT; ++s) {
                            const uint32_t x = pack_bf16x2_rn(p0, p1);
                            p0 -= __uint_as_float(x << 16);
                            p1 -= __uint_as_float(x & 0xffff0000u);
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
                                for (int c = SPLIT - 1; c >= 0; --c) mma_bf16(d, xa[2 * h], xa[2 * h + 1], xb[2 * h], xb[2 * h + 1], pb[c][0], pb[c][1]);
                                acc[0] += d[0]; acc[1] += d[1]; acc[2] += d[2]; acc[3] += d[3];
                            } else {
                                mma_bf16(acc, xa[2 * h], xa[2 * h + 1], xb[2 * h], xb[2 * h + 1], pb[0][0], pb[0][1]);
                            }
                        }
                    }
                }
            }
            __syncwarp();                      // every lane has read the stage
            if (issued < n_mine) issue();
        }

        // ---- the run's result: a lane holds slots [16 g, 16 g + 16) of rows 2 t and 2 t + 1
        const bool whole = k0 == 0 && k1 == cc.n;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float l = l_run[e];
            l += __shfl_xor_sync(0xffffffffu, l, 4);
            l += __shfl_xor_sync(0xffffffffu, l, 8);
            l += __shfl_xor_sync(0xffffffffu, l, 16);
            const int r = 2 * t + e, row = rt * ROWS + r;
            const int i = row / a.group, hq = hk * a.group + row - i * a.group;
            const float m = m_run[e];
            if (!whole) {
                if (row < R) {
                    float* dst = a.partials + ((int64_t)(2 * me + (k0 == 0 ? 1 : 0)) * a.part_rows + r) * kAttnPart;
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        reinterpret_cast<float4*>(dst + 16 * g)[c] = make_float4(o[2 * c][e], o[2 * c][2 + e], o[2 * c + 1][e], o[2 * c + 1][2 + e]);
                    if (g == 0) { dst[D] = m; dst[D + 1] = l; }
                }
                continue;
            }
            const bool live = row < R && (!a.tree || i < sv.nd) && l != 0.f;
            const float inv = live ? kValueUp / l : 0.f;
            float v[16];
#pragma unroll
            for (int s = 0; s < 16; ++s) v[s] = live ? o[s >> 1][2 * (s & 1) + e] * inv : 0.f;
            const int64_t at = (((int64_t)b * a.n_draft + i) * a.n_q_heads + hq) * D;
            if (a.lse && row < R && g == 0) a.lse[(int64_t)b * a.n_q_heads + hq] = l > 0.f ? m + log2f(l) : (l == 0.f ? INFINITY : l);
            if (!a.inv_perm_v) {
                if (row < R) {
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
                for (int tt = 0; tt < 4; ++tt) {
                    if (rt * ROWS + 2 * tt + e >= R) break;
                    __syncwarp();
                    if (t == tt) {
#pragma unroll
                        for (int s = 0; s < 16; ++s) orow[16 * g + s] = v[s];
                    }
                    __syncwarp();
                    const int64_t to = __shfl_sync(0xffffffffu, at, tt) + 4 * lane;
                    const float y0 = orow[sl[0]], y1 = orow[sl[1]], y2 = orow[sl[2]], y3 = orow[sl[3]];
                    if (F32) *reinterpret_cast<float4*>(static_cast<float*>(a.out) + to) = make_float4(y0, y1, y2, y3);
                    else *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.out) + to) = make_uint2(pack_bf16x2_rn(y0, y1), pack_bf16x2_rn(y2, y3));
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

template <int P, bool N16, bool F32>
kvbfp_status launch_attn(const AttnArgs& a, int grid, cudaStream_t s) {
    auto kernel = attn_rows<P, N16, F32>;
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
    KVBFP_CUDA(launch_pdl(kernel, dim3(grid), dim3(kAttnWarps * 32), AGeo<P>::smem_bytes(kHeadDim / a.fmt.block), s, a, k_map, v_map));
    KVBFP_LAUNCH_CHECK("attn_rows");
    return KVBFP_OK;
}

template <int P>
kvbfp_status launch_attn_p(const AttnArgs& a, int grid, cudaStream_t s) {
    const bool n16 = a.fmt.block == 16;
    if (a.q_is_bf16) return n16 ? launch_attn<P, true, false>(a, grid, s) : launch_attn<P, false, false>(a, grid, s);
    return n16 ? launch_attn<P, true, true>(a, grid, s) : launch_attn<P, false, true>(a, grid, s);
}

}  // namespace
}  // namespace kvbfp
