// Attention of up to 64 bf16 query rows per (batch, kv head) over the packed cache on the fifth-generation tensor cores.
//
//   S^T[tokens x rows] = K . pi(Q)^T          K: tensor memory, pi(Q): shared memory
//   y = log2(e) * (cap * tanh(scale * S / cap) - slope * distance) ;  P = 2^(y - m)
//   O^T[slots x rows] += V^T . P^T            V, P: shared memory (both with the token as the slow index)
//
// Why: with the query rows as the narrow side of the product a tile of 128 tokens costs the tensor cores rows / 64 x 128
// cycles per product, so what is left to do per cached element is its conversion, and that is done once for all rows
// (the warp-level kernel converts per 16 rows and its matrix instructions run at a third of the rate).
//
// One persistent thread block per SM, tiles of 128 tokens, a contiguous range of tiles per block (attn.cuh).  Roles:
//   warp 16      copies packed tiles into a ring of stages and pi(Q) of the next (sequence, head, row tile) ahead
//   warps 8..15  conversion, two groups on alternate tiles, a thread per token: its K row goes to tensor memory (the A
//                operand of the first product), its V row to shared memory (the A operand of the second, slots contiguous)
//   warp 17      issues the matrix instructions: S of tile i, then O of tile i - 1
//   warps 0..7   softmax, a thread per token, each group half of the query rows: scores from tensor memory, masks,
//                running maximum, P to shared memory; at the end of a run O^T from tensor memory to the result
// Cached values are converted relative to their row's largest exponent (see below); magnitudes of 2^118 and above are
// outside the range.
// The row maximum runs across threads here, so it is only taken when a score passes the reference by 8 (a factor 2^8),
// which a barrier over the group tells; then O is rescaled in tensor memory.  Sums are kept per thread and reduced at
// the end of a run.
//
// Shared memory traffic per token (4 bits, 64 rows): packed rows 272 bytes in and out, V 256 written and 256 read, P
// and the re-read pi(Q) 512: 1.3 kB at 128 bytes a cycle, against 1.6 kB that the copy bandwidth would let pass.
#pragma once
#include "attn_common.cuh"
#include "umma.cuh"

namespace kvbfp {
namespace {

constexpr int kUTile = 128;
constexpr int kUThreads = 18 * 32;

// Slot at position `m` of a converted row (the order the fields unpack in); K and V alike.
template <int P>
__device__ __forceinline__ int umma_slot(int m) {
    if (P != 8) return (m & ~7) | ((m & 1) << 2) | ((m >> 1) & 3);
    return (m & ~3) | ((m & 1) << 1) | ((m >> 1) & 1);
}

template <int P, int N>
struct UGeo {
    static constexpr int ROW_M = kHeadDim * P / 8;
    static constexpr int STAGES = P == 4 ? (N == 64 ? 3 : 4) : 2;
    static constexpr int VBUF = P == 8 && N == 64 ? 2 : 3;       // converted V tiles: one being written, the others in use
    static constexpr int MANT = 2 * kUTile * ROW_M;              // K and V rows of a stage
    static constexpr int V_OFF = STAGES * MANT;                  // converted V, buffers of 32 KB
    static constexpr int V_BYTES = kUTile * kHeadDim * 2;
    static constexpr int P_OFF = V_OFF + VBUF * V_BYTES;
    static constexpr int P_BYTES = kUTile * N * 2;
    static constexpr int Q_OFF = P_OFF + 2 * P_BYTES;
    static constexpr int Q_BYTES = N * kHeadDim * 2;
    static constexpr int E_OFF = Q_OFF + 2 * Q_BYTES;            // exponent bytes: STAGES x 2 x 128 x row_e
    // behind them: factors of the tokens, row data, drafted positions, channel table, references, reduction, barriers
    static constexpr int SMALL = 8 * kUTile * 4 + N * 16 + 2 * kAttnMaxDraft * 4 + 2 * kHeadDim * 4 + N * 4 * 4 + 8 * N / 2 * 4 + 16 +
                                 (2 * STAGES + 12) * 8 + 16;
    __host__ __device__ static int smem_bytes(int row_e) { return E_OFF + STAGES * 2 * kUTile * row_e + SMALL; }
};

// pi(Q) of one (sequence, kv head, row tile) per block, as the shared-memory image of the B operand: two panels of 64
// positions, lines of 128 bytes per row, 16-byte pieces at piece ^ (row % 8).
template <int P, int N>
__global__ void __launch_bounds__(128) umma_prep(const AttnArgs a) {
    __shared__ float sq[N][kHeadDim + 4];
    __shared__ int sp[kHeadDim];
    prep_common<N, false>(a, sq, sp);
    uint8_t* to = reinterpret_cast<uint8_t*>(a.qfrag) + (int64_t)blockIdx.x * (N * kHeadDim * 2);
    for (int x = threadIdx.x; x < N * 16; x += 128) {       // 16-byte pieces: row, positions [8 c, 8 c + 8)
        const int c = x & 15, row = x >> 4;
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            w[j] = pack_bf16x2_rn(sq[row][sp[umma_slot<P>(8 * c + 2 * j)]], sq[row][sp[umma_slot<P>(8 * c + 2 * j + 1)]]);
        *reinterpret_cast<uint4*>(to + (c >> 3) * (N * 128) + row * 128 + (((c & 7) ^ (row & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// Conversion.  A field that lies within the low eight bits of a 16-bit half IS a bf16 number: the half masked down to
// it, read as bf16, is the field times 2^-133 (times 4 or 16 where it lies higher), for below 2^-125 bf16 counts in equal
// steps.  One bf16x2 fma turns two of them into (field - offset) times the block's weight, exactly; nothing is or-ed
// under an exponent and fields need no shift to bit 0, which takes a third of the integer instructions out (the integer
// pipe bounds the conversion).  For the multiplier 2^133 to stay in range the weights are relative to the row's largest
// exponent E (2^-8 for the block that has it, down to 2^-108); 2^E comes back as a factor per token: on the scores for K,
// on the weights P for V.
struct UW {
    uint32_t s, s2, c;      // multipliers of fields at bit 0 and higher up, -offset * weight
};
template <int P>
__device__ __forceinline__ UW umma_weights(int below) {      // steps of two below the row's largest exponent
    const uint32_t d = (uint32_t)min(below, 100) * 0x00800080u;
    UW w;
    w.s = 0x7E007E00u - d;                                             // 2^(133 - 8 - d)
    w.s2 = (P == 4 ? 0x7C007C00u : 0x7D007D00u) - d;                   // / 16, / 4
    w.c = (P == 4 ? 0xBD00BD00u : P == 6 ? 0xBE00BE00u : 0xBF00BF00u) - d;     // -8, -32, -128 times 2^(-8 - d)
    return w;
}
// Exponent bytes of a row as (byte j: slots 32 j ..) or, for blocks of 16, two words (byte j: slots 16 j ..).
template <bool N16>
__device__ __forceinline__ void umma_exps(const uint8_t* e, int row_e, uint32_t (&w)[2]) {
    if (N16) {
        const uint2 x = *reinterpret_cast<const uint2*>(e);
        w[0] = x.x;
        w[1] = x.y;
    } else {
        w[0] = row_e == 4 ? *reinterpret_cast<const uint32_t*>(e)
               : row_e == 2 ? prmt(*reinterpret_cast<const uint16_t*>(e), 0u, 0x1100u) : prmt(*e, 0u, 0u);
        w[1] = w[0];
    }
}
// The row's blocks (4 or 8) relative to its largest exponent byte, which is returned (254 at most).
template <int P, bool N16>
__device__ __forceinline__ int umma_row(const uint32_t (&w)[2], UW (&g)[N16 ? 8 : 4]) {
    int e[N16 ? 8 : 4], top = 0;
#pragma unroll
    for (int j = 0; j < (N16 ? 8 : 4); ++j) {
        e[j] = (int)((w[j >> 2] >> (8 * (j & 3))) & 0xffu);
        top = max(top, e[j]);
    }
#pragma unroll
    for (int j = 0; j < (N16 ? 8 : 4); ++j) g[j] = umma_weights<P>(top - e[j]);
    return min(top, 254);
}
// 32 slots (four 16-byte pieces of bf16) of a packed row, from slot 32 i on.
template <int P>
__device__ __forceinline__ void convert32(const uint8_t* tile, int row, int i, const UW& g0, const UW& g1, uint32_t (&r)[16]) {
    if (P == 4) {
        const int line = row >> 1, at = ((row & 1) << 6) ^ ((line & 7) << 4);
        const uint4 x = *reinterpret_cast<const uint4*>(tile + line * 128 + (at ^ (16 * i)));
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const UW& g = j < 2 ? g0 : g1;
            const uint32_t y = w[j] >> 8;
            r[4 * j] = fma_bf16x2(w[j] & 0x000F000Fu, g.s, g.c);
            r[4 * j + 1] = fma_bf16x2(w[j] & 0x00F000F0u, g.s2, g.c);
            r[4 * j + 2] = fma_bf16x2(y & 0x000F000Fu, g.s, g.c);
            r[4 * j + 3] = fma_bf16x2(y & 0x00F000F0u, g.s2, g.c);
        }
    } else if (P == 8) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint4 x = *reinterpret_cast<const uint4*>(tile + row * 128 + ((32 * i + 16 * h) ^ ((row & 7) << 4)));
            const uint32_t w[4] = {x.x, x.y, x.z, x.w};
            const UW& g = h ? g1 : g0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                r[8 * h + 2 * j] = fma_bf16x2(w[j] & 0x00FF00FFu, g.s, g.c);
                r[8 * h + 2 * j + 1] = fma_bf16x2(prmt(w[j], 0u, 0x4341u), g.s, g.c);
            }
        }
    } else {
        uint32_t w[6];
#pragma unroll
        for (int j = 0; j < 3; ++j) {
            const uint2 x = *reinterpret_cast<const uint2*>(tile + row * 96 + 24 * i + 8 * j);
            w[2 * j] = x.x;
            w[2 * j + 1] = x.y;
        }
        // eight slots are two runs of three bytes; a 16-bit half holds bytes 0, 1 (then 1, 2) of the first run, the other
        // half those of the second: slots 0 | 4, 1 | 5 and 2 | 6, 3 | 7
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int b = 6 * j, word = b >> 2;                      // first byte of the eight slots: 0, 6, 12, 18
            const bool odd = (b & 3) != 0;
            const uint32_t lo = prmt(w[word], w[word + 1], odd ? 0x6532u : 0x4310u), hi = prmt(w[word], w[word + 1], odd ? 0x7643u : 0x5421u);
            const UW& g = j < 2 ? g0 : g1;
            r[4 * j] = fma_bf16x2(lo & 0x003F003Fu, g.s, g.c);
            r[4 * j + 1] = fma_bf16x2((lo >> 4) & 0x00FC00FCu, g.s2, g.c);
            r[4 * j + 2] = fma_bf16x2((hi >> 2) & 0x00FC00FCu, g.s2, g.c);
            r[4 * j + 3] = fma_bf16x2((hi >> 8) & 0x00FC00FCu, g.s2, g.c);
        }
    }
}

// Sums (MAX: maxima) of C values a thread over the lanes of a warp: afterwards lane l holds column l >> (5 - log2 C).
template <int C, bool MAX>
__device__ __forceinline__ float across_lanes(float (&v)[C], int lane) {
#pragma unroll
    for (int step = 0; step < 5; ++step) {
        const int off = 16 >> step, have = C >> step;          // columns left before this step
        if (have > 1) {
            const bool upper = (lane & off) != 0;
#pragma unroll
            for (int j = 0; j < C / 2; ++j)
                if (j < have / 2) {
                    const float keep = upper ? v[j + have / 2] : v[j], give = upper ? v[j] : v[j + have / 2];
                    const float got = __shfl_xor_sync(0xffffffffu, give, off);
                    v[j] = MAX ? fmaxf(keep, got) : keep + got;
                }
        } else {
            const float got = __shfl_xor_sync(0xffffffffu, v[0], off);
            v[0] = MAX ? fmaxf(v[0], got) : v[0] + got;
        }
    }
    return v[0];
}

template <int P, bool N16, int N>
__global__ void __launch_bounds__(kUThreads, 1) attn_umma(const AttnArgs a, const __grid_constant__ CUtensorMap k_map,
                                                          const __grid_constant__ CUtensorMap v_map) {
    using G_ = UGeo<P, N>;
    constexpr int D = kHeadDim, ROW_M = G_::ROW_M, STAGES = G_::STAGES, C = N / 2, SWP = 2 * N;      // bytes of a P line
    constexpr uint32_t TM_S = 0, TM_O = 2 * N, TM_K = 4 * N, TM_COLS = 4 * N + 128 <= 256 ? 256 : 512;
    extern __shared__ __align__(1024) uint8_t smem[];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int row_e = D / a.fmt.block, exp_half = kUTile * row_e;
    uint8_t* rest = smem + G_::E_OFF + STAGES * 2 * exp_half;
    float* kfac = reinterpret_cast<float*>(rest);            // 2^E of the K and V rows of four tiles
    float* vfac = kfac + 4 * kUTile;
    RowInfo* ri_all = reinterpret_cast<RowInfo*>(vfac + 4 * kUTile);
    int* dpos_all = reinterpret_cast<int*>(ri_all + N);
    int* chan_all = dpos_all + 2 * kAttnMaxDraft;
    float* mref_all = reinterpret_cast<float*>(chan_all + 2 * D);
    float* mstep_all = mref_all + N;        // step of a reference change, and the factor of the sums so far
    float* mfac_all = mstep_all + N;
    float* lsum_all = mfac_all + N;
    float* red_all = lsum_all + N;          // [8 warps][C]
    int* unset_all = reinterpret_cast<int*>(red_all + 8 * C);     // [2] rows that have seen nothing yet, as a bit mask
    uint32_t* tm_slot = reinterpret_cast<uint32_t*>(unset_all + 2);
    const uint32_t bars = (smem_u32(tm_slot) + 4 + 7) & ~7u;
    const uint32_t b_full = bars, b_empty = bars + 8 * STAGES, b_kv = b_empty + 8 * STAGES, b_qk = b_kv + 16, b_p = b_qk + 16,
                   b_pv = b_p + 16, b_qfull = b_pv + 16, b_qfree = b_qfull + 16;

    if (tid == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(b_full + 8 * s, 1);
            mbar_init(b_empty + 8 * s, 4);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(b_kv + 8 * i, 4);
            mbar_init(b_qk + 8 * i, 1);
            mbar_init(b_p + 8 * i, 8);
            mbar_init(b_pv + 8 * i, 1);
            mbar_init(b_qfull + 8 * i, 1);
            mbar_init(b_qfree + 8 * i, 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async_shared();
    }
    if (warp == 17) tmem_alloc(smem_u32(tm_slot), TM_COLS);
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const uint32_t tm = *tm_slot;
    pdl_wait();       // what umma_prep wrote is read by plain loads below: read-only ones could be moved above this line

    const int B = a.fmt.batch, Hkv = a.fmt.n_kv_heads, HR = Hkv * a.n_row_tiles, max_seq = a.fmt.max_seq;
    const int n_items = a.plan[B] * HR, workers = min(a.workers, n_items), me = blockIdx.x;
    const int i0 = me < workers ? worker_start(me, n_items, workers) : 0;
    const int i1 = me < workers ? worker_start(me + 1, n_items, workers) : 0;
    const int n_mine = i1 - i0;
    struct Cursor {      // an item: sequence, kv head and row tile (hr), tile k of n
        int b, hr, k, n;
    };
    auto seek = [&]() {
        int lo = 0, hi = B - 1;                 // last sequence that begins at or before the item
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (a.plan[mid] * HR <= i0) lo = mid; else hi = mid - 1;
        }
        Cursor c;
        const int c0 = a.plan[lo], in = i0 - c0 * HR;
        c.b = lo;
        c.n = a.plan[lo + 1] - c0;
        c.hr = in / c.n;
        c.k = in - c.hr * c.n;
        return c;
    };
    auto next_pair = [&](Cursor& c) {
        c.k = 0;
        if (++c.hr == HR) {
            c.hr = 0;
            c.n = 0;
            while (c.n == 0 && ++c.b < B) c.n = a.plan[c.b + 1] - a.plan[c.b];
        }
    };
    bool dead = false;          // a wait ran out: no more waits, the flag is up, results are void
    auto wait = [&](uint32_t bar, uint32_t parity) {
        if (!dead && !mbar_try(bar, parity) && !mbar_wait_bounded(bar, parity)) {
            dead = true;
            raise_flag(a.status, KVBFP_FLAG_WAIT_TIMEOUT);
        }
    };

    if (n_mine <= 0) {
        // nothing to do
    } else if (warp == 16) {
        // ================================================================ copies
        if (lane == 0) {
            Cursor c = seek();
            SeqView sv = a.views[c.b];
            bool first = true;
            int run = 0;
            for (int i = 0; i < n_mine && !dead; ++i) {
                if (first) {
                    const int q = run & 1;
                    if (run >= 2) wait(b_qfree + 8 * q, (uint32_t)((run >> 1) - 1) & 1u);
                    mbar_expect_tx(b_qfull + 8 * q, G_::Q_BYTES);
                    bulk_g2s(smem_u32(smem) + G_::Q_OFF + q * G_::Q_BYTES,
                             reinterpret_cast<const uint8_t*>(a.qfrag) + ((int64_t)c.b * HR + c.hr) * G_::Q_BYTES, G_::Q_BYTES, b_qfull + 8 * q);
                    first = false;
                }
                const int s = i % STAGES;
                if (i >= STAGES) wait(b_empty + 8 * s, (uint32_t)(i / STAGES - 1) & 1u);
                if (dead) break;
                const int tt = tile_token(sv, c.k, kUTile);
                const int64_t row0 = ((int64_t)c.b * Hkv + c.hr / a.n_row_tiles) * max_seq + tt;
                const int rows = min(kUTile, max_seq - tt);           // a multiple of 16
                const uint32_t dst = smem_u32(smem) + s * G_::MANT, de = smem_u32(smem) + G_::E_OFF + s * 2 * exp_half, br = b_full + 8 * s;
                const uint32_t mant = (P == 6 ? rows : kUTile) * ROW_M;       // a tiled copy always brings its whole box
                mbar_expect_tx(br, 2 * mant + 2 * rows * row_e);
                if (P == 6) {
                    bulk_g2s(dst, a.k_mant + row0 * ROW_M, mant, br);
                    bulk_g2s(dst + G_::MANT / 2, a.v_mant + row0 * ROW_M, mant, br);
                } else {
                    const int y = (int)(P == 4 ? row0 >> 1 : row0);
                    tensor_g2s_2d(dst, &k_map, 0, y, br);
                    tensor_g2s_2d(dst + G_::MANT / 2, &v_map, 0, y, br);
                }
                bulk_g2s(de, a.k_exp + row0 * row_e, rows * row_e, br);
                bulk_g2s(de + exp_half, a.v_exp + row0 * row_e, rows * row_e, br);
                if (++c.k == c.n) {
                    const int b = c.b;
                    next_pair(c);
                    if (c.b != b && c.b < B) sv = a.views[c.b];
                    first = true;
                    ++run;
                }
            }
            if (dead)       // give the copies still in flight a bounded chance to land before the shared memory is released
                for (int s = 0; s < STAGES; ++s) {
                    (void)mbar_wait_bounded(b_full + 8 * s, 0);
                    (void)mbar_wait_bounded(b_full + 8 * s, 1);
                }
        }
    } else if (warp == 17) {
        // ================================================================ matrix instructions
        constexpr uint32_t id_s = umma_idesc(128, N, false, false), id_o = umma_idesc(128, N, true, true);
        const uint32_t tmu = __shfl_sync(0xffffffffu, tm, 0), base = smem_u32(smem);
        Cursor c = seek();
        int run = 0, vslot = 0;
        bool first = true, o_first = true;       // first tile of its run: the tile whose S comes next / whose O comes next
        auto product_o = [&](int i) {
            const int b = i & 1;
            wait(b_p + 8 * b, (uint32_t)(i >> 1) & 1u);
            __syncwarp();
            tmem_fence_after();
            const uint64_t v = umma_desc<128>(base + G_::V_OFF + vslot * G_::V_BYTES, kUTile * 128, 1024);
            const uint64_t p = umma_desc<SWP>(base + G_::P_OFF + b * G_::P_BYTES, 16, 8 * SWP);
#pragma unroll
            for (int ks = 0; ks < kUTile / 16; ++ks)
                umma_ss(tmu + TM_O, v + ks * (2048 >> 4), p + ks * (16 * SWP >> 4), id_o, ks > 0 || !o_first);
            umma_commit(b_pv + 8 * b);
            vslot = vslot == G_::VBUF - 1 ? 0 : vslot + 1;
        };
        for (int i = 0; i < n_mine; ++i) {
            const int b = i & 1, q = run & 1;
            wait(b_kv + 8 * b, (uint32_t)(i >> 1) & 1u);
            if (first) wait(b_qfull + 8 * q, (uint32_t)(run >> 1) & 1u);
            __syncwarp();
            tmem_fence_after();
            const uint64_t qd = umma_desc<128>(base + G_::Q_OFF + q * G_::Q_BYTES, 16, 1024);
#pragma unroll
            for (int ks = 0; ks < 8; ++ks)
                umma_ts(tmu + TM_S + b * N, tmu + TM_K + b * 64 + ks * 8, qd + (((ks >> 2) * (N * 128) + (ks & 3) * 32) >> 4), id_s, ks > 0);
            umma_commit(b_qk + 8 * b);
            const bool was_first = first;
            first = false;
            if (++c.k == c.n) {
                umma_commit(b_qfree + 8 * q);
                next_pair(c);
                first = true;
                ++run;
            }
            if (i > 0) product_o(i - 1);
            o_first = was_first;
        }
        product_o(n_mine - 1);
        if (__any_sync(0xffffffffu, dead)) {       // let what was issued come to its end before the tensor memory goes
            umma_commit(b_qfree);
            (void)mbar_wait_bounded(b_qfree, 0);
            (void)mbar_wait_bounded(b_qfree, 1);
        }
    } else if (warp >= 8) {
        // ================================================================ conversion: a thread per token
        const int grp = (warp - 8) >> 2, row = tid & 127;
        const uint32_t tk = tm + TM_K + grp * 64 + ((uint32_t)(warp & 3) << 21);        // lane field: 32 * quarter << 16
        int vslot = grp;
        for (int i = grp; i < n_mine; i += 2) {
            const int s = i % STAGES;
            wait(b_full + 8 * s, (uint32_t)(i / STAGES) & 1u);
            const uint8_t* km = smem + s * G_::MANT;
            const uint8_t* ke = smem + G_::E_OFF + s * 2 * exp_half + row * row_e;
            if (i >= 2) {
                wait(b_qk + 8 * grp, (uint32_t)((i >> 1) - 1) & 1u);            // K of the tile before is used up
                tmem_fence_after();
            }
            __syncwarp();
            UW g[N16 ? 8 : 4];
            uint32_t ew[2];
            umma_exps<N16>(ke, row_e, ew);
            int top = umma_row<P, N16>(ew, g);
            kfac[(i & 3) * kUTile + row] = __uint_as_float((uint32_t)top << 23);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t r[16];
                convert32<P>(km, row, j, g[N16 ? 2 * j : j], g[N16 ? 2 * j + 1 : j], r);
                tmem_st<16>(tk + 16 * j, r);
            }
            umma_exps<N16>(ke + exp_half, row_e, ew);
            top = umma_row<P, N16>(ew, g);
            vfac[(i & 3) * kUTile + row] = __uint_as_float((uint32_t)max(top - 9, 0) << 23);
            // the buffer's last tile was i - VBUF
            if (i >= G_::VBUF) wait(b_pv + 8 * ((i - G_::VBUF) & 1), (uint32_t)((i - G_::VBUF) >> 1) & 1u);
            uint8_t* vb = smem + G_::V_OFF + vslot * G_::V_BYTES + row * 128;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t r[16];
                convert32<P>(km + G_::MANT / 2, row, j, g[N16 ? 2 * j : j], g[N16 ? 2 * j + 1 : j], r);
                uint8_t* to = vb + (j >> 1) * (kUTile * 128);
#pragma unroll
                for (int x = 0; x < 4; ++x)       // 16-byte pieces 4 j + x of the row: panel of 64 slots, swizzled
                    *reinterpret_cast<uint4*>(to + (((4 * (j & 1) + x) ^ (row & 7)) << 4)) = make_uint4(r[4 * x], r[4 * x + 1], r[4 * x + 2], r[4 * x + 3]);
            }
            vslot = (vslot + 2) % G_::VBUF;
            __syncwarp();
            tmem_wait_st();
            fence_async_shared();
            tmem_fence_before();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(b_kv + 8 * grp);
                mbar_arrive(b_empty + 8 * s);
            }
        }
    } else {
        // ================================================================ softmax: a thread per token, C of the rows
        const int wg = warp >> 2, m_pos = tid & 127, w4 = warp & 3, bar_id = 1 + wg;
        const uint32_t quarter = (uint32_t)w4 << 21;
        RowInfo* ri = ri_all + wg * C;
        int* dpos = dpos_all + wg * kAttnMaxDraft;
        int* chan = chan_all + wg * D;
        float *mref = mref_all + wg * C, *mstep = mstep_all + wg * C, *mfac = mfac_all + wg * C, *lsum = lsum_all + wg * C, *red = red_all + wg * 4 * C;
        int* unset = unset_all + wg;
        const int R = a.n_draft * a.group;
        const float up = a.scale * (P == 4 ? 64.f : P == 6 ? 16.f : 4.f), to_log2 = 1.4426950408889634f;      // 2^8 2^-(P-2)
        const float cap_in = a.softcap > 0.f ? up / a.softcap * 2.8853900817779268f : 0.f;
        // the column a lane ends up with: its upper log2(C) lane bits
        const int my_col = C == 32 ? lane : C == 16 ? lane >> 1 : lane >> 2;
        const bool my_first = C == 32 || (C == 16 ? (lane & 1) == 0 : (lane & 3) == 0);

        Cursor c = seek();
        int it = 0;
        while (it < n_mine) {
            const int b = c.b, hk = c.hr / a.n_row_tiles, rt = c.hr - hk * a.n_row_tiles;
            const int k0 = c.k, k1 = min(c.n, k0 + n_mine - it), row0 = rt * N + wg * C;
            const SeqView sv = a.views[b];
            named_sync(bar_id, 128);
            if (m_pos < C) {
                ri[m_pos] = a.rows[((int64_t)b * HR + c.hr) * N + wg * C + m_pos];
                mref[m_pos] = 0.f;
            }
            if (m_pos == 0) *unset = (int)(C == 32 ? 0xffffffffu : (1u << C) - 1u);
            if (a.tree && m_pos < kAttnMaxDraft) dpos[m_pos] = a.dpos[b * kAttnMaxDraft + m_pos];
            if (a.inv_perm_v) chan[a.inv_perm_v[hk * D + m_pos] & (D - 1)] = m_pos;
            named_sync(bar_id, 128);
            int clear_lo = sv.first;      // tokens [clear_lo, ctx) and [0, pf) are visible to every row
            if (a.window > 0) clear_lo = max(clear_lo, sv.ctx + (a.tree ? a.n_draft - 1 : -1) - a.window + 1);
            float l[C];
#pragma unroll
            for (int j = 0; j < C; ++j) l[j] = 0.f;
            for (int k = k0; k < k1; ++k, ++it) {
                const int s = it & 1, tt = tile_token(sv, k, kUTile), tok = tt + m_pos;
                wait(b_qk + 8 * s, (uint32_t)(it >> 1) & 1u);
                __syncwarp();
                tmem_fence_after();
                uint32_t raw[C];
                tmem_ld<C>(tm + TM_S + s * N + wg * C + quarter, raw);
                tmem_wait_ld(raw);
                float y[C];
#pragma unroll
                for (int j = 0; j < C; ++j) y[j] = __uint_as_float(raw[j]);
                // ---- cap, bias, masks: y * mul in log2 units
                const float kf = kfac[(it & 3) * kUTile + m_pos];
                float mul = up * to_log2 * kf;
                if (a.softcap > 0.f) {
                    mul = a.softcap * to_log2;
                    const float in = cap_in * kf;
#pragma unroll
                    for (int j = 0; j < C; ++j) y[j] = 1.f - __fdividef(2.f, 1.f + ex2_approx(y[j] * in));      // tanh x = 1 - 2 / (1 + e^2x): about 2e-7 absolute
                }
                if (a.slopes != nullptr || !(tt + kUTile <= sv.ctx && (tt >= clear_lo || tt + kUTile <= sv.pf))) {
                    const bool in_ctx = tok < sv.ctx;
                    const int jd = in_ctx ? 0 : min(tok - sv.ctx, kAttnMaxDraft - 1);
                    const bool drafted = !in_ctx && tok - sv.ctx < sv.nd;
                    const int kpos = in_ctx || !drafted ? tok : dpos[jd];
                    const bool always = tok < sv.pf, from = tok >= sv.first;
#pragma unroll
                    for (int j = 0; j < C; ++j) {
                        const RowInfo x = ri[j];
                        const int dist = x.pos - kpos;
                        const bool near = a.window == 0 || dist < a.window;
                        const bool bit = (((jd < 32 ? x.m0 : x.m1) >> (jd & 31)) & 1u) != 0u;
                        const bool see = in_ctx ? (from && near) || always : drafted && bit && near;
                        y[j] = see ? y[j] * mul - x.slope * to_log2 * (float)dist : -INFINITY;
                    }
                    mul = 1.f;
                }
                if (a.scores && tok < max_seq) {
                    float* to = a.scores + ((int64_t)b * a.n_q_heads + hk * a.group + row0) * max_seq + tok;
#pragma unroll
                    for (int j = 0; j < C; ++j)
                        if (row0 + j < R) to[(int64_t)j * max_seq] = y[j] * mul;
                }
                // ---- running softmax against the references
                float top = -INFINITY;
#pragma unroll
                for (int j = 0; j < C; ++j) {
                    y[j] = fmaf(y[j], mul, -mref[j]);
                    top = fmaxf(top, y[j]);
                }
                if (named_any(bar_id, 128, top > 8.f || *unset != 0)) {
                    float v[C];
#pragma unroll
                    for (int j = 0; j < C; ++j) v[j] = y[j];
                    const float mine = across_lanes<C, true>(v, lane);
                    if (my_first) red[w4 * C + my_col] = mine;
                    named_sync(bar_id, 128);
                    if (m_pos < 32) {
                        float step = 0.f;
                        bool none = false;
                        if (lane < C) {
                            const float x = fmaxf(fmaxf(red[lane], red[C + lane]), fmaxf(red[2 * C + lane], red[3 * C + lane]));
                            const bool is_unset = (*unset >> lane) & 1;
                            none = is_unset && x == -INFINITY;
                            step = none ? 0.f : (is_unset ? x : fmaxf(x, 0.f));
                            mstep[lane] = step;
                            mfac[lane] = is_unset ? 1.f : ex2_approx(-step);      // (a row that has seen nothing has sums 0)
                            mref[lane] += step;
                        }
                        const uint32_t left = __ballot_sync(0xffffffffu, none);
                        if (lane == 0) *unset = (int)left;
                    }
                    named_sync(bar_id, 128);
#pragma unroll
                    for (int j = 0; j < C; ++j) {
                        y[j] -= mstep[j];
                        l[j] *= mfac[j];
                    }
                    if (k > k0) {
                        wait(b_pv + 8 * (s ^ 1), (uint32_t)((it - 1) >> 1) & 1u);
                        __syncwarp();
                        tmem_fence_after();
#pragma unroll
                        for (int j = 0; j < C; j += 8) {
                            uint32_t o[8];
                            const uint32_t at = tm + TM_O + wg * C + j + quarter;
                            tmem_ld<8>(at, o);
                            tmem_wait_ld(o);
#pragma unroll
                            for (int e = 0; e < 8; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * mfac[j + e]);
                            tmem_st<8>(at, o);
                        }
                        tmem_wait_st();
                    }
                }
                // ---- P: weights of this token, bf16, a line of 2 N bytes
                if (it >= 2) wait(b_pv + 8 * s, (uint32_t)((it >> 1) - 1) & 1u);
                uint8_t* pb = smem + G_::P_OFF + s * G_::P_BYTES;
                const float vf = vfac[(it & 3) * kUTile + m_pos];
#pragma unroll
                for (int j = 0; j < C; j += 8) {
                    uint32_t w[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float p0 = ex2_approx(y[j + 2 * e]), p1 = ex2_approx(y[j + 2 * e + 1]);
                        l[j + 2 * e] += p0;
                        l[j + 2 * e + 1] += p1;
                        w[e] = pack_bf16x2_rn(p0 * vf, p1 * vf);
                    }
                    const uint32_t off = m_pos * SWP + (wg * C + j) * 2;
                    *reinterpret_cast<uint4*>(pb + (off ^ (((off >> 7) & (SWP / 16 - 1)) << 4))) = make_uint4(w[0], w[1], w[2], w[3]);
                }
                fence_async_shared();
                tmem_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(b_p + 8 * s);
            }
            // ---- the run's result: this thread holds slot umma_slot(m_pos) of C rows
            {
                const float mine = across_lanes<C, false>(l, lane);
                if (my_first) red[w4 * C + my_col] = mine;
            }
            wait(b_pv + 8 * ((it - 1) & 1), (uint32_t)((it - 1) >> 1) & 1u);
            __syncwarp();
            tmem_fence_after();
            named_sync(bar_id, 128);
            const bool whole = k0 == 0 && k1 == c.n;
            const int slot = umma_slot<P>(m_pos);
            float* part = a.partials + ((int64_t)(2 * me + (k0 == 0 ? 1 : 0)) * a.part_rows + wg * C) * kAttnPart;
            if (m_pos < C) {
                const int row = row0 + m_pos;
                const float ls = red[m_pos] + red[C + m_pos] + red[2 * C + m_pos] + red[3 * C + m_pos];
                const float m = ((*unset >> m_pos) & 1) ? -3.4028235e38f : mref[m_pos];
                lsum[m_pos] = ls;
                if (row < R) {
                    const int i = row / a.group, hq = hk * a.group + row - i * a.group;
                    if (!whole) {
                        part[m_pos * kAttnPart + D] = m;
                        part[m_pos * kAttnPart + D + 1] = ls;
                    } else if (a.lse) {
                        a.lse[(int64_t)b * a.n_q_heads + hq] = ls > 0.f ? m + log2f(ls) : (ls == 0.f ? INFINITY : ls);
                    }
                }
            }
            named_sync(bar_id, 128);
            const int ch = a.inv_perm_v ? chan[slot] : slot;
#pragma unroll
            for (int j = 0; j < C; j += 8) {
                uint32_t o[8];
                tmem_ld<8>(tm + TM_O + wg * C + j + quarter, o);
                tmem_wait_ld(o);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int row = row0 + j + e;
                    if (row < R) {
                        if (whole) {
                            const int i = row / a.group, hq = hk * a.group + row - i * a.group;
                            const float ls = lsum[j + e];
                            const bool live = (!a.tree || i < sv.nd) && ls != 0.f;
                            const float v = live ? __uint_as_float(o[e]) * (a.out_up / ls) : 0.f;
                            static_cast<__nv_bfloat16*>(a.out)[(((int64_t)b * a.n_draft + i) * a.n_q_heads + hq) * D + ch] = __float2bfloat16_rn(v);
                        } else {
                            part[(j + e) * kAttnPart + slot] = __uint_as_float(o[e]);
                        }
                    }
                }
            }
            tmem_fence_before();
            c.k = k1;
            if (k1 == c.n) next_pair(c);
        }
    }
    __syncwarp();
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    if (warp == 17) tmem_dealloc(tm, TM_COLS);
    pdl_trigger();
}

template <int P, bool N16, int N>
kvbfp_status launch_umma(const AttnArgs& a, int grid, cudaStream_t s) {
    using G_ = UGeo<P, N>;
    auto kernel = attn_umma<P, N16, N>;
    static std::atomic<bool> attr_set[64];      // per device; setting the attribute twice is harmless
    int dev = 0;
    KVBFP_CUDA(cudaGetDevice(&dev));
    if (dev < 0 || dev >= 64) return KVBFP_ERR_UNSUPPORTED;
    if (!attr_set[dev].load(std::memory_order_acquire)) {
        KVBFP_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, G_::smem_bytes(8)));
        attr_set[dev].store(true, std::memory_order_release);
    }
    CUtensorMap k_map, v_map;
    if (P != 6) {
        const uint64_t rows = (uint64_t)a.fmt.batch * a.fmt.n_kv_heads * a.fmt.max_seq * P / 8;     // lines of 128 bytes
        kvbfp_status st = make_row_map(&k_map, a.k_mant, rows, 128, kUTile * P / 8);
        if (st == KVBFP_OK) st = make_row_map(&v_map, a.v_mant, rows, 128, kUTile * P / 8);
        if (st != KVBFP_OK) return st;
    }
    KVBFP_CUDA(launch_pdl(umma_prep<P, N>, dim3(a.fmt.batch * a.fmt.n_kv_heads * a.n_row_tiles), dim3(128), 0, s, a));
    KVBFP_LAUNCH_CHECK("umma_prep");
    KVBFP_CUDA(launch_pdl(kernel, dim3(grid), dim3(kUThreads), G_::smem_bytes(kHeadDim / a.fmt.block), s, a, k_map, v_map));
    KVBFP_LAUNCH_CHECK("attn_umma");
    return KVBFP_OK;
}

template <int P>
kvbfp_status launch_umma_p(const AttnArgs& a, int grid, cudaStream_t s) {
    const bool n16 = a.fmt.block == 16;
    if (a.rows_tile == 16) return n16 ? launch_umma<P, true, 16>(a, grid, s) : launch_umma<P, false, 16>(a, grid, s);
    if (a.rows_tile == 32) return n16 ? launch_umma<P, true, 32>(a, grid, s) : launch_umma<P, false, 32>(a, grid, s);
    return n16 ? launch_umma<P, true, 64>(a, grid, s) : launch_umma<P, false, 64>(a, grid, s);
}

}  // namespace
}  // namespace kvbfp
