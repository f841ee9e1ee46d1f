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
// One persistent thread block per SM, tiles of 128 tokens.  Teams of warps, each a worker with a contiguous range of
// tiles of its own (attn.cuh), a thread per token (three teams of four warps: 4-bit
// rows, up to 32 query rows) or two (two teams of eight: what shared memory holds of wider rows):
//   K rows converted to tensor memory (the A operand of the first product)
//   V rows converted to shared memory (the A operand of the second, slots contiguous) while the first product runs
//   scores from tensor memory: masks, running maximum, P to shared memory
//   at the end of a run O^T from tensor memory to the result or a partial
// While one team waits (for a product, a barrier, a copy) the others work.  A warp per team issues its matrix
// instructions, one warp copies packed tiles into a ring of units that the teams draw from in turn and pi(Q) of the runs.
// (Groups of their own for conversion and softmax, with two to three tiles between them, took twice as long: the buffers
// between the phases were what everything waited for.)
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

// Slot at position `m` of a converted row (the order the fields unpack in); K and V alike.
template <int P>
__device__ __forceinline__ int umma_slot(int m) {
    if (P != 8) return (m & ~7) | ((m & 1) << 2) | ((m >> 1) & 3);
    return (m & ~3) | ((m & 1) << 1) | ((m >> 1) & 1);
}

template <int P, int N>
struct UGeo {
    static constexpr int ROW_M = kHeadDim * P / 8;
    static constexpr int TEAMS = attn_teams(P, N);
    static constexpr int H = TEAMS == 3 ? 1 : 2;                 // threads per token
    static constexpr int WGS = TEAMS * H;                        // groups of four warps
    static constexpr int THREADS = (WGS * 4 + TEAMS + 1) * 32;
    static constexpr int C = N / H;                              // query rows of a thread
    static constexpr int UNIT = kUTile * ROW_M;                  // a tile's K or V rows
    static constexpr int UNITS = P == 4 ? (N == 32 ? 8 : 9) : P == 6 ? (N == 64 ? 6 : 8) : (N == 64 ? 5 : 6);
    static constexpr int QBUF = N == 16 ? 2 : 1;
    static constexpr int V_OFF = UNITS * UNIT;                   // per team: converted V
    static constexpr int V_BYTES = kUTile * kHeadDim * 2;
    static constexpr int P_OFF = V_OFF + TEAMS * V_BYTES;        // per team: P
    static constexpr int P_BYTES = kUTile * N * 2;
    static constexpr int Q_OFF = P_OFF + TEAMS * P_BYTES;        // per team: pi(Q)
    static constexpr int Q_BYTES = N * kHeadDim * 2;
    static constexpr int E_OFF = Q_OFF + TEAMS * QBUF * Q_BYTES; // exponent bytes: UNITS x 128 x row_e
    // behind them (in floats), per group of four warps: row data, drafted positions and view of two runs, references,
    // steps, factors, sums, reduction, channel table; then barriers
    static constexpr int F_RI = 0, F_DPOS = F_RI + WGS * 2 * C * 4, F_VIEW = F_DPOS + WGS * 2 * kAttnMaxDraft,
                         F_MREF = F_VIEW + WGS * 2 * 8, F_STEP = F_MREF + WGS * C, F_FAC = F_STEP + WGS * C, F_SUM = F_FAC + WGS * C,
                         F_RED = F_SUM + WGS * C, F_CHAN = F_RED + WGS * 4 * C, F_UNSET = F_CHAN + WGS * kHeadDim, F_END = F_UNSET + 6;
    static constexpr int SMALL = F_END * 4 + (2 * UNITS + TEAMS * (4 + 2 * QBUF)) * 8;
    __host__ __device__ static int smem_bytes(int row_e) { return E_OFF + UNITS * kUTile * row_e + SMALL; }
    // tensor memory columns of a team: K, S, O
    static constexpr uint32_t TM_K = 0, TM_S = 64, TM_O = 64 + N, TM_TEAM = 64 + 2 * N, TM_COLS = TEAMS * TM_TEAM <= 256 ? 256 : 512;
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
// The blocks of a row (H = 1) or of its half (slots 64 half ..) relative to the whole row's largest exponent byte, which
// is returned (254 at most).
template <int P, bool N16, int H>
__device__ __forceinline__ int umma_row(const uint32_t (&w)[2], int half, UW (&g)[(N16 ? 8 : 4) / H]) {
    constexpr int NB = N16 ? 8 : 4;
    int top = 0;
#pragma unroll
    for (int j = 0; j < NB; ++j) top = max(top, (int)((w[j >> 2] >> (8 * (j & 3))) & 0xffu));
#pragma unroll
    for (int j = 0; j < NB / H; ++j) {
        uint32_t e = w[j >> 2] >> (8 * (j & 3));
        if (H == 2) e = (N16 ? (half ? w[1] : w[0]) : w[0] >> (16 * half)) >> (8 * j);
        g[j] = umma_weights<P>(top - (int)(e & 0xffu));
    }
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
__global__ void __launch_bounds__(UGeo<P, N>::THREADS, 1) attn_umma(const AttnArgs a, const __grid_constant__ CUtensorMap k_map,
                                                          const __grid_constant__ CUtensorMap v_map) {
    using G_ = UGeo<P, N>;
    constexpr int D = kHeadDim, ROW_M = G_::ROW_M, UNITS = G_::UNITS, QBUF = G_::QBUF, C = G_::C, H = G_::H, TEAMS = G_::TEAMS;
    constexpr int TEAM_WARPS = G_::WGS * 4, SWP = 2 * N;      // bytes of a P line
    extern __shared__ __align__(1024) uint8_t smem[];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int row_e = D / a.fmt.block, exp_unit = kUTile * row_e;
    float* fl = reinterpret_cast<float*>(smem + G_::E_OFF + UNITS * exp_unit);
    uint32_t* tm_slot = reinterpret_cast<uint32_t*>(fl + G_::F_UNSET + 4);
    const uint32_t bars = smem_u32(fl + G_::F_END);
    // ring: full, empty; per team: K ready, S done, P ready, O done, pi(Q) full, pi(Q) free
    const uint32_t b_full = bars, b_empty = bars + 8 * UNITS, b_team = b_empty + 8 * UNITS;
    constexpr int TB = 8 * (4 + 2 * QBUF);
    auto b_k = [&](int t) { return b_team + t * TB; };
    auto b_s = [&](int t) { return b_team + t * TB + 8; };
    auto b_p = [&](int t) { return b_team + t * TB + 16; };
    auto b_o = [&](int t) { return b_team + t * TB + 24; };
    auto b_qfull = [&](int t, int q) { return b_team + t * TB + 32 + 8 * q; };
    auto b_qfree = [&](int t, int q) { return b_team + t * TB + 32 + 8 * (QBUF + q); };

    if (tid == 0) {
        for (int s = 0; s < UNITS; ++s) {
            mbar_init(b_full + 8 * s, 1);
            mbar_init(b_empty + 8 * s, 4 * H);
        }
        for (int t = 0; t < TEAMS; ++t) {
            mbar_init(b_k(t), 4 * H);
            mbar_init(b_s(t), 1);
            mbar_init(b_p(t), 4 * H);
            mbar_init(b_o(t), 1);
            for (int q = 0; q < QBUF; ++q) {
                mbar_init(b_qfull(t, q), 1);
                mbar_init(b_qfree(t, q), 1);
            }
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async_shared();
    }
    if (warp == TEAM_WARPS) tmem_alloc(smem_u32(tm_slot), G_::TM_COLS);
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const uint32_t tm = *tm_slot;
    pdl_wait();       // what umma_prep wrote is read by plain loads below: read-only ones could be moved above this line

    const int B = a.fmt.batch, Hkv = a.fmt.n_kv_heads, HR = Hkv * a.n_row_tiles, max_seq = a.fmt.max_seq;
    const int n_items = a.plan[B] * HR, workers = min(a.workers, n_items);
    // team t of this block is worker blockIdx + t * blocks: few tiles are spread over the blocks first
    auto range = [&](int t, int& first) {
        const int w = blockIdx.x + t * gridDim.x;
        first = w < workers ? worker_start(w, n_items, workers) : 0;
        return w < workers ? worker_start(w + 1, n_items, workers) - first : 0;
    };
    int start[TEAMS], count[TEAMS], least, last_rank[TEAMS];
#pragma unroll
    for (int t = 0; t < TEAMS; ++t) count[t] = range(t, start[t]);
    // units of the ring in the order they are filled and drawn: K, V of tile s of every team, then those of tile s + 1 ..
    // (counts differ by one at most: behind the least of them some teams are left)
    least = count[0];
#pragma unroll
    for (int t = 1; t < TEAMS; ++t) least = min(least, count[t]);
#pragma unroll
    for (int t = 0, left = 0; t < TEAMS; ++t) {
        last_rank[t] = left;
        left += count[t] > least;
    }
    int total = 0;
#pragma unroll
    for (int t = 0; t < TEAMS; ++t) total += count[t];
    struct Cursor {      // an item: sequence, kv head and row tile (hr), tile k of n
        int b, hr, k, n;
    };
    auto seek = [&](int item) {
        // last sequence that begins at or before the item: 32 looked at per step
        int last = 0;
        for (int b0 = 0; b0 < B; b0 += 32) {
            const bool in = b0 + lane < B && a.plan[b0 + lane] * HR <= item;
            const uint32_t v = __ballot_sync(0xffffffffu, in);
            if (v) last = b0 + 31 - __clz(v);
            if (v != 0xffffffffu) break;
        }
        Cursor c;
        const int c0 = a.plan[last], in = item - c0 * HR;
        c.b = last;
        c.n = max(a.plan[last + 1] - c0, 1);
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
    auto wait = [&](uint32_t bar, int phase) {
        if (!dead && !mbar_try(bar, (uint32_t)phase & 1u) && !mbar_wait_bounded(bar, (uint32_t)phase & 1u)) {
            dead = true;
            raise_flag(a.status, KVBFP_FLAG_WAIT_TIMEOUT);
        }
    };

    if (total == 0) {
        // nothing to do
    } else if (warp == TEAM_WARPS + TEAMS) {
        // ================================================================ copies
        Cursor c[TEAMS];
#pragma unroll
        for (int t = 0; t < TEAMS; ++t) c[t] = seek(start[t]);
        if (lane == 0) {
            bool first[TEAMS];
            int run[TEAMS], issued = 0;
#pragma unroll
            for (int t = 0; t < TEAMS; ++t) {
                first[t] = true;
                run[t] = 0;
            }
            for (int s = 0; s < least + 1 && !dead; ++s) {
#pragma unroll
                for (int t = 0; t < TEAMS; ++t) {
                    if (s >= count[t] || dead) continue;
                    Cursor& x = c[t];
                    if (first[t]) {
                        const int q = run[t] % QBUF, n = run[t] / QBUF;
                        if (n > 0) wait(b_qfree(t, q), n - 1);
                        if (dead) continue;
                        mbar_expect_tx(b_qfull(t, q), G_::Q_BYTES);
                        bulk_g2s(smem_u32(smem) + G_::Q_OFF + (t * QBUF + q) * G_::Q_BYTES,
                                 reinterpret_cast<const uint8_t*>(a.qfrag) + ((int64_t)x.b * HR + x.hr) * G_::Q_BYTES, G_::Q_BYTES, b_qfull(t, q));
                        first[t] = false;
                    }
                    const SeqView sv = a.views[x.b];
                    const int tt = tile_token(sv, x.k, kUTile);
                    const int64_t row0 = ((int64_t)x.b * Hkv + x.hr / a.n_row_tiles) * max_seq + tt;
                    const int rows = min(kUTile, max_seq - tt);           // a multiple of 16
                    const uint32_t mant = (P == 6 ? rows : kUTile) * ROW_M;       // a tiled copy always brings its whole box
#pragma unroll
                    for (int kv = 0; kv < 2; ++kv, ++issued) {
                        const int u = issued % UNITS;
                        if (issued >= UNITS) wait(b_empty + 8 * u, issued / UNITS - 1);
                        if (dead) break;
                        const uint32_t dst = smem_u32(smem) + u * G_::UNIT, de = smem_u32(smem) + G_::E_OFF + u * exp_unit, br = b_full + 8 * u;
                        mbar_expect_tx(br, mant + rows * row_e);
                        if (P == 6) bulk_g2s(dst, (kv ? a.v_mant : a.k_mant) + row0 * ROW_M, mant, br);
                        else tensor_g2s_2d(dst, kv ? &v_map : &k_map, 0, (int)(P == 4 ? row0 >> 1 : row0), br);
                        bulk_g2s(de, (kv ? a.v_exp : a.k_exp) + row0 * row_e, rows * row_e, br);
                    }
                    if (++x.k == x.n) {
                        next_pair(x);
                        first[t] = true;
                        ++run[t];
                    }
                }
            }
            if (dead)       // give the copies still in flight a bounded chance to land before the shared memory is released
                for (int s = 0; s < UNITS; ++s) {
                    (void)mbar_wait_bounded(b_full + 8 * s, 0);
                    (void)mbar_wait_bounded(b_full + 8 * s, 1);
                }
        }
    } else if (warp >= TEAM_WARPS) {
        // ================================================================ matrix instructions of a team
        constexpr uint32_t id_s = umma_idesc(128, N, false, false), id_o = umma_idesc(128, N, true, true);
        const int t = __shfl_sync(0xffffffffu, warp - TEAM_WARPS, 0);
        const uint32_t tmt = __shfl_sync(0xffffffffu, tm, 0) + t * G_::TM_TEAM, base = smem_u32(smem);
        const uint64_t vd = umma_desc<128>(base + G_::V_OFF + t * G_::V_BYTES, kUTile * 128, 1024);
        const uint64_t pd = umma_desc<SWP>(base + G_::P_OFF + t * G_::P_BYTES, 16, 8 * SWP);
        int n_mine = 0, first_item = 0;
#pragma unroll
        for (int x = 0; x < TEAMS; ++x)
            if (x == t) { n_mine = count[x]; first_item = start[x]; }
        Cursor c = seek(first_item);
        int run = 0;
        bool first = true;                       // the tile begins a run
        for (int i = 0; i < n_mine; ++i) {
            const int q = run % QBUF;
            if (first) wait(b_qfull(t, q), run / QBUF);
            wait(b_k(t), i);
            __syncwarp();
            tmem_fence_after();
            const uint64_t qd = umma_desc<128>(base + G_::Q_OFF + (t * QBUF + q) * G_::Q_BYTES, 16, 1024);
#pragma unroll
            for (int ks = 0; ks < 8; ++ks)
                umma_ts(tmt + G_::TM_S, tmt + G_::TM_K + ks * 8, qd + (((ks >> 2) * (N * 128) + (ks & 3) * 32) >> 4), id_s, ks > 0);
            umma_commit(b_s(t));
            const bool fresh = first;
            first = ++c.k == c.n;
            if (first) {
                umma_commit(b_qfree(t, q));
                next_pair(c);
                ++run;
            }
            wait(b_p(t), i);
            __syncwarp();
            tmem_fence_after();
#pragma unroll
            for (int ks = 0; ks < kUTile / 16; ++ks)
                umma_ss(tmt + G_::TM_O, vd + ks * (2048 >> 4), pd + ks * (16 * SWP >> 4), id_o, ks > 0 || !fresh);
            umma_commit(b_o(t));
        }
        if (__any_sync(0xffffffffu, dead)) {       // let what was issued come to its end before the tensor memory goes
            umma_commit(b_s(t));
            (void)mbar_wait_bounded(b_s(t), 0);
            (void)mbar_wait_bounded(b_s(t), 1);
        }
    } else {
        // ================================================================ a team: H threads per token
        const int wg = warp >> 2, team = wg / H, half = H == 2 ? wg & 1 : 0, m_pos = tid & 127, w4 = warp & 3, bar_id = 1 + wg;
        const uint32_t tmt = tm + team * G_::TM_TEAM + ((uint32_t)w4 << 21);        // lane field: 32 * quarter << 16
        float *mref = fl + G_::F_MREF + wg * C, *mstep = fl + G_::F_STEP + wg * C, *mfac = fl + G_::F_FAC + wg * C,
              *lsum = fl + G_::F_SUM + wg * C, *red = fl + G_::F_RED + wg * 4 * C;
        int* chan = reinterpret_cast<int*>(fl + G_::F_CHAN) + wg * D;
        int* unset = reinterpret_cast<int*>(fl + G_::F_UNSET) + wg;         // rows that have seen nothing yet, as a bit mask
        uint8_t* vline = smem + G_::V_OFF + team * G_::V_BYTES + half * (kUTile * 128) + m_pos * 128;       // (a panel holds 64 slots)
        int n_mine = 0, first_item = 0, rank = 0;
#pragma unroll
        for (int x = 0; x < TEAMS; ++x)
            if (x == team) { n_mine = count[x]; first_item = start[x]; rank = last_rank[x]; }
        const int me = blockIdx.x + team * gridDim.x;
        const int R = a.n_draft * a.group;
        const float up = a.scale * (P == 4 ? 64.f : P == 6 ? 16.f : 4.f), to_log2 = 1.4426950408889634f;      // 2^8 2^-(P-2)
        const float cap_in = a.softcap > 0.f ? up / a.softcap * 2.8853900817779268f : 0.f;
        // the column a lane ends up with after across_lanes: its upper log2(C) lane bits
        const int my_col = C == 32 ? lane : C == 16 ? lane >> 1 : lane >> 2;
        const bool my_first = C == 32 || (C == 16 ? (lane & 1) == 0 : (lane & 3) == 0);
        // row data, drafted positions and view of a run, asynchronously into the buffers of its parity
        auto fetch = [&](const Cursor& c, int par) {
            if (c.b < B) {
                if (m_pos < C)
                    cp_async16(smem_u32(fl + G_::F_RI + ((wg * 2 + par) * C + m_pos) * 4), a.rows + ((int64_t)c.b * HR + c.hr) * N + half * C + m_pos);
                else if (m_pos >= 64 && m_pos < 64 + kAttnMaxDraft / 4 && a.tree)
                    cp_async16(smem_u32(fl + G_::F_DPOS + (wg * 2 + par) * kAttnMaxDraft + (m_pos - 64) * 4), a.dpos + c.b * kAttnMaxDraft + (m_pos - 64) * 4);
                else if (m_pos >= 96 && m_pos < 98)
                    cp_async16(smem_u32(fl + G_::F_VIEW + (wg * 2 + par) * 8 + (m_pos - 96) * 4), reinterpret_cast<const int*>(a.views + c.b) + (m_pos - 96) * 4);
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        Cursor c = seek(first_item), cn = c;
        int unit = 2 * (least > 0 ? team : rank), round = 0;          // the ring's next unit of this team, and how often the ring went round
        fetch(c, 0);
        int it = 0, run = 0;
        while (it < n_mine) {
            const int b = c.b, hk = c.hr / a.n_row_tiles, rt = c.hr - hk * a.n_row_tiles, par = run & 1;
            const int k0 = c.k, k1 = min(c.n, k0 + n_mine - it), row0 = rt * N + half * C;
            cn = c;
            next_pair(cn);
            asm volatile("cp.async.wait_group 0;" ::: "memory");
            if (m_pos < C) mref[m_pos] = 0.f;
            if (m_pos == 0) *unset = (int)(C == 32 ? 0xffffffffu : (1u << C) - 1u);
            if (a.inv_perm_v) chan[a.inv_perm_v[hk * D + m_pos] & (D - 1)] = m_pos;
            named_sync(bar_id, 128);
            if (it + k1 - k0 < n_mine) fetch(cn, par ^ 1);
            const RowInfo* ri = reinterpret_cast<const RowInfo*>(fl + G_::F_RI) + (wg * 2 + par) * C;
            const int* dpos = reinterpret_cast<const int*>(fl + G_::F_DPOS) + (wg * 2 + par) * kAttnMaxDraft;
            const SeqView sv = *reinterpret_cast<const SeqView*>(fl + G_::F_VIEW + (wg * 2 + par) * 8);
            const uint32_t tm_o = tmt + G_::TM_O + half * C;
            int clear_lo = sv.first;      // tokens [clear_lo, ctx) and [0, pf) are visible to every row
            if (a.window > 0) clear_lo = max(clear_lo, sv.ctx + (a.tree ? a.n_draft - 1 : -1) - a.window + 1);
            float l[C];
#pragma unroll
            for (int j = 0; j < C; ++j) l[j] = 0.f;
            for (int k = k0; k < k1; ++k, ++it) {
                // ---- K to tensor memory (the product of the tile before has read it: waited for below, a tile ago), then, while the
                // tensor cores are on S, V to shared memory.  (One loop for both: the code of a tile has to stay in the
                // instruction cache.)
                uint32_t top2[2];
#pragma unroll 1
                for (int kv = 0; kv < 2; ++kv) {
                    wait(b_full + 8 * unit, round);
                    if (kv == 1 && it > 0) wait(b_o(team), it - 1);          // the product of the tile before has read V and P
                    __syncwarp();
                    const uint8_t* tile = smem + unit * G_::UNIT;
                    uint32_t ew[2];
                    umma_exps<N16>(smem + G_::E_OFF + unit * exp_unit + m_pos * row_e, row_e, ew);
                    UW g[(N16 ? 8 : 4) / H];
                    const uint32_t top = (uint32_t)umma_row<P, N16, H>(ew, half, g);
                    if (kv == 0) top2[0] = top; else top2[1] = top;
#pragma unroll
                    for (int j = 0; j < 4 / H; ++j) {
                        uint32_t r[16];
                        convert32<P>(tile, m_pos, 2 * half + j, g[N16 ? 2 * j : j], g[N16 ? 2 * j + 1 : j], r);
                        if (kv == 0) {
                            tmem_st<16>(tmt + G_::TM_K + half * 32 + 16 * j, r);
                        } else {
                            uint8_t* to = vline + (j >> 1) * (kUTile * 128);
#pragma unroll
                            for (int x = 0; x < 4; ++x)       // 16-byte pieces 4 j + x, swizzled
                                *reinterpret_cast<uint4*>(to + (((4 * (j & 1) + x) ^ (m_pos & 7)) << 4)) = make_uint4(r[4 * x], r[4 * x + 1], r[4 * x + 2], r[4 * x + 3]);
                        }
                    }
                    if (kv == 0) {
                        tmem_wait_st();
                        tmem_fence_before();
                    }
                    __syncwarp();
                    if (lane == 0) {
                        if (kv == 0) mbar_arrive(b_k(team));
                        mbar_arrive(b_empty + 8 * unit);
                    }
                    if (kv == 0 && ++unit == UNITS) { unit = 0; ++round; }
                }
                unit += 2 * TEAMS - 1 - (it + 1 == least ? 2 * (team - rank) : 0);
                while (unit >= UNITS) { unit -= UNITS; ++round; }
                const uint32_t k_top = top2[0], v_top = top2[1];
                // ---- scores
                const int tt = tile_token(sv, k, kUTile), tok = tt + m_pos;
                const float kf = __uint_as_float(k_top << 23), vf = __uint_as_float((uint32_t)max((int)v_top - 9, 0) << 23);
                wait(b_s(team), it);
                __syncwarp();
                tmem_fence_after();
                uint32_t raw[C];
                tmem_ld<C>(tmt + G_::TM_S + half * C, raw);
                tmem_wait_ld(raw);
                float y[C];
#pragma unroll
                for (int j = 0; j < C; ++j) y[j] = __uint_as_float(raw[j]);
                // ---- cap, bias, masks: y * mul in log2 units
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
                        bool none = false;
                        if (lane < C) {
                            const float x = fmaxf(fmaxf(red[lane], red[C + lane]), fmaxf(red[2 * C + lane], red[3 * C + lane]));
                            const bool is_unset = (*unset >> lane) & 1;
                            none = is_unset && x == -INFINITY;
                            const float step = none ? 0.f : (is_unset ? x : fmaxf(x, 0.f));
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
                    if (k > k0) {          // (the product of the tile before is done: waited for above)
                        tmem_fence_after();
#pragma unroll
                        for (int j = 0; j < C; j += 8) {
                            uint32_t o[8];
                            tmem_ld<8>(tm_o + j, o);
                            tmem_wait_ld(o);
#pragma unroll
                            for (int e = 0; e < 8; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * mfac[j + e]);
                            tmem_st<8>(tm_o + j, o);
                        }
                        tmem_wait_st();
                    }
                }
                // ---- P: weights of this token times its V row's 2^E, bf16, a line of 2 N bytes
                uint8_t* pb = smem + G_::P_OFF + team * G_::P_BYTES;
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
                    const uint32_t off = m_pos * SWP + (half * C + j) * 2;
                    *reinterpret_cast<uint4*>(pb + (off ^ (((off >> 7) & (SWP / 16 - 1)) << 4))) = make_uint4(w[0], w[1], w[2], w[3]);
                }
                fence_async_shared();
                tmem_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(b_p(team));
            }
            // ---- the run's result: this thread holds slot umma_slot(m_pos) of C rows
            {
                const float mine = across_lanes<C, false>(l, lane);
                if (my_first) red[w4 * C + my_col] = mine;
            }
            named_sync(bar_id, 128);
            const bool whole = k0 == 0 && k1 == c.n;
            const int slot = umma_slot<P>(m_pos);
            float* part = a.partials + ((int64_t)(2 * me + (k0 == 0 ? 1 : 0)) * a.part_rows + half * C) * kAttnPart;
            if (m_pos < C) {
                const int row = row0 + m_pos;
                const float ls = red[m_pos] + red[C + m_pos] + red[2 * C + m_pos] + red[3 * C + m_pos];
                const float m = ((*unset >> m_pos) & 1) ? -3.4028235e38f : mref[m_pos];
                lsum[m_pos] = ls;
                if (row < R) {
                    if (!whole) {
                        part[m_pos * kAttnPart + D] = m;
                        part[m_pos * kAttnPart + D + 1] = ls;
                    } else if (a.lse) {
                        const int i = row / a.group, hq = hk * a.group + row - i * a.group;
                        a.lse[(int64_t)b * a.n_q_heads + hq] = ls > 0.f ? m + log2f(ls) : (ls == 0.f ? INFINITY : ls);
                    }
                }
            }
            wait(b_o(team), it - 1);
            __syncwarp();
            tmem_fence_after();
            named_sync(bar_id, 128);
            const int ch = a.inv_perm_v ? chan[slot] : slot;
#pragma unroll 1
            for (int j = 0; j < C; j += 8) {
                uint32_t o[8];
                tmem_ld<8>(tm_o + j, o);
                tmem_wait_ld(o);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int row = row0 + j + e;
                    if (row >= R) break;
                    if (whole) {
                        const int i = row / a.group, hq = hk * a.group + row - i * a.group;
                        const float ls = lsum[j + e];
                        const bool live = (!a.tree || i < sv.nd) && ls != 0.f;
                        static_cast<__nv_bfloat16*>(a.out)[(((int64_t)b * a.n_draft + i) * a.n_q_heads + hq) * D + ch] =
                            __float2bfloat16_rn(live ? __uint_as_float(o[e]) * (a.out_up / ls) : 0.f);
                    } else {
                        part[(j + e) * kAttnPart + slot] = __uint_as_float(o[e]);
                    }
                }
            }
            tmem_fence_before();
            c.k = k1;
            if (k1 == c.n) c = cn;
            ++run;
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
    }
    __syncwarp();
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    if (warp == TEAM_WARPS) tmem_dealloc(tm, G_::TM_COLS);
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
    KVBFP_CUDA(launch_pdl(kernel, dim3(grid), dim3(G_::THREADS), G_::smem_bytes(kHeadDim / a.fmt.block), s, a, k_map, v_map));
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
