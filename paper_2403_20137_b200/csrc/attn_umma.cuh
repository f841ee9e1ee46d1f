// Attention of drafted trees with 9 to 64 bf16 query rows per (batch, kv head), or more in items of 64, over the packed
// cache on the fifth-generation tensor cores.
//
//   S^T[tokens x rows] = K . pi(Q)^T          K: tensor memory, pi(Q): shared memory
//   y = log2(e) * (cap * tanh(scale * S / cap) - slope * distance) ;  P = 2^(y - m)
//   O^T[slots x rows] += V^T . P^T            V, P: shared memory (both with the token as the slow index)
//
// Why: with the query rows as the narrow side of the product a tile of 128 tokens costs the tensor cores rows / 64 x 128
// cycles per product, so what is left to do per cached element is its conversion, and that is done once for all rows
// (the warp-level kernel converts per eight rows and its matrix instructions run at a third of the rate).
//
// One persistent thread block per SM, tiles of 128 tokens.  Teams of warps, each a worker with a contiguous range of
// tiles of its own (attn.cuh), a thread per token (three teams of four warps: 4-bit rows, up to 32 query rows) or two
// (two teams of eight: what shared memory holds of wider rows).  Per tile i a team
//   converts the K rows of tile i + 1 to tensor memory (the A operand of the first product)
//   converts the V rows of tile i to shared memory (the A operand of the second, slots contiguous)
//   reads the scores of tile i from tensor memory: masks, running maximum, P to shared memory
// so that what it needs next was started most of a tile ago: a hand-over between warps takes some 250 cycles, a product
// 150 to 400, a copy 1500.  At the end of a run O^T goes from tensor memory to the result or a partial.  A warp per team
// issues its matrix instructions and the copies of its packed rows and pi(Q).  (One warp that copied for all teams took
// 500 to 1000 cycles per copy: its code had gone from the instruction cache each time.)
// (Groups of their own for conversion and softmax, with two to three tiles between them, took twice as long: the buffers
// between the phases were what everything waited for.)
// Rare paths (masks, raising a reference, results) are loops over eight columns of tensor memory: straight code that is
// not in the instruction cache runs at some nine cycles an instruction.
// Cached values are converted relative to their row's largest exponent (see below); magnitudes of 2^118 and above are
// outside the range.
// The row maximum runs across threads here, so it is only taken when a score passes the reference by 8 (a factor 2^8),
// which a barrier over the group tells; then O is rescaled in tensor memory.  Sums are kept per thread and reduced at
// the end of a run.
//
// What bounds it: neither memory (0.44 of the copy rate at 16 rows) nor the tensor cores (7 to 15 % busy) but the warps'
// instructions and the latency between them: some 700 to 940 a warp and tile, 0.5 to 0.6 issued a cycle by the 12 to 16
// warps that registers and shared memory allow.  16 x 32 heads of up to 8192 4-bit rows, 16 drafted tokens: 119 us; 8 x 8
// heads of 32768 rows, 64 query rows: 156 us; 8 x 8 heads of up to 8191 8-bit rows, 256 capped query rows: 164 us.
// (The instances for 64 rows spill 64 to 84 bytes a thread: 18 warps leave 96 registers.)
// (V^T in tensor memory, filled through transposing loads, halves the shared-memory traffic and was 6 % slower: it costs
// integer instructions.  Conversion as loops instead of straight code: 2 to 6 % slower.)
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
    static constexpr int THREADS = (WGS * 4 + TEAMS) * 32;
    static constexpr int C = N / H;                           // query rows of a thread
    static constexpr int UNIT = kUTile * ROW_M;                  // a tile's K or V rows
    static constexpr int KS = P == 4 && N == 32 || P == 8 && N == 64 ? 1 : 2;       // packed K rows a team keeps
    static constexpr int VS = P == 4 && N == 64 || P == 6 && N <= 32 ? 2 : 1;       // and V rows
    static constexpr int RING = KS + VS, UNITS = TEAMS * RING;
    static constexpr int V_OFF = UNITS * UNIT;                   // per team: converted V
    static constexpr int V_BYTES = kUTile * kHeadDim * 2;
    static constexpr int P_OFF = V_OFF + TEAMS * V_BYTES;        // per team: P
    static constexpr int P_BYTES = kUTile * N * 2;
    static constexpr int Q_OFF = P_OFF + TEAMS * P_BYTES;        // per team: pi(Q)
    static constexpr int Q_BYTES = N * kHeadDim * 2;
    static constexpr int E_OFF = Q_OFF + TEAMS * Q_BYTES;        // exponent bytes: UNITS x 128 x row_e
    // behind them (in floats), per group of four warps: row data, drafted positions and view of two runs, references,
    // factors, sums, reduction, channel table; then barriers
    static constexpr int F_RI = 0, F_DPOS = F_RI + WGS * 2 * C * 4, F_VIEW = F_DPOS + WGS * 2 * kAttnMaxDraft,
                         F_MREF = F_VIEW + WGS * 2 * 8, F_FAC = F_MREF + WGS * C, F_SUM = F_FAC + WGS * C,
                         F_RED = F_SUM + WGS * C, F_CHAN = F_RED + WGS * 4 * C, F_UNSET = F_CHAN + WGS * kHeadDim, F_END = F_UNSET + 8;
    static constexpr int SMALL = F_END * 4 + TEAMS * (RING + 7) * 8;
    __host__ __device__ static int smem_bytes(int row_e) { return E_OFF + UNITS * kUTile * row_e + SMALL; }
    // tensor memory columns of a team: K, two S, O
    static constexpr uint32_t TM_K = 0, TM_S = 64, TM_O = 64 + 2 * N, TM_TEAM = 64 + 3 * N, TM_COLS = TEAMS * TM_TEAM <= 256 ? 256 : 512;
};

// pi(Q) of one (sequence, kv head, row tile) per block, as the shared-memory image of the B operand: two panels of 64
// positions, lines of 128 bytes per row, 16-byte pieces at piece ^ (row % 8).
template <int P, int N>
__global__ void __launch_bounds__(128) umma_prep(const AttnArgs a) {
    __shared__ float sq[N][kHeadDim + 4];
    __shared__ int sp[kHeadDim];
    prep_common<N>(a, sq, sp);
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
// exponent E (2^-8 for the block that has it, down to bf16's last step); 2^E comes back as a factor per token: on the scores for K,
// on the weights P for V.
struct UW {
    uint32_t s, s2, c;      // multipliers of fields at bit 0 and higher up, -offset * weight
};
// Weights of two blocks, `below` (16-bit halves) steps of two below the row's largest exponent.  The other two are products
// of the first, so that far below (from 125 steps on, where no bf16 number is left) all three run out into zeros together.
template <int P>
__device__ __forceinline__ void umma_weights(uint32_t below, UW& a, UW& b) {
    uint32_t d;
    asm("min.s16x2 %0, %1, %2;" : "=r"(d) : "r"(below), "r"(252u * 0x00010001u));
    const uint32_t s = 0x7E007E00u - d * 0x80u;                                      // 2^(133 - 8 - d), 0 at 252
    const uint32_t s2 = mul_bf16x2(s, P == 4 ? 0x3D803D80u : 0x3E803E80u);           // / 16, / 4
    const uint32_t c = mul_bf16x2(s, P == 4 ? 0x80088008u : P == 6 ? 0x80208020u : 0x80808080u);      // -8, -32, -128 times 2^-133
    a.s = prmt(s, 0u, 0x1010u);
    b.s = prmt(s, 0u, 0x3232u);
    a.s2 = prmt(s2, 0u, 0x1010u);
    b.s2 = prmt(s2, 0u, 0x3232u);
    a.c = prmt(c, 0u, 0x1010u);
    b.c = prmt(c, 0u, 0x3232u);
}
__device__ __forceinline__ uint32_t max_s16x2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("max.s16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
// Exponent bytes of a row: byte j for slots 32 j .. (longer blocks: repeated, by the selector `sel` from the aligned word
// that holds them) or, for blocks of 16, two words (byte j: slots 16 j ..).
__device__ __forceinline__ uint32_t umma_exp_sel(int row, int row_e) {
    return row_e == 4 ? 0x3210u : row_e == 2 ? ((row & 1) ? 0x3322u : 0x1100u) : (uint32_t)(row & 3) * 0x1111u;
}
template <bool N16>
__device__ __forceinline__ void umma_exps(const uint8_t* e, uint32_t sel, uint32_t (&w)[2]) {
    if (N16) {
        const uint2 x = *reinterpret_cast<const uint2*>(e);
        w[0] = x.x;
        w[1] = x.y;
    } else {
        w[0] = w[1] = prmt(*reinterpret_cast<const uint32_t*>(e), 0u, sel);
    }
}
// The blocks of a row (H = 1) or of its half (slots 64 half ..) relative to the whole row's largest exponent byte, which
// is returned (254 at most).
template <int P, bool N16, int H>
__device__ __forceinline__ int umma_row(const uint32_t (&w)[2], int half, UW (&g)[(N16 ? 8 : 4) / H]) {
    const uint32_t lo = w[0] & 0x00FF00FFu, hi = prmt(w[0], 0u, 0x4341u);            // blocks 0 | 2, 1 | 3
    uint32_t m = max_s16x2(lo, hi);
    if (N16) m = max_s16x2(m, max_s16x2(w[1] & 0x00FF00FFu, prmt(w[1], 0u, 0x4341u)));
    const int top = max((int)(m & 0xffffu), (int)(m >> 16));
    const uint32_t t2 = (uint32_t)top * 0x00010001u;
    if constexpr (!N16 && H == 2) {
        umma_weights<P>(t2 - prmt(w[0], 0u, half ? 0x4342u : 0x4140u), g[0], g[1]);
    } else {
#pragma unroll
        for (int j = 0; j < (N16 ? 2 : 1) / (N16 ? H : 1); ++j) {
            const uint32_t x = N16 && (H == 2 ? half : j) ? w[1] : w[0];
            umma_weights<P>(t2 - (x & 0x00FF00FFu), g[4 * j], g[4 * j + 2]);
            umma_weights<P>(t2 - prmt(x, 0u, 0x4341u), g[4 * j + 1], g[4 * j + 3]);
        }
    }
    return min(top, 254);
}
// Where a thread finds the row `row` of a unit: the offset whose exclusive or with 16 i (bytes of the row, 16-byte pieces)
// is the piece's place (units start on multiples of 1024).  96-byte rows are not swizzled.
template <int P>
__device__ __forceinline__ uint32_t row_place(int row) {
    if (P == 4) return (row >> 1) * 128 + (((row & 1) << 6) ^ (((row >> 1) & 7) << 4));
    if (P == 8) return row * 128 + ((row & 7) << 4);
    return row * 96;
}
// 32 slots of a packed row, from slot 32 i on, as they are stored; `at`: unit plus row_place.
template <int P>
__device__ __forceinline__ void load32(uint32_t at, int i, uint32_t (&w)[P]) {
    if (P == 6) {
#pragma unroll
        for (int j = 0; j < 3; ++j) {
            const uint2 x = lds64(at + 24 * i + 8 * j);
            w[2 * j] = x.x;
            w[2 * j + 1] = x.y;
        }
    } else {
#pragma unroll
        for (int h = 0; h < P / 4; ++h) {
            const uint4 x = lds128(at ^ (4 * P * i + 16 * h));
            w[4 * h] = x.x;
            w[4 * h + 1] = x.y;
            w[4 * h + 2] = x.z;
            w[4 * h + 3] = x.w;
        }
    }
}
// 32 slots as 16 bf16 pairs (four 16-byte pieces).
template <int P>
__device__ __forceinline__ void convert32(const uint32_t (&w)[P], const UW& g0, const UW& g1, uint32_t (&r)[16]) {
    if (P == 4) {
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
        for (int j = 0; j < 8; ++j) {
            const UW& g = j < 4 ? g0 : g1;
            r[2 * j] = fma_bf16x2(w[j] & 0x00FF00FFu, g.s, g.c);
            r[2 * j + 1] = fma_bf16x2(prmt(w[j], 0u, 0x4341u), g.s, g.c);
        }
    } else {
        // eight slots are two runs of three bytes; a 16-bit half holds bytes 0, 1 (then 1, 2) of the first run, the other
        // half those of the second: slots 0 | 4, 1 | 5 and 2 | 6, 3 | 7
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int b = 6 * j, word = b >> 2;                      // first byte of the eight slots: 0, 6, 12, 18
            const bool odd = (b & 3) != 0;
            const uint32_t lo = prmt(w[word], w[(word + 1) % P], odd ? 0x6532u : 0x4310u), hi = prmt(w[word], w[(word + 1) % P], odd ? 0x7643u : 0x5421u);
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

// Changes the scores of a tile by fn(value, column): up to eight columns a thread stay in registers, more are changed in
// tensor memory, eight at a time.
template <int C, class F>
__device__ __forceinline__ void change_scores(uint32_t tm_s, uint32_t (&raw)[C], F fn) {
    if constexpr (C <= 8) {
#pragma unroll
        for (int e = 0; e < C; ++e) raw[e] = __float_as_uint(fn(__uint_as_float(raw[e]), e));
    } else {
#pragma unroll 1
        for (int j = 0; j < C; j += 8) {
            uint32_t r[8];
            tmem_ld<8>(tm_s + j, r);
            tmem_wait_ld(r);
#pragma unroll
            for (int e = 0; e < 8; ++e) r[e] = __float_as_uint(fn(__uint_as_float(r[e]), j + e));
            tmem_st<8>(tm_s + j, r);
        }
        tmem_wait_st();
    }
}

__device__ __noinline__ bool umma_wait_slow(uint32_t bar, uint32_t parity) { return mbar_wait_bounded(bar, parity); }

template <int P, bool N16, int N>
__global__ void __launch_bounds__(UGeo<P, N>::THREADS, 1) attn_umma(const AttnArgs a, const __grid_constant__ CUtensorMap k_map,
                                                                    const __grid_constant__ CUtensorMap v_map) {
    using G_ = UGeo<P, N>;
    constexpr int D = kHeadDim, ROW_M = G_::ROW_M, UNITS = G_::UNITS, RING = G_::RING, KS = G_::KS, VS = G_::VS, C = G_::C, H = G_::H, TEAMS = G_::TEAMS;
    constexpr bool KEEP = C <= 8;          // scores stay in registers
    constexpr int TEAM_WARPS = G_::WGS * 4, SWP = 2 * N;      // bytes of a P line
    extern __shared__ __align__(1024) uint8_t smem[];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int row_e = D / a.fmt.block, exp_unit = kUTile * row_e;
    float* fl = reinterpret_cast<float*>(smem + G_::E_OFF + UNITS * exp_unit);
    uint32_t* tm_slot = reinterpret_cast<uint32_t*>(fl + G_::F_UNSET + 6);
    // barriers of a team: packed K rows there (KS), packed V rows there (VS), pi(Q) there, K converted, V converted, P written,
    // S done (two), O done
    const uint32_t bars = smem_u32(fl + G_::F_END);
    constexpr int TB = 8 * (RING + 7);
    auto b_kf = [&](int t, int i) { return bars + t * TB + 8 * (i % KS); };
    auto b_vf = [&](int t, int i) { return bars + t * TB + 8 * (KS + i % VS); };
    auto b_q = [&](int t) { return bars + t * TB + 8 * RING; };
    auto b_k = [&](int t) { return bars + t * TB + 8 * RING + 8; };
    auto b_v = [&](int t) { return bars + t * TB + 8 * RING + 16; };
    auto b_p = [&](int t) { return bars + t * TB + 8 * RING + 24; };
    auto b_s = [&](int t, int i) { return bars + t * TB + 8 * RING + 32 + 8 * (i & 1); };
    auto b_o = [&](int t) { return bars + t * TB + 8 * RING + 48; };

    if (tid == 0) {
        for (int t = 0; t < TEAMS; ++t) {
            for (int i = 0; i < KS; ++i) mbar_init(b_kf(t, i), 1);
            for (int i = 0; i < VS; ++i) mbar_init(b_vf(t, i), 1);
            mbar_init(b_q(t), 1);
            mbar_init(b_k(t), 4 * H);
            mbar_init(b_v(t), 4 * H);
            mbar_init(b_p(t), 4 * H);
            mbar_init(b_s(t, 0), 1);
            mbar_init(b_s(t, 1), 1);
            mbar_init(b_o(t), 1);
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
        if (!mbar_try(bar, (uint32_t)phase & 1u) && !dead && !umma_wait_slow(bar, (uint32_t)phase & 1u)) {
            dead = true;
            raise_flag(a.status, KVBFP_FLAG_WAIT_TIMEOUT);
        }
    };

    if (warp >= TEAM_WARPS) {
        // ================================================================ matrix instructions and copies of a team
        constexpr uint32_t id_s = umma_idesc(128, N, false, false), id_o = umma_idesc(128, N, true, true);
        const int t = __shfl_sync(0xffffffffu, warp - TEAM_WARPS, 0);
        const uint32_t tmt = __shfl_sync(0xffffffffu, tm, 0) + t * G_::TM_TEAM, base = smem_u32(smem);
        const uint64_t vd = umma_desc<128>(base + G_::V_OFF + t * G_::V_BYTES, kUTile * 128, 1024);
        const uint64_t pd = umma_desc<SWP>(base + G_::P_OFF + t * G_::P_BYTES, 16, 8 * SWP);
        const uint64_t qd = umma_desc<128>(base + G_::Q_OFF + t * G_::Q_BYTES, 16, 1024);
        int first_item;
        const int n_mine = range(t, first_item);
        struct Walk {                  // the next packed rows to copy: cursor, np and lo of the sequence's view
            Cursor c;
            int np, lo;
        };
        Cursor c = seek(first_item);
        Walk wk = {c, a.views[c.b].np, a.views[c.b].lo}, wv = wk;
        auto copy = [&](Walk& w, int u, uint32_t bar, const uint8_t* mant_plane, const CUtensorMap* map, const uint8_t* exp_plane) {
            const int tt = (w.c.k < w.np ? w.c.k : w.c.k - w.np + w.lo) * kUTile;
            const int64_t row0 = ((int64_t)w.c.b * Hkv + w.c.hr / a.n_row_tiles) * max_seq + tt;
            const int rows = min(kUTile, max_seq - tt);           // a multiple of 16
            const uint32_t mant = (P == 6 ? rows : kUTile) * ROW_M;       // a tiled copy always brings its whole box
            if (lane == 0) {
                mbar_expect_tx(bar, mant + rows * row_e);
                if (P == 6) bulk_g2s(base + u * G_::UNIT, mant_plane + row0 * ROW_M, mant, bar);
                else tensor_g2s_2d(base + u * G_::UNIT, map, 0, (int)(P == 4 ? row0 >> 1 : row0), bar);
                bulk_g2s(base + G_::E_OFF + u * exp_unit, exp_plane + row0 * row_e, rows * row_e, bar);
            }
            if (++w.c.k == w.c.n) {
                const int b = w.c.b;
                next_pair(w.c);
                if (w.c.b != b && w.c.b < B) { w.np = a.views[w.c.b].np; w.lo = a.views[w.c.b].lo; }
            }
            __syncwarp();
        };
        auto copy_k = [&](int i) { copy(wk, t * RING + i % KS, b_kf(t, i), a.k_mant, &k_map, a.k_exp); };
        auto copy_v = [&](int i) { copy(wv, t * RING + KS + i % VS, b_vf(t, i), a.v_mant, &v_map, a.v_exp); };
        auto copy_q = [&]() {
            if (lane == 0) {
                mbar_expect_tx(b_q(t), G_::Q_BYTES);
                bulk_g2s(base + G_::Q_OFF + t * G_::Q_BYTES, reinterpret_cast<const uint8_t*>(a.qfrag) + ((int64_t)c.b * HR + c.hr) * G_::Q_BYTES, G_::Q_BYTES, b_q(t));
            }
            __syncwarp();
        };
        if (n_mine > 0) {
            copy_k(0);
            copy_q();
            copy_v(0);
            if (KS > 1 && n_mine > 1) copy_k(1);
            if (VS > 1 && n_mine > 1) copy_v(1);
        }
        int run = 0;
        bool first = true, fresh = true, fresh_next = true;             // the tile of the next S, of this O, of the next O begins a run
        for (int i = -1; i < n_mine && !__any_sync(0xffffffffu, dead); ++i) {
            if (i + 1 < n_mine) {            // S of tile i + 1; its packed K rows are used up
                if (first) wait(b_q(t), run);
                wait(b_k(t), i + 1);
                __syncwarp();
                tmem_fence_after();
#pragma unroll
                for (int ks = 0; ks < 8; ++ks)
                    umma_ts(tmt + G_::TM_S + ((i + 1) & 1) * N, tmt + G_::TM_K + ks * 8, qd + (((ks >> 2) * (N * 128) + (ks & 3) * 32) >> 4), id_s, ks > 0);
                umma_commit(b_s(t, i + 1));
                if (i + 1 + KS < n_mine) copy_k(i + 1 + KS);
                fresh_next = first;
                first = ++c.k == c.n;
                if (first) {
                    next_pair(c);
                    ++run;
                }
            }
            if (i >= 0) {                    // O of tile i
                wait(b_v(t), i);
                __syncwarp();
                if (i + VS < n_mine) copy_v(i + VS);
                wait(b_p(t), i);
                __syncwarp();
                tmem_fence_after();
#pragma unroll
                for (int ks = 0; ks < kUTile / 16; ++ks)
                    umma_ss(tmt + G_::TM_O, vd + ks * (2048 >> 4), pd + ks * (16 * SWP >> 4), id_o, ks > 0 || !fresh);
                umma_commit(b_o(t));
            }
            if (first && i + 2 < n_mine) {   // the next S is of another run
                wait(b_s(t, i + 1), (i + 1) >> 1);
                __syncwarp();
                copy_q();
            }
            fresh = fresh_next;
        }
        if (__any_sync(0xffffffffu, dead)) {
            // let what was issued come to its end, and copies in flight land, before the memory goes
            umma_commit(b_o(t));
            for (int x = 0; x < RING + 1; ++x) {
                (void)mbar_wait_bounded(bars + t * TB + 8 * x, 0);
                (void)mbar_wait_bounded(bars + t * TB + 8 * x, 1);
            }
            (void)mbar_wait_bounded(b_o(t), 0);
            (void)mbar_wait_bounded(b_o(t), 1);
        }
    } else {
        // ================================================================ a team: H threads per token
        const int wg = warp >> 2, team = wg / H, half = H == 2 ? wg & 1 : 0, m_pos = tid & 127, w4 = warp & 3, bar_id = 1 + wg;
        const uint32_t tmt = tm + team * G_::TM_TEAM + ((uint32_t)w4 << 21);        // lane field: 32 * quarter << 16
        float *mref = fl + G_::F_MREF + wg * C, *mfac = fl + G_::F_FAC + wg * C,
              *lsum = fl + G_::F_SUM + wg * C, *red = fl + G_::F_RED + wg * 4 * C;
        int* chan = reinterpret_cast<int*>(fl + G_::F_CHAN) + wg * D;
        int* unset = reinterpret_cast<int*>(fl + G_::F_UNSET) + wg;         // rows that have seen nothing yet, as a bit mask
        // places whose exclusive or with 16 times the piece's number is the piece's: packed row, V row (panels of 64 slots), P line
        const uint32_t place = row_place<P>(m_pos), exp_at = N16 ? m_pos * 8 : (m_pos * row_e) & ~3, exp_sel = umma_exp_sel(m_pos, row_e);
        const uint32_t vline = smem_u32(smem) + G_::V_OFF + team * G_::V_BYTES + half * (kUTile * 128) + m_pos * 128 + ((m_pos & 7) << 4);
        const uint32_t pline = smem_u32(smem) + G_::P_OFF + team * G_::P_BYTES + ((m_pos * SWP) ^ ((((m_pos * SWP) >> 7) & (SWP / 16 - 1)) << 4));
        int first_item;
        const int n_mine = range(team, first_item), me = blockIdx.x + team * gridDim.x;
        const int R = a.n_draft * a.group;
        const float up = a.scale * (P == 4 ? 64.f : P == 6 ? 16.f : 4.f), to_log2 = 1.4426950408889634f;      // 2^8 2^-(P-2)
        const float cap_in = a.softcap > 0.f ? up / a.softcap * 2.8853900817779268f : 0.f;
        // row data, drafted positions and view of a run, asynchronously into the buffers of its parity
        auto fetch = [&](const Cursor& c, int par) {
            if (c.b < B) {
                if (m_pos < C)
                    cp_async16(smem_u32(fl + G_::F_RI + ((wg * 2 + par) * C + m_pos) * 4), a.rows + ((int64_t)c.b * HR + c.hr) * N + half * C + m_pos);
                else if (m_pos >= 64 && m_pos < 64 + kAttnMaxDraft / 4)
                    cp_async16(smem_u32(fl + G_::F_DPOS + (wg * 2 + par) * kAttnMaxDraft + (m_pos - 64) * 4), a.dpos + c.b * kAttnMaxDraft + (m_pos - 64) * 4);
                else if (m_pos >= 96 && m_pos < 98)
                    cp_async16(smem_u32(fl + G_::F_VIEW + (wg * 2 + par) * 8 + (m_pos - 96) * 4), reinterpret_cast<const int*>(a.views + c.b) + (m_pos - 96) * 4);
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        // Converts this thread's slots of the packed rows in unit `u` and hands them to `put` (part j: 32 slots, 16
        // registers); returns the row's largest exponent byte.
        auto convert = [&](int u, auto put) {
            const uint32_t at = smem_u32(smem) + u * G_::UNIT + place;
            uint32_t ew[2];
            umma_exps<N16>(smem + G_::E_OFF + u * exp_unit + exp_at, exp_sel, ew);
            uint32_t w[4 / H][P];          // (all loads first: they may not be moved across what follows)
#pragma unroll
            for (int j = 0; j < 4 / H; ++j) load32<P>(at, 2 * half + j, w[j]);
            UW g[(N16 ? 8 : 4) / H];
            const int top = umma_row<P, N16, H>(ew, half, g);
#pragma unroll
            for (int j = 0; j < 4 / H; ++j) {
                uint32_t r[16];
                convert32<P>(w[j], g[N16 ? 2 * j : j], g[N16 ? 2 * j + 1 : j], r);
                put(j, r);
            }
            return top;
        };
        auto convert_k = [&](int i) {
            wait(b_kf(team, i), i / KS);
            __syncwarp();
            const int top = convert(team * RING + i % KS, [&](int j, const uint32_t (&r)[16]) { tmem_st<16>(tmt + G_::TM_K + half * 32 + 16 * j, r); });
            tmem_wait_st();
            tmem_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(b_k(team));
            return top;
        };


        Cursor c = seek(first_item), cn = c;
        fetch(c, 0);
        int it = 0, run = 0, k_next = n_mine > 0 ? convert_k(0) : 0;
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
            if (a.window > 0) clear_lo = max(clear_lo, sv.ctx + a.n_draft - a.window);
            F2 l[C / 2];
#pragma unroll
            for (int j = 0; j < C / 2; ++j) l[j] = f2(0.f, 0.f);
            bool behind = true;           // a row of the group has seen nothing yet
            for (int k = k0; k < k1; ++k, ++it) {
                const uint32_t k_top = (uint32_t)k_next;
                wait(b_s(team, it), it >> 1);                 // S of this tile is there, its K rows are used up
                tmem_fence_after();
                if (it + 1 < n_mine) k_next = convert_k(it + 1);
                if (it > 0) wait(b_o(team), it - 1);          // V and P of the tile before are used up
                wait(b_vf(team, it), it / VS);
                __syncwarp();
                const uint32_t v_top = (uint32_t)convert(team * RING + KS + it % VS, [&](int j, const uint32_t (&r)[16]) {
#pragma unroll
                    for (int x = 0; x < 4; ++x)       // 16-byte pieces 4 j + x, swizzled
                        sts128((vline ^ ((4 * (j & 1) + x) << 4)) + (j >> 1) * (kUTile * 128), r[4 * x], r[4 * x + 1], r[4 * x + 2], r[4 * x + 3]);
                });
                __syncwarp();
                if (lane == 0) mbar_arrive(b_v(team));
                // ---- scores
                const uint32_t tm_s = tmt + G_::TM_S + (it & 1) * N + half * C;
                const int tt = tile_token(sv, k, kUTile);
                float mul = finite_factor(up * to_log2 * __uint_as_float(k_top << 23));
                uint32_t raw[C];
                if (KEEP) {
                    tmem_ld<C>(tm_s, raw);
                    tmem_wait_ld(raw);
                }
                if (a.softcap > 0.f) {
                    const float in = finite_factor(cap_in * __uint_as_float(k_top << 23));
                    mul = a.softcap * to_log2;
                    if (a.softcap > kCapFast) {
                        const float to_x = finite_factor(up * __uint_as_float(k_top << 23)), inv_cap = 1.f / a.softcap;      // (in two steps: their product may be too small)
                        change_scores<C>(tm_s, raw, [&](float y, int) { return tanh_relative(y * to_x * inv_cap); });
                    } else {
                        change_scores<C>(tm_s, raw, [&](float y, int) { return fmaf(-2.f, rcp_approx(1.f + ex2_approx(y * in)), 1.f); });      // tanh x = 1 - 2 / (1 + e^2x): about 2e-7 absolute
                    }
                }
                const bool masked = a.slopes != nullptr || !(tt + kUTile <= sv.ctx && (tt >= clear_lo || tt + kUTile <= sv.pf));
                if (masked) {
                    // bias and masks: log2 units afterwards
                    const int tok = tt + m_pos;
                    const bool in_ctx = tok < sv.ctx;
                    const int jd = in_ctx ? 0 : min(tok - sv.ctx, kAttnMaxDraft - 1);
                    const bool drafted = !in_ctx && tok - sv.ctx < sv.nd;
                    const int kpos = in_ctx || !drafted ? tok : dpos[jd];
                    const bool always = tok < sv.pf, from = tok >= sv.first;
                    change_scores<C>(tm_s, raw, [&](float y, int e) {
                        const RowInfo x = ri[e];
                        const int dist = x.pos - kpos;
                        const bool near = a.window == 0 || dist < a.window;
                        const bool bit = (((jd < 32 ? x.m0 : x.m1) >> (jd & 31)) & 1u) != 0u;
                        const bool see = in_ctx ? (from && near) || always : drafted && bit && near;
                        return see ? y * mul - x.slope * to_log2 * (float)dist : -INFINITY;
                    });
                    mul = 1.f;
                }
                // ---- running softmax against the references, which are raised at most once per tile
                F2 y[C / 2];
                const F2 mul2 = f2(mul, mul);
#pragma unroll 1
                for (int pass = 0;; ++pass) {
                    if (!KEEP) {
                        tmem_ld<C>(tm_s, raw);
                        tmem_wait_ld(raw);
                    }
                    float top = -INFINITY;
#pragma unroll
                    for (int j = 0; j < C; j += 4) {
                        const float4 m = *reinterpret_cast<const float4*>(mref + j);       // (negative references)
                        y[j / 2] = f2_fma(f2(__uint_as_float(raw[j]), __uint_as_float(raw[j + 1])), mul2, f2(m.x, m.y));
                        y[j / 2 + 1] = f2_fma(f2(__uint_as_float(raw[j + 2]), __uint_as_float(raw[j + 3])), mul2, f2(m.z, m.w));
                        float y0, y1;
                        f2_split(y[j / 2], y0, y1);
                        top = max3(top, y0, y1);
                        f2_split(y[j / 2 + 1], y0, y1);
                        top = max3(top, y0, y1);
                    }
                    if (pass != 0 || !named_any(bar_id, 128, top > 8.f || behind)) break;
#pragma unroll (KEEP ? C / 8 : 1)
                    for (int j = 0; j < C; j += 8) {
                        uint32_t r[8];
                        if (!KEEP) {
                            tmem_ld<8>(tm_s + j, r);
                            tmem_wait_ld(r);
                        }
                        float v[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] = fmaf(__uint_as_float(KEEP ? raw[j + e] : r[e]), mul, mref[j + e]);
                        const float mine = across_lanes<8, true>(v, lane);
                        constexpr int GAP = 32 / 8;          // lanes that end up with the same column
                        if (lane % GAP == 0) red[w4 * C + j + lane / GAP] = mine;
                    }
                    named_sync(bar_id, 128);
                    if (m_pos < 32) {
                        bool none = false;
                        if (lane < C) {
                            const float x = fmaxf(fmaxf(red[lane], red[C + lane]), fmaxf(red[2 * C + lane], red[3 * C + lane]));
                            const bool is_unset = (*unset >> lane) & 1;
                            none = is_unset && x == -INFINITY;
                            const float step = none ? 0.f : (is_unset ? x : fmaxf(x, 0.f));
                            mfac[lane] = is_unset ? 1.f : ex2_approx(-step);      // (a row that has seen nothing has sums 0)
                            mref[lane] -= step;
                        }
                        const uint32_t left = __ballot_sync(0xffffffffu, none);
                        if (lane == 0) *unset = (int)left;
                    }
                    named_sync(bar_id, 128);
                    behind = *unset != 0;
#pragma unroll
                    for (int j = 0; j < C; j += 2) l[j / 2] = f2_mul(l[j / 2], *reinterpret_cast<const F2*>(mfac + j));
                    if (k > k0) {          // (the product of the tile before is done: waited for above)
                        tmem_fence_after();
#pragma unroll 1
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
                const float vf = __uint_as_float((uint32_t)max((int)v_top - 9, 0) << 23);
                const F2 vf2 = f2(vf, vf);
#pragma unroll
                for (int j = 0; j < C; j += 8) {
                    uint32_t w[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float y0, y1;
                        f2_split(y[j / 2 + e], y0, y1);
                        const F2 p = f2(ex2_approx(y0), ex2_approx(y1));
                        l[j / 2 + e] = f2_add(l[j / 2 + e], p);
                        float p0, p1;
                        f2_split(f2_mul(p, vf2), p0, p1);
                        w[e] = pack_bf16x2_rn(p0, p1);
                    }
                    sts128(pline ^ ((half * C + j) * 2), w[0], w[1], w[2], w[3]);
                }
                fence_async_shared();
                tmem_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(b_p(team));
            }
            // ---- the run's result: this thread holds slot umma_slot(m_pos) of C rows
            {
                float v[C];
#pragma unroll
                for (int j = 0; j < C / 2; ++j) f2_split(l[j], v[2 * j], v[2 * j + 1]);
                const float mine = across_lanes<C, false>(v, lane);
                constexpr int GAP = 32 / C;                   // lanes that end up with the same column
                if (lane % GAP == 0) red[w4 * C + lane / GAP] = mine;
            }
            named_sync(bar_id, 128);
            const bool whole = k0 == 0 && k1 == c.n;
            const int slot_of = umma_slot<P>(m_pos);
            float* part = a.partials + ((int64_t)(2 * me + (k0 == 0 ? 1 : 0)) * a.part_rows + half * C) * kAttnPart;
            if (m_pos < C) {
                const int row = row0 + m_pos;
                const float ls = red[m_pos] + red[C + m_pos] + red[2 * C + m_pos] + red[3 * C + m_pos];
                const float m = ((*unset >> m_pos) & 1) ? -3.4028235e38f : -mref[m_pos];
                lsum[m_pos] = ls;
                if (row < R && !whole) {
                    part[m_pos * kAttnPart + D] = m;
                    part[m_pos * kAttnPart + D + 1] = ls;
                }
            }
            // (read before the barrier: a warp that is through with its results writes the next head's table.  Cut to a channel: of
            // an inv_perm_v that is no permutation some entries are never written.)
            const int ch = a.inv_perm_v ? chan[slot_of] & (D - 1) : slot_of;
            wait(b_o(team), it - 1);
            __syncwarp();
            tmem_fence_after();
            named_sync(bar_id, 128);
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
                        const bool live = i < sv.nd && ls != 0.f;
                        static_cast<__nv_bfloat16*>(a.out)[(((int64_t)b * a.n_draft + i) * a.n_q_heads + hq) * D + ch] =
                            __float2bfloat16_rn(live ? __uint_as_float(o[e]) * (a.out_up / ls) : 0.f);
                    } else {
                        part[(j + e) * kAttnPart + slot_of] = __uint_as_float(o[e]);
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
