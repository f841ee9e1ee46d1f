// Attention of whole prompts and longer chunks over the packed cache on the fifth-generation tensor cores: bf16 query rows in
// items of 256 per kv head.
//
//   S[rows x tokens] = pi(Q) . K^T            pi(Q), K: shared memory
//   P = 2^(mul S - m), masked                 from tensor memory through registers back to tensor memory
//   O[rows x slots] += P . V                  P: tensor memory, V: shared memory (tokens the slow index)
//
// One persistent block per SM, a worker; tiles of 128 tokens.  A tile's packed rows are converted to bf16 once for 256 query
// rows, by four warps that read them straight from the cache (a thread per token, the next tile's row already in registers,
// so that pages need nothing but an address per thread).  The rows are two halves of 128, a warp group and an S and an O of their
// own each: while one half's exponentials run, the tensor cores work for the other.  A thread owns a query row: its maximum, sum and
// rescaling stay in the thread.  P takes the columns of the S it came from (two bf16 numbers a column), so that two S and two O fill
// the 512 columns.  One warp issues all matrix instructions; they run in its order, which is what lets S of the next tile
// overwrite P of this one without a wait.
//
//   warps 0..7   rows: S -> P, rescaling, pi(Q) into shared memory, results     (halves 0 and 1)
//   warps 8..11  packed rows -> K, V in shared memory, two stages
//   warp 12      matrix instructions
//
// The reference maximum only moves when a score passes it by 8 (a factor 2^8 that fp32 sums and bf16 weights take without
// harm); then O is rescaled in tensor memory, which waits for the products under way and is rare after a row's first tiles.
// Tiles on the border of what rows see are masked in a pass of their own over S in tensor memory.
#pragma once
#include "attn_rows.cuh"
#include "ragged.cuh"
#include "umma.cuh"

namespace kvbfp {
namespace {

constexpr int kPRows = 256, kPTile = 128, kPThreads = 13 * 32;
constexpr int kPQ = 0, kPK = 65536, kPV = 131072, kPEnd = 196608;      // shared memory: Q (two halves), K, V (two stages each)
constexpr int kPPanel = kPTile * 128;                                  // 64 positions of 128 rows
constexpr int kPSmem = kPEnd + 256;

// Slot at position m of a converted row: the order the fields unpack in.
template <int P>
__device__ __forceinline__ int prompt_slot(int m) {
    if (P != 8) return (m & ~7) | ((m & 1) << 2) | ((m >> 1) & 3);
    return (m & ~3) | ((m & 1) << 1) | ((m >> 1) & 1);
}
// Position of slot s within its group of eight.
template <int P>
__device__ __forceinline__ constexpr int prompt_pos(int s) {
    return P != 8 ? 2 * (s & 3) + (s >> 2) : (s & 4) | ((s & 1) << 1) | ((s >> 1) & 1);
}
// Byte place of 16-byte piece p (8 positions) of row r.
__device__ __forceinline__ uint32_t prompt_place(int r, int p) { return (p >> 3) * kPPanel + r * 128 + (((p & 7) ^ (r & 7)) << 4); }

// 32 slots of a packed row to 16 bf16 pairs in position order.
template <int P>
__device__ __forceinline__ void prompt_convert(const uint32_t (&w)[P], const AW& g0, const AW& g1, uint32_t (&r)[16]) {
    if (P == 4) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const AW& g = j < 2 ? g0 : g1;
            r[4 * j] = acvt<4>(w[j], g);
            r[4 * j + 1] = acvt<4>(w[j] >> 4, g);
            r[4 * j + 2] = acvt<4>(w[j] >> 8, g);
            r[4 * j + 3] = acvt<4>(w[j] >> 12, g);
        }
    } else if (P == 8) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const AW& g = j < 4 ? g0 : g1;
            r[2 * j] = acvt<8>(w[j], g);
            r[2 * j + 1] = acvt<8>(w[j] >> 8, g);
        }
    } else {
        // eight slots are two runs of three bytes; a 16-bit half holds bytes 0, 1 (then 1, 2) of the first run, the other half
        // those of the second: slots 0 | 4, 1 | 5 and 2 | 6, 3 | 7
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int b = 6 * j, word = b >> 2;                      // first byte of the eight slots: 0, 6, 12, 18
            const bool odd = (b & 3) != 0;
            const uint32_t lo = prmt(w[word], w[(word + 1) % P], odd ? 0x6532u : 0x4310u), hi = prmt(w[word], w[(word + 1) % P], odd ? 0x7643u : 0x5421u);
            const AW& g = j < 2 ? g0 : g1;
            r[4 * j] = acvt<6>(lo, g);
            r[4 * j + 1] = acvt<6>(lo >> 6, g);
            r[4 * j + 2] = acvt<6>(hi >> 4, g);
            r[4 * j + 3] = acvt<6>(hi >> 10, g);
        }
    }
}

__device__ __noinline__ bool prompt_wait_slow(uint32_t bar, uint32_t parity) { return mbar_wait_bounded(bar, parity); }

template <int P, bool N16>
__global__ void __launch_bounds__(kPThreads, 1) ragged_umma(const RaggedArgs a) {
    constexpr int D = kHeadDim, ROW_M = D * P / 8;
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ int s_scan[kPThreads / 32];
    __shared__ uint32_t s_tmem;
    int (&s_items)[kMaxPagedBatch + 1] = *reinterpret_cast<int (*)[kMaxPagedBatch + 1]>(smem);      // (until rows come here)
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t base = smem_u32(smem), bars = base + kPEnd;
    auto b_kf = [&](int s) { return bars + 8 * s; };            // K of a stage converted
    auto b_ke = [&](int s) { return bars + 16 + 8 * s; };       //   and used
    auto b_vf = [&](int s) { return bars + 32 + 8 * s; };
    auto b_ve = [&](int s) { return bars + 48 + 8 * s; };
    auto b_s = [&](int h) { return bars + 64 + 8 * h; };        // S of a half done
    auto b_p = [&](int h) { return bars + 80 + 8 * h; };        // P written
    auto b_o = [&](int h) { return bars + 96 + 8 * h; };        // O done
    auto b_q = [&](int h) { return bars + 112 + 8 * h; };       // pi(Q) of a run there
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(b_kf(i), 4); mbar_init(b_ke(i), 1); mbar_init(b_vf(i), 4); mbar_init(b_ve(i), 1);
            mbar_init(b_s(i), 1); mbar_init(b_p(i), 4); mbar_init(b_o(i), 1); mbar_init(b_q(i), 4);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async_shared();
    }
    if (warp == 12) tmem_alloc(smem_u32(&s_tmem), 512);
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const uint32_t tm = __shfl_sync(0xffffffffu, s_tmem, 0);
    pdl_wait();
    ragged_count<kPThreads>(a, s_items, s_scan, kPRows, kPTile);
    const int H = a.fmt.n_kv_heads, n_items = s_items[a.batch], me = blockIdx.x;
    const int workers = min(a.workers, n_items);
    const int i0 = me < workers ? worker_start(me, n_items, workers) : 0;
    const int n_mine = me < workers ? worker_start(me + 1, n_items, workers) - i0 : 0;
    const int b_first = ragged_find(a, s_items, i0), at_first = i0 - s_items[b_first];
    __syncthreads();
    RaggedCursor c;
    if (n_mine > 0) ragged_seek(a, c, b_first, at_first, kPRows, kPTile);
    auto next_tile = [&]() {           // true: the next tile begins another run
        if (++c.k < c.v.n) return false;
        ragged_next(a, c, kPRows, kPTile);
        return true;
    };
    auto two = [&]() { return c.s.n * a.group > c.rt * kPRows + 128; };       // does the entry have rows in half 1
    bool dead = false;                 // a wait ran out: no more waits, the flag is up, results are void
    auto wait = [&](uint32_t bar, int phase) {
        if (!mbar_try(bar, (uint32_t)phase & 1u) && !dead && !prompt_wait_slow(bar, (uint32_t)phase & 1u)) {
            dead = true;
            raise_flag(a.status, KVBFP_FLAG_WAIT_TIMEOUT);
        }
    };

    if (warp == 12) {
        // ================================================================ matrix instructions
        constexpr uint32_t id_s = umma_idesc(128, 128, false, false), id_o = umma_idesc(128, 128, false, true);
        const uint64_t qd = umma_desc<128>(base + kPQ, 16, 1024), kd = umma_desc<128>(base + kPK, 16, 1024);
        const uint64_t vd = umma_desc<128>(base + kPV, kPPanel, 1024);
        int n_run[2] = {0, 0}, n_tile[2] = {0, 0};        // runs and tiles of each half so far
        auto qk = [&](int i, int h, bool first, bool last_half) {
            if (first) wait(b_q(h), n_run[h]++);
            if (h == 0) wait(b_kf(i & 1), i >> 1);
            __syncwarp();
            tmem_fence_after();
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) {
                const uint32_t step = ((ks >> 2) * kPPanel + (ks & 3) * 32) >> 4;
                umma_ss(tm + 128 * h, qd + ((h * 32768) >> 4) + step, kd + (((i & 1) * 32768) >> 4) + step, id_s, ks > 0);
            }
            umma_commit(b_s(h));
            if (last_half) umma_commit(b_ke(i & 1));
        };
        auto pv = [&](int i, int h, bool first, bool last_half) {
            if (h == 0) wait(b_vf(i & 1), i >> 1);
            wait(b_p(h), n_tile[h]++);
            __syncwarp();
            tmem_fence_after();
#pragma unroll
            for (int ks = 0; ks < 8; ++ks)
                umma_ts(tm + 256 + 128 * h, tm + 128 * h + ks * 8, vd + (((i & 1) * 32768 + ks * 2048) >> 4), id_o, ks > 0 || !first);
            umma_commit(b_o(h));
            if (last_half) umma_commit(b_ve(i & 1));
        };
        bool first = true, both = n_mine > 0 && two();
        if (n_mine > 0) {
            qk(0, 0, true, !both);
            if (both) qk(0, 1, true, true);
        }
        for (int i = 0; i < n_mine && !__any_sync(0xffffffffu, dead); ++i) {
            const bool more = i + 1 < n_mine, first_next = more && next_tile(), both_next = more && two();
            pv(i, 0, first, !both);
            if (more) qk(i + 1, 0, first_next, !both_next);
            if (both) pv(i, 1, first, true);
            if (both_next) qk(i + 1, 1, first_next, true);
            first = first_next;
            both = both_next;
        }
        if (__any_sync(0xffffffffu, dead)) {
            // let what was issued come to its end before the memory goes
            umma_commit(b_o(0));
            (void)mbar_wait_bounded(b_o(0), 0);
            (void)mbar_wait_bounded(b_o(0), 1);
        }
    } else if (warp >= 8) {
        // ================================================================ packed rows to bf16
        const int r = tid & 127, row_e = D / a.fmt.block;
        const uint32_t sel = row_e == 4 ? 0x3210u : row_e == 2 ? 0x1100u : 0x0000u;
        uint32_t kw[4][P], vw[4][P], ke[2] = {0, 0}, ve[2] = {0, 0};
        int page = -1;                // of this thread's token of the next tile to load, -1: not seen by any row
        auto look_up = [&]() {
            page = -1;
            const int tok = ragged_token(c.v, c.k, kPTile) + r;
            if (tok <= c.v.p1 && (a.window == 0 || tok > c.v.p0 - a.window || tok < a.n_sink)) {
                page = token_page(a.map, c.b, tok);
                if (page < 0) raise_flag(a.status, KVBFP_FLAG_POSITION);
            }
        };
        int64_t row = -1;             // the token's row in the planes, of the tile to load
        auto to_row = [&]() {
            const int tok = ragged_token(c.v, c.k, kPTile) + r;
            row = page >= 0 ? ((int64_t)page * H + c.hk) * a.fmt.max_seq + token_row(a.map, tok) : -1;
        };
        auto load = [&](const uint8_t* mant, const uint8_t* exps, uint32_t (&w)[4][P], uint32_t (&e)[2]) {
            if (row < 0) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int x = 0; x < P; ++x) w[j][x] = 0u;
                e[0] = e[1] = 0u;
                return;
            }
            const uint4* p = reinterpret_cast<const uint4*>(mant + row * ROW_M);
#pragma unroll
            for (int x = 0; x < P; ++x) {
                const uint4 y = p[x];
                w[(4 * x) / P][(4 * x) % P] = y.x;
                w[(4 * x + 1) / P][(4 * x + 1) % P] = y.y;
                w[(4 * x + 2) / P][(4 * x + 2) % P] = y.z;
                w[(4 * x + 3) / P][(4 * x + 3) % P] = y.w;
            }
            const uint8_t* q = exps + row * row_e;
            if (N16) {
                const uint2 y = *reinterpret_cast<const uint2*>(q);
                e[0] = y.x;
                e[1] = y.y;
            } else {
                e[0] = row_e == 4 ? *reinterpret_cast<const uint32_t*>(q) : row_e == 2 ? *reinterpret_cast<const uint16_t*>(q) : *q;
            }
        };
        auto convert = [&](uint32_t to, const uint32_t (&w)[4][P], const uint32_t (&e)[2]) {
            const uint32_t eb = N16 ? 0u : prmt(e[0], 0u, sel);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                AW g0, g1;
                if (N16) {
                    g0 = aw_make<P>(prmt(e[j >> 1], 0u, 0x4040u + 0x0101u * (2 * (j & 1))));
                    g1 = aw_make<P>(prmt(e[j >> 1], 0u, 0x4040u + 0x0101u * (2 * (j & 1) + 1)));
                } else {
                    g0 = g1 = aw_make<P>(prmt(eb, 0u, 0x4040u + 0x0101u * j));
                }
                uint32_t x[16];
                prompt_convert<P>(w[j], g0, g1, x);
#pragma unroll
                for (int y = 0; y < 4; ++y) sts128(to + prompt_place(r, 4 * j + y), x[4 * y], x[4 * y + 1], x[4 * y + 2], x[4 * y + 3]);
            }
            fence_async_shared();
            __syncwarp();
        };
        int ahead = 0;                // tiles whose row is known
        auto step = [&]() {           // to the next tile's row; its successor's page is asked for
            to_row();
            if (++ahead < n_mine) {
                (void)next_tile();
                look_up();
            }
        };
        if (n_mine > 0) {
            look_up();
            step();
            load(a.k_mant, a.k_exp, kw, ke);
            load(a.v_mant, a.v_exp, vw, ve);
        }
        for (int i = 0; i < n_mine; ++i) {
            const int st = i & 1;
            const bool more = i + 1 < n_mine;
            if (i >= 2) wait(b_ke(st), (i >> 1) - 1);
            convert(base + kPK + st * 32768, kw, ke);
            if (lane == 0) mbar_arrive(b_kf(st));
            if (more) {
                step();
                load(a.k_mant, a.k_exp, kw, ke);
            }
            if (i >= 2) wait(b_ve(st), (i >> 1) - 1);
            convert(base + kPV + st * 32768, vw, ve);
            if (lane == 0) mbar_arrive(b_vf(st));
            if (more) load(a.v_mant, a.v_exp, vw, ve);
        }
    } else {
        // ================================================================ rows
        const int h = warp >> 2, w4 = warp & 3, r = tid & 127;                   // half, quarter of its rows, row
        const uint32_t tms = tm + 128 * h + ((uint32_t)w4 << 21), tmo = tms + 256;      // lane field: 32 * quarter << 16
        const uint32_t q_at = base + kPQ + h * 32768;
        const float mul = finite_factor(a.scale * kValueUp * 1.4426950408889634f);      // scores to log2 units
        int4 rec = make_int4(-1, 0, 0, 0);
        // pi(Q) of the entry at the cursor, this warp's 32 rows: a lane has four positions
        auto write_q = [&]() {
            const int row0 = c.rt * kPRows + h * 128 + w4 * 32, R = c.s.n * a.group;
            int ch[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int slot = prompt_slot<P>(4 * lane + x);
                ch[x] = a.perm_k ? a.perm_k[c.hk * D + slot] & (D - 1) : slot;
            }
            const unsigned short* q = static_cast<const unsigned short*>(a.q);
#pragma unroll 1
            for (int x0 = 0; x0 < 32; x0 += 8) {
                uint32_t v[8][4];
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    const int row = row0 + x0 + x, i = row / a.group;
                    const unsigned short* p = q + ((int64_t)(c.s.start + i) * a.n_q_heads + c.hk * a.group + row - i * a.group) * D;
#pragma unroll
                    for (int y = 0; y < 4; ++y) v[x][y] = row < R ? p[ch[y]] : 0u;
                }
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    const uint32_t at = q_at + prompt_place(w4 * 32 + x0 + x, lane >> 1) + (lane & 1) * 8;
                    asm volatile("st.shared.v2.u32 [%0], {%1,%2};" ::"r"(at), "r"(v[x][0] | v[x][1] << 16), "r"(v[x][2] | v[x][3] << 16) : "memory");
                }
            }
            fence_async_shared();
            __syncwarp();
            if (lane == 0) mbar_arrive(b_q(h));
        };
        int n_tile = 0;               // tiles of this half so far
        if (n_mine > 0 && (h == 0 || two())) write_q();
        for (int it = 0; it < n_mine;) {
            // ---- a run: tiles [k0, k1) of one entry
            const int k0 = c.k, k1 = min(c.v.n, k0 + n_mine - it), n_tiles = c.v.n;
            const bool here = h == 0 || two();
            const int R = c.s.n * a.group, row = c.rt * kPRows + h * 128 + r;
            const int pos = c.s.base + min(row, R - 1) / a.group;
            const int pos_lo = c.s.base + min(row - r, R - 1) / a.group, pos_hi = c.s.base + min(row - r + 127, R - 1) / a.group;
            const int see_lo = a.window > 0 ? pos - a.window + 1 : 0;
            float m = -3.4028235e38f;
            F2 l2 = f2(0.f, 0.f);
            if (here) {
                for (int k = k0; k < k1; ++k, ++n_tile) {
                    const int tt = ragged_token(c.v, k, kPTile);
                    wait(b_s(h), n_tile);
                    __syncwarp();
                    tmem_fence_after();
                    const bool clear = tt + 127 <= pos_lo && (a.window == 0 || tt > pos_hi - a.window || tt + 128 <= a.n_sink);
                    if (!clear) {
#pragma unroll 1
                        for (int j = 0; j < 4; ++j) {
                            uint32_t s[32];
                            tmem_ld<32>(tms + 32 * j, s);
                            const int t0 = tt + 32 * j;
                            // bits of the tokens seen: up to pos, from see_lo on or among the first ones
                            auto below = [](int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; };
                            const uint32_t see = below(pos - t0 + 1) & (~below(see_lo - t0) | below(a.n_sink - t0));
                            tmem_wait_ld(s);
#pragma unroll
                            for (int e = 0; e < 32; ++e) s[e] = (see >> e) & 1u ? s[e] : 0xff800000u;
                            tmem_st<32>(tms + 32 * j, s);
                        }
                        tmem_wait_st();
                    }
                    float top = -INFINITY;
                    {
                        uint32_t s[2][32];
                        tmem_ld<32>(tms, s[0]);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            tmem_wait_ld(s[j & 1]);
                            if (j < 3) tmem_ld<32>(tms + 32 * (j + 1), s[(j + 1) & 1]);
                            float t0 = __uint_as_float(s[j & 1][0]), t1 = __uint_as_float(s[j & 1][1]);
#pragma unroll
                            for (int e = 2; e < 32; e += 4) {
                                t0 = max3(t0, __uint_as_float(s[j & 1][e]), __uint_as_float(s[j & 1][e + 1]));
                                if (e + 3 < 32) t1 = max3(t1, __uint_as_float(s[j & 1][e + 2]), __uint_as_float(s[j & 1][e + 3]));
                            }
                            top = max3(top, t0, t1);
                        }
                    }
                    top *= mul;
                    const bool grow = top > m + 8.f;
                    if (__any_sync(0xffffffffu, grow)) {
                        const float x = fmaxf(m, top), al = ex2_approx(m - x);
                        m = x;
                        l2 = f2_mul(l2, f2(al, al));
                        if (k > k0) {
                            wait(b_o(h), n_tile - 1);
                            __syncwarp();
                            tmem_fence_after();
#pragma unroll 1
                            for (int j = 0; j < 4; ++j) {
                                uint32_t o[32];
                                tmem_ld<32>(tmo + 32 * j, o);
                                tmem_wait_ld(o);
#pragma unroll
                                for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * al);
                                tmem_st<32>(tmo + 32 * j, o);
                            }
                            tmem_wait_st();
                        }
                    }
                    const F2 mul2 = f2(mul, mul), neg2 = f2(-m, -m);
                    uint32_t s[2][32];
                    tmem_ld<32>(tms, s[0]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        tmem_wait_ld(s[j & 1]);
                        if (j < 3) tmem_ld<32>(tms + 32 * (j + 1), s[(j + 1) & 1]);
                        uint32_t p[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            float x0, x1;
                            f2_split(f2_fma(f2(__uint_as_float(s[j & 1][2 * e]), __uint_as_float(s[j & 1][2 * e + 1])), mul2, neg2), x0, x1);
                            x0 = ex2_approx(x0);
                            x1 = ex2_approx(x1);
                            l2 = f2_add(l2, f2(x0, x1));
                            p[e] = pack_bf16x2_rn(x0, x1);
                        }
                        tmem_st<16>(tms + 16 * j, p);
                    }
                    tmem_wait_st();
                    tmem_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(b_p(h));
                }
            }
            it += k1 - k0;
            // ---- the run's result; pi(Q) of the next run first where it need not wait for it
            const bool whole = k0 == 0 && k1 == n_tiles;
            if (k0 > 0 && k1 == n_tiles) rec = make_int4(c.b, c.rt, c.hk, worker_of(i0 + it - n_tiles, n_items, workers));
            const int i = row / a.group, hk = c.hk;
            const bool wanted = here && row < R && (!whole || pos >= 0);
            const int64_t out_row = (int64_t)(c.s.start + i) * a.n_q_heads + hk * a.group + row - i * a.group;
            float* part = a.partials + ((int64_t)(2 * me + (k0 == 0 ? 1 : 0)) * a.part_rows + h * 128 + r) * kAttnPart;
            c.k = k1 - 1;
            if (it < n_mine) (void)next_tile();
            const bool next_here = it < n_mine && (h == 0 || two());
            const bool staged = whole && a.inv_perm_v != nullptr;
            if (next_here && !staged) write_q();
            if (here) {
                float la, lb;
                f2_split(l2, la, lb);
                const float l = la + lb, inv = l != 0.f ? kValueUp / l : 0.f;
                wait(b_o(h), n_tile - 1);
                __syncwarp();
                tmem_fence_after();
#pragma unroll 1
                for (int j = 0; j < 4; ++j) {
                    uint32_t o[32];
                    tmem_ld<32>(tmo + 32 * j, o);
                    tmem_wait_ld(o);
#pragma unroll
                    for (int x = 0; x < 4; ++x) {         // eight slots
                        float v[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(o[8 * x + prompt_pos<P>(e)]);
                        if (!whole) {
                            if (wanted) {
                                float4* to = reinterpret_cast<float4*>(part + 32 * j + 8 * x);
                                to[0] = make_float4(v[0], v[1], v[2], v[3]);
                                to[1] = make_float4(v[4], v[5], v[6], v[7]);
                            }
                            continue;
                        }
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] = l != 0.f ? v[e] * inv : 0.f;
                        const uint32_t y0 = pack_bf16x2_rn(v[0], v[1]), y1 = pack_bf16x2_rn(v[2], v[3]), y2 = pack_bf16x2_rn(v[4], v[5]), y3 = pack_bf16x2_rn(v[6], v[7]);
                        if (staged) sts128(q_at + prompt_place(r, 4 * j + x), y0, y1, y2, y3);
                        else if (wanted) reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.out) + out_row * D)[4 * j + x] = make_uint4(y0, y1, y2, y3);
                    }
                }
                tmem_fence_before();
                if (!whole && wanted) {
                    part[D] = m;
                    part[D + 1] = l;
                }
                if (staged) {         // channels in their own order: a row at a time, four channels a lane
                    __syncwarp();
                    int sl[4];
#pragma unroll
                    for (int x = 0; x < 4; ++x) sl[x] = a.inv_perm_v[hk * D + 4 * lane + x] & (D - 1);
#pragma unroll 1
                    for (int x = 0; x < 32; ++x) {
                        const int64_t to = __shfl_sync(0xffffffffu, out_row, x);
                        uint32_t v[4];
#pragma unroll
                        for (int y = 0; y < 4; ++y)
                            asm volatile("ld.shared.u16 %0, [%1];" : "=r"(v[y]) : "r"(q_at + prompt_place(w4 * 32 + x, sl[y] >> 3) + (sl[y] & 7) * 2) : "memory");
                        if (__shfl_sync(0xffffffffu, (int)wanted, x))
                            *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.out) + to * D + 4 * lane) = make_uint2(v[0] | v[1] << 16, v[2] | v[3] << 16);
                    }
                    __syncwarp();
                }
            }
            if (next_here && staged) write_q();
        }
        if (tid == 0) a.rec[me] = rec;
    }
    __syncwarp();
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    if (warp == 12) tmem_dealloc(tm, 512);
    pdl_trigger();
}

template <int P, bool N16>
kvbfp_status launch_prompt(const RaggedArgs& a, int grid, cudaStream_t s) {
    auto kernel = ragged_umma<P, N16>;
    static std::atomic<bool> attr_set[64];      // per device; setting the attribute twice is harmless
    int dev = 0;
    KVBFP_CUDA(cudaGetDevice(&dev));
    if (dev < 0 || dev >= 64) return KVBFP_ERR_UNSUPPORTED;
    if (!attr_set[dev].load(std::memory_order_acquire)) {
        KVBFP_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kPSmem));
        attr_set[dev].store(true, std::memory_order_release);
    }
    KVBFP_CUDA(launch_pdl(kernel, dim3(grid), dim3(kPThreads), kPSmem, s, a));
    KVBFP_LAUNCH_CHECK("ragged_umma");
    return KVBFP_OK;
}

}  // namespace
}  // namespace kvbfp
