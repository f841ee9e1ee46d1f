// Attention of whole prompts and longer chunks over the packed cache on the fifth-generation tensor cores: bf16 query rows in
// items of 256 per kv head.
//
//   S[rows x tokens] = pi(Q) . K^T            pi(Q), K: shared memory
//   P = 2^(mul S - m), masked                 from tensor memory through registers back to tensor memory
//   O[rows x slots] += P . V                  P: tensor memory, V: shared memory (tokens the slow index)
//
// One persistent block per SM, a worker; tiles of 128 tokens.  A tile's packed rows are converted to bf16 once for 256 query
// rows, by eight warps that read them straight from the cache, the next tile's already in registers, so that pages need nothing
// but an address per row.  The rows are two halves of 128, a warp group, an S and an O of
// their own each: while one half's exponentials run, the tensor cores work for the other.  A thread owns a query row: maximum,
// sum and rescaling stay in the thread.  P takes the columns of the S it came from (two bf16 numbers a column), so that two S
// and two O fill the 512 columns.  One warp issues all matrix instructions, PV of a tile and S of the next one after the other
// for each half; they run in its order, which is what lets the next S overwrite P without a wait, and tells the rows that O is
// at rest.  (Every completion that it reports costs it some 250 cycles, so it reports S, the use of K and V, and O at the end of
// a run only.  S in pieces of 64 tokens, so that a half need not wait for the tensor cores: a product with N = 64 takes them as
// long as one with N = 128.  P handed over in two pieces: the second report costs more than the earlier start gives.)
//
//   warp 0        matrix instructions
//   warp 1        where the tiles lie (2, 3: only there to give up their registers)
//   warps 4..11   rows: S -> P, rescaling, pi(Q) into shared memory, results     (halves 0 and 1)
//   warps 12..19  packed rows -> K (12..15), V in shared memory, two stages
//
// There is no pass for the maximum: P is formed under the row's reference, and where the sum of 32 weights passes 2^16 they are
// done again under a new one, their scores' maximum, after O was rescaled in tensor memory.  That happens with a row's first
// tokens and hardly ever after.  (With the maximum taken on the side of every score: a prompt of 8192 tokens 690 us, 660 so.)
//
// P is rounded to one bf16 term (2^-8 relative at most, at random; the output is rounded to bf16 too).  With a second term for what the
// rounding leaves (P as many columns as S, 16 products a half for O instead of eight) a prompt of 8192 took 1126 us, chunks 1240.
//
// What bounds it: two chains of about the same length.  The matrix instructions of a tile, one half's after the other's: 16 take 1400
// to 1700 cycles from the first issue to the last (64 each at the pipe's rate; both operands of S come from shared memory, which
// conversion and results use too), and waits and reports some 400 more.  And a half by itself: P some 2200, its products, 250 for
// each to learn of the other.  A tile takes some 4400; the tensor pipe is half busy.  Two warps a row (16 warps, 64 tokens each)
// took 4 to 7 % off 8-bit chunks only, and added 20 % to a prompt, whose entries begin and end more often; unrolling the issuing
// loop over halves and stages added 15 to 25 %; waiting for the next step's rows between the halves and not after them took 2 to
// 4 % off.  A prompt of 8192 tokens, 32 heads, 4 bits: 644 us, 854 TFLOP/s of the visible products; four chunks of 2048 under a
// window of 4096, 8 bits: 752 us.
#pragma once
#include "attn_rows.cuh"
#include "ragged.cuh"
#include "umma.cuh"

namespace kvbfp {
namespace {

constexpr int kPRows = 256, kPTile = 128, kPThreads = 20 * 32;
// shared memory: Q (two halves), K, V (two stages each), 32 lines of 128 bytes for each warp's results, barriers
constexpr int kPQ = 0, kPK = 65536, kPV = 131072, kPOut = 196608, kPBars = kPOut + 8 * 4096, kPSmem = kPBars + 256;
// So large may the sum of 32 weights become before the reference follows: P, its sums and O are floating-point numbers, which
// lose nothing by a common factor, and have room for it.
constexpr float kPLimit = 65536.f;
constexpr int kPPanel = kPTile * 128;                                  // 64 positions of 128 rows

// Registers a thread after the split, of the 96 that the launch gives each: rows, packed rows, the rest (2 x 136 + 2 x 80 + 48 =
// 5 x 96).
constexpr int kPRegsRows = 136, kPRegsConv = 80, kPRegsRest = 48;
template <int N> __device__ __forceinline__ void regs_more() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void regs_less() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

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

// Cached values are carried times 2^-16 here.  Fields become bf16 numbers by one fma (convert32) while the block's weight times
// 2^133 is one, up to exponent bytes of kPFast (values below 2^11 to 2^16); rows with larger ones are rare and take the longer way, over an
// exponent or-ed in.
constexpr int kPDown = 16;
template <int P>
constexpr int kPFast = 135 + P;
// Weights of a block, its exponent byte `e2` in both halves: multipliers 2^(e - 127 - (P - 2) - 16 + 133), the same for fields
// further up, -2^(P-1) times the weight.  Blocks below 2^-110 turn into zeros.
template <int P>
__device__ __forceinline__ UW prompt_weights(uint32_t e2) {
    uint32_t e;
    asm("max.s16x2 %0, %1, %2;" : "=r"(e) : "r"(e2), "r"(15u * 0x00010001u));
    UW w;
    w.s = e * 0x80u + (119u - P) * 0x00800080u;
    w.s2 = w.s - (P == 4 ? 4u : 2u) * 0x00800080u;
    w.c = e * 0x80u - 15u * 0x00800080u + 0x80008000u;
    return w;
}
template <int P>
__device__ __forceinline__ AW prompt_weights_large(uint32_t e2) {
    AW w;
    asm("max.s16x2 %0, %1, %2;" : "=r"(w.s) : "r"(e2), "r"((P - 2 + kPDown) * 0x00010001u));
    w.s = w.s * 0x80u - (P - 2 + kPDown) * 0x00800080u;
    w.c = mul_bf16x2(w.s, AFmt<P>::bias);
    w.s16 = (P == 8) ? mul_bf16x2(w.s, 0x41804180u) : 0u;
    return w;
}
// 32 slots of a packed row to 16 bf16 pairs in position order, for any exponent byte.
template <int P>
__device__ __forceinline__ void prompt_convert_large(const uint32_t (&w)[P], const AW& g0, const AW& g1, uint32_t (&r)[16]) {
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

// Matrix instructions whose descriptors differ in their lower words only (all operands here: groups of eight lines 1024 bytes
// apart, 128-byte swizzle), which is what their registers hold.
constexpr uint32_t kPDescUpper = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t prompt_desc(uint32_t smem_addr, uint32_t lbo) { return ((smem_addr >> 4) & 0x3fffu) | ((lbo >> 4) & 0x3fffu) << 16; }
// Eight steps of 16 positions (two panels) of S; eight steps of 16 tokens of O.  The whole warp calls, one thread issues.
__device__ __forceinline__ void prompt_s(uint32_t d, uint32_t q, uint32_t k, uint32_t idesc) {
    asm volatile("{\n\t.reg .pred e;\n\t.reg .b64 x, y;\n\telect.sync _|e, 0xffffffff;\n\tmov.b64 x, {%1, %4};\n\tmov.b64 y, {%2, %4};\n\t"
                 "@e tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, 0;\n\t"
                 "add.s64 x, x, 2;\n\tadd.s64 y, y, 2;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, 1;\n\t"
                 "add.s64 x, x, 2;\n\tadd.s64 y, y, 2;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, 1;\n\t"
                 "add.s64 x, x, 2;\n\tadd.s64 y, y, 2;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, 1;\n\t"
                 "add.s64 x, x, %5;\n\tadd.s64 y, y, %5;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, 1;\n\t"
                 "add.s64 x, x, 2;\n\tadd.s64 y, y, 2;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, 1;\n\t"
                 "add.s64 x, x, 2;\n\tadd.s64 y, y, 2;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, 1;\n\t"
                 "add.s64 x, x, 2;\n\tadd.s64 y, y, 2;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, 1;\n\t}"
                 ::"r"(d), "r"(q), "r"(k), "r"(idesc), "n"(kPDescUpper), "n"((kPPanel >> 4) - 6) : "memory");
}
__device__ __forceinline__ void prompt_o(uint32_t d, uint32_t p, uint32_t v, uint32_t idesc, bool add) {
    asm volatile("{\n\t.reg .pred p, e;\n\t.reg .b64 y;\n\t.reg .b32 x;\n\telect.sync _|e, 0xffffffff;\n\tmov.b64 y, {%2, %4};\n\tsetp.ne.u32 p, %5, 0;\n\t"
                 "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %3, p;\n\t"
                 "add.u32 x, %1, 8;\n\tadd.s64 y, y, 128;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], [x], y, %3, 1;\n\t"
                 "add.u32 x, %1, 16;\n\tadd.s64 y, y, 128;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], [x], y, %3, 1;\n\t"
                 "add.u32 x, %1, 24;\n\tadd.s64 y, y, 128;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], [x], y, %3, 1;\n\t"
                 "add.u32 x, %1, 32;\n\tadd.s64 y, y, 128;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], [x], y, %3, 1;\n\t"
                 "add.u32 x, %1, 40;\n\tadd.s64 y, y, 128;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], [x], y, %3, 1;\n\t"
                 "add.u32 x, %1, 48;\n\tadd.s64 y, y, 128;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], [x], y, %3, 1;\n\t"
                 "add.u32 x, %1, 56;\n\tadd.s64 y, y, 128;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], [x], y, %3, 1;\n\t}"
                 ::"r"(d), "r"(p), "r"(v), "r"(idesc), "n"(kPDescUpper), "r"((uint32_t)add) : "memory");
}

template <int P, bool N16>
__global__ void __launch_bounds__(kPThreads, 1) ragged_umma(const RaggedArgs a) {
    constexpr int D = kHeadDim, ROW_M = D * P / 8;
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ int s_scan[2][kPThreads / 32];
    __shared__ uint32_t s_tmem;
    __shared__ RaggedCursor s_at[8];         // of each warp of rows, while it needs its registers
    __shared__ int64_t s_rows[16][8];        // of a tile, by its number mod 16: the plane's row of every 16th token, -1: not to be read
    __shared__ int s_flags[16];      // of a tile: 1 it begins a run, 2 its entry has rows in half 1, 4 it ends a run
    int *s_items = reinterpret_cast<int*>(smem), *s_entries = s_items + kMaxPagedBatch + 1;      // (until rows come here)
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t base = smem_u32(smem), bars = base + kPBars;
    // step j of a block: K of its tile j and V of its tile j - 1
    auto b_full = [&](int j) { return bars + 8 * (j & 1); };                    // both converted
    auto b_s = [&](int h, int j) { return bars + 16 + 16 * h + 8 * (j & 1); };  // S of tile j, half h done; h = 1: all of step j
    auto b_p = [&](int h) { return bars + 48 + 8 * h; };                        // P of a half written
    auto b_o = [&](int h) { return bars + 64 + 8 * h; };                        // O of a run done
    auto b_q = [&](int h) { return bars + 80 + 8 * h; };                        // pi(Q) of a run there
    auto b_plan = [&](int i) { return bars + 96 + 8 * ((i >> 3) & 1); };        // rows and flags of tile i and its batch of eight there
    auto b_used = [&](int i) { return bars + 112 + 8 * ((i >> 3) & 1); };       //   and used
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(b_full(i), 8); mbar_init(b_s(i, 0), 1); mbar_init(b_s(i, 1), 1);
            mbar_init(b_p(i), 4); mbar_init(b_o(i), 1); mbar_init(b_q(i), 4);
            mbar_init(b_plan(8 * i), 1); mbar_init(b_used(8 * i), 9);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async_shared();
    }
    // (so that a warp whose wait for the plan ran out finds rows that are not to be read)
    if (tid < 16 * 8) (&s_rows[0][0])[tid] = -1;
    if (warp == 0) tmem_alloc(smem_u32(&s_tmem), 512);
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const uint32_t tm = __shfl_sync(0xffffffffu, s_tmem, 0);
    pdl_wait();
    ragged_count<kPThreads>(a, s_items, s_entries, s_scan, kPRows, kPTile);
    const int H = a.fmt.n_kv_heads, n_items = s_items[a.batch], me = blockIdx.x;
    const int workers = min(a.workers, n_items);
    // this block's tiles: from its first item to its successor's
    RaggedCursor c;
    int n_mine = 0, first_worker = 0;         // tiles; the worker that the entry of the first one begins in
    if (me < workers) {
        auto tiles_before = [&](int item, int& at) {
            const int b = ragged_find(a, s_items, item);
            int before;
            at = ragged_seek(a, c, b, item - s_items[b], kPRows, kPTile, before);
            return item - at + c.k - a.extra * (s_entries[b] + before);
        };
        int at;
        n_mine = me + 1 < workers ? tiles_before(worker_start(me + 1, n_items, workers), at) : n_items - a.extra * s_entries[a.batch];
        const int item = worker_start(me, n_items, workers);
        n_mine -= tiles_before(item, at);
        first_worker = worker_of(item - at + a.extra, n_items, workers);
    }
    __syncthreads();
    auto next_tile = [&]() {           // true: the next tile begins another run
        if (++c.k < c.v.n) return false;
        ragged_next(a, c, kPRows, kPTile);
        return true;
    };
    auto park = [&]() {
        __syncwarp();
        if (lane == 0) s_at[warp - 4] = c;
        __syncwarp();
    };
    auto two = [&]() { return c.s.n * a.group > c.rt * kPRows + 128; };       // does the entry have rows in half 1
    bool dead = false;                 // a wait ran out: no more waits, the flag is up, results are void
    auto wait = [&](uint32_t bar, int phase) {
        if (!mbar_try(bar, (uint32_t)phase & 1u) && !dead && !mbar_wait_bounded(bar, (uint32_t)phase & 1u)) {
            dead = true;
            raise_flag(a.status, KVBFP_FLAG_WAIT_TIMEOUT);
        }
    };

    if (warp == 2 || warp == 3) {
        regs_less<kPRegsRest>();
    } else if (warp == 1) {
        // ================================================================ what comes: rows and flags of the tiles, up to 16 ahead
        // (one warp walks the tiles for the nine that only need to know where they are)
        regs_less<kPRegsRest>();
        bool first = true;
        for (int i = 0; i < n_mine; ++i) {
            if (i >= 16 && (i & 7) == 0) wait(b_used(i), (i >> 4) - 1);
            if (lane < 8) {
                // are any of the 16 tokens seen: they begin at `tok`, the last row sees up to p1, the first from p0 - window + 1 on
                const int tok = ragged_token(c.v, c.k, kPTile) + 16 * lane;
                int64_t row = -1;
                if (tok <= c.v.p1 && (a.window == 0 || tok + 15 > c.v.p0 - a.window || tok < a.n_sink)) {
                    const int page = token_page(a.map, c.b, tok);
                    if (page >= 0) row = ((int64_t)page * H + c.hk) * a.fmt.max_seq + token_row(a.map, tok);
                    else raise_flag(a.status, KVBFP_FLAG_POSITION);
                }
                s_rows[i & 15][lane] = row;
            }
            int flags = (first ? 1 : 0) | (two() ? 2 : 0);
            first = i + 1 == n_mine || next_tile();
            if (first) flags |= 4;
            if (lane == 0) s_flags[i & 15] = flags;
            if ((i & 7) == 7 || i + 1 == n_mine) {
                __syncwarp();
                if (lane == 0) mbar_arrive(b_plan(i));
            }
        }
    } else if (warp == 0) {
        // ================================================================ matrix instructions
        // (one warp for both halves: their products alternate, and so the halves fall half a period apart)
        regs_less<kPRegsRest>();
        constexpr uint32_t id_s = umma_idesc(128, 128, false, false), id_o = umma_idesc(128, 128, false, true);
        const int n = __shfl_sync(0xffffffffu, n_mine, 0);
        const uint32_t tmu = __shfl_sync(0xffffffffu, tm, 0);
        const uint32_t qd = prompt_desc(base + kPQ, 16), kd = prompt_desc(base + kPK, 16), vd = prompt_desc(base + kPV, kPPanel);
        int runs = 0;                 // parities of the runs of the halves so far (bits 0 and 1)
        int now = 0, next = 0;        // flags of tiles j - 1 and j
        auto flags_of = [&](int j) {       // of tile j, once what step j needs is converted
            wait(b_full(j), j >> 1);
            if (j >= n) return 0;
            if ((j & 7) == 0) wait(b_plan(j), j >> 4);
            const int f = __shfl_sync(0xffffffffu, *(volatile int*)&s_flags[j & 15], 0);
            if ((j & 7) == 7 && lane == 0) mbar_arrive(b_used(j));
            return f;
        };
        if (n > 0) next = flags_of(0);
        for (int j = 0; j <= n && n > 0; ++j) {
            const int st = j & 1;
            int after = 0;
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
                const uint32_t tmh = tmu + 128 * h;
                if (j > 0) {                             // O of tile j - 1
                    wait(b_p(h), j - 1);
                    __syncwarp();
                    tmem_fence_after();
                    if (h == 0 || (now & 2)) {
                        prompt_o(tmh + 256, tmh, vd + ((st * 32768) >> 4), id_o, !(now & 1));
                        if (now & 4) umma_commit(b_o(h));
                    }
                }
                if (j < n) {                             // S of tile j
                    if (h == 0 || (next & 2)) {
                        if (next & 1) {
                            wait(b_q(h), runs >> h);
                            runs ^= 1 << h;
                            __syncwarp();
                            tmem_fence_after();
                        }
                        prompt_s(tmh, qd + ((h * 32768) >> 4), kd + ((st * 32768) >> 4), id_s);
                    }
                    umma_commit(b_s(h, j));
                    if (h == 0) after = flags_of(j + 1);          // (between the halves, where it costs nothing)
                }
            }
            now = next;
            next = after;
            if (__any_sync(0xffffffffu, dead)) break;
        }
        if (__any_sync(0xffffffffu, dead)) {
            // let what was issued come to its end before the memory goes
            umma_commit(b_o(0));
            (void)mbar_wait_bounded(b_o(0), 0);
            (void)mbar_wait_bounded(b_o(0), 1);
        }
    } else if (warp >= 12) {
        // ================================================================ packed rows to bf16
        regs_less<kPRegsConv>();
        // LANES lanes to a row, 128 / LANES slots each.  8 bits: four, so that whole lines are read (a thread per row reads 16 bytes of
        // 32 rows at a time: four chunks over 14 000 rows each 3.0 ms, 2.65 this way).  4 and 6 bits: one, whose weights serve a
        // whole row (2.18 ms against 2.28 with four; 6 bits 689 us against 775 for a prompt of 8192).
        constexpr int LANES = P == 8 ? 4 : 1, ROWS = LANES;        // rows of a thread
        const int row_e = D / a.fmt.block, w4 = warp & 3, u = lane % LANES, flip = u >> 1;      // (flip: below)
        const int plane = (warp - 12) >> 2;                 // K, V
        const uint8_t *mant = plane ? a.v_mant : a.k_mant, *exps = plane ? a.v_exp : a.k_exp;
        const uint32_t stages = base + (plane ? kPV : kPK);
        const uint32_t sel = row_e == 4 ? 0x3210u : row_e == 2 ? 0x1100u : 0x0000u;
        const int e_at = N16 ? 2 * u : row_e == 4 ? u : row_e == 2 ? flip : 0;
        uint32_t w[4][P], e[4];              // 32 slots each: of four rows, or a whole row (then e: its exponent bytes)
        auto row_of = [&](int x) { return LANES == 1 ? 32 * w4 + lane : 32 * w4 + 8 * x + (lane >> 2); };
        auto load = [&](int i) {             // the rows of tile i
            if ((i & 7) == 0) wait(b_plan(i), i >> 4);
            int64_t first[2];
#pragma unroll
            for (int x = 0; x < 2; ++x) first[x] = *(volatile int64_t*)&s_rows[i & 15][2 * w4 + (LANES == 1 ? lane >> 4 : x)];
            __syncwarp();
            if ((i & 7) == 7 && lane == 0) mbar_arrive(b_used(i));
#pragma unroll
            for (int x = 0; x < ROWS; ++x) {
                const int64_t f = first[x >> 1], row = f + (row_of(x) & 15);
                if (f < 0) {
#pragma unroll
                    for (int z = 0; z < 4; ++z) {
                        if (LANES != 1 && z != x) continue;
                        e[z] = 0u;
#pragma unroll
                        for (int y = 0; y < P; ++y) w[z][y] = 0u;
                    }
                    continue;
                }
                const uint8_t *p = mant + row * ROW_M + 4 * P * u, *q = exps + row * row_e;
                if (LANES == 1) {
#pragma unroll
                    for (int y = 0; y < P; ++y) {
                        const uint4 v = reinterpret_cast<const uint4*>(p)[y];
                        w[(4 * y) / P][(4 * y) % P] = v.x;
                        w[(4 * y + 1) / P][(4 * y + 1) % P] = v.y;
                        w[(4 * y + 2) / P][(4 * y + 2) % P] = v.z;
                        w[(4 * y + 3) / P][(4 * y + 3) % P] = v.w;
                    }
                    if (N16) {
                        const uint2 v = *reinterpret_cast<const uint2*>(q);
                        e[0] = v.x;
                        e[1] = v.y;
                    } else {
                        e[0] = row_e == 4 ? *reinterpret_cast<const uint32_t*>(q) : row_e == 2 ? *reinterpret_cast<const uint16_t*>(q) : *q;
                    }
                } else {
                    // (the lanes of a row's second half take the halves of their 32 slots the other way round, so that eight lanes store to
                    // all banks)
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const uint4 v = *reinterpret_cast<const uint4*>(p + 16 * (flip ^ y));
                        w[x][(4 * y) % P] = v.x;
                        w[x][(4 * y + 1) % P] = v.y;
                        w[x][(4 * y + 2) % P] = v.z;
                        w[x][(4 * y + 3) % P] = v.w;
                    }
                    e[x] = N16 ? *reinterpret_cast<const uint16_t*>(q + e_at) : q[e_at];
                }
            }
        };
        auto convert = [&](uint32_t to) {
            uint32_t top = e[0];
            if (LANES == 1) top = N16 ? vmaxu4(e[0], e[1]) : prmt(e[0], 0u, sel);
            else
#pragma unroll
                for (int x = 1; x < 4; ++x) top = vmaxu4(top, e[x]);
            const bool large = __vcmpgtu4(top, kPFast<P> * 0x01010101u) != 0u;
            const bool slow = __any_sync(0xffffffffu, large);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                // exponent bytes of the 32 slots' halves, as they lie in w, in both halves of a word
                uint32_t e0, e1;
                if (LANES == 1) {
                    e0 = N16 ? prmt(e[x >> 1], 0u, 0x4040u + 0x0101u * (2 * (x & 1))) : prmt(top, 0u, 0x4040u + 0x0101u * x);
                    e1 = N16 ? prmt(e[x >> 1], 0u, 0x4040u + 0x0101u * (2 * (x & 1) + 1)) : e0;
                } else {
                    e0 = N16 ? prmt(e[x], 0u, flip ? 0x4141u : 0x4040u) : e[x] * 0x00010001u;
                    e1 = N16 ? prmt(e[x], 0u, flip ? 0x4040u : 0x4141u) : e0;
                }
                uint32_t v[16];
                if (!slow) convert32<P>(w[x], prompt_weights<P>(e0), prompt_weights<P>(e1), v);
                else prompt_convert_large<P>(w[x], prompt_weights_large<P>(e0), prompt_weights_large<P>(e1), v);
#pragma unroll
                for (int y = 0; y < 4; ++y)
                    sts128(to + prompt_place(row_of(x), LANES == 1 ? 4 * x + y : 4 * u + (y ^ (2 * flip))), v[4 * y], v[4 * y + 1], v[4 * y + 2], v[4 * y + 3]);
            }
            fence_async_shared();
            __syncwarp();
        };
        if (n_mine > 0) load(0);
        if (n_mine > 0 && plane && lane == 0) mbar_arrive(b_full(0));        // (no V in the first step, no K in the last)
        for (int i = 0; i < n_mine; ++i) {
            const int j = i + plane;
            if (j >= 2) wait(b_s(1, j), (j >> 1) - 1);
            convert(stages + (j & 1) * 32768);
            if (lane == 0) mbar_arrive(b_full(j));
            if (i + 1 < n_mine) load(i + 1);
        }
        if (n_mine > 0 && !plane) {
            if (n_mine >= 2) wait(b_s(1, n_mine), (n_mine >> 1) - 1);
            if (lane == 0) mbar_arrive(b_full(n_mine));
        }
    } else {
        // ================================================================ rows
        regs_more<kPRegsRows>();
        const int h = (warp >> 2) - 1, w4 = warp & 3, r = tid & 127;                   // half, quarter of its rows, row
        const uint32_t tms = tm + 128 * h + ((uint32_t)w4 << 21), tmo = tms + 256;      // lane field: 32 * quarter << 16
        const uint32_t q_at = base + kPQ + h * 32768;
        const float mul = finite_factor(a.scale * (float)(1 << kPDown) * 1.4426950408889634f);      // scores to log2 units
        int4 rec = make_int4(-1, 0, 0, 0);
        // This lane's row of q among the warp's 32 rows of the entry at a cursor (NULL: behind the last)
        auto q_row = [&](const RaggedCursor& e) -> const uint8_t* {
            const int row = e.rt * kPRows + h * 128 + w4 * 32 + lane, i = row / a.group;
            if (row >= e.s.n * a.group) return nullptr;
            return static_cast<const uint8_t*>(a.q) + ((int64_t)(e.s.start + i) * a.n_q_heads + e.hk * a.group + row - i * a.group) * (2 * D);
        };
        // pi(Q) of the entry at the cursor, this warp's 32 rows: as they are first, then slot by slot (a lane has four positions)
        auto write_q = [&]() {
            const uint64_t mine = reinterpret_cast<uint64_t>(q_row(c));
#pragma unroll
            for (int x = 0; x < 32; x += 2) {
                const uint64_t src = __shfl_sync(0xffffffffu, mine, x + (lane >> 4));
                const uint32_t dst = q_at + prompt_place(w4 * 32 + x + (lane >> 4), lane & 15);
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src ? src + (lane & 15) * 16 : reinterpret_cast<uint64_t>(a.q)), "r"(src ? 16 : 0) : "memory");
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
            int ch[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int slot = prompt_slot<P>(4 * lane + x);
                ch[x] = a.perm_k ? a.perm_k[c.hk * D + slot] & (D - 1) : slot;
            }
            {          // the rows of the run after this one on their way to the L2 cache
                RaggedCursor e = c;
                ragged_next(a, e, kPRows, kPTile);
                if (e.b < a.batch) {
                    const uint8_t* p = q_row(e);
                    if (p) asm volatile("prefetch.global.L2 [%0];\n\tprefetch.global.L2 [%0+128];" ::"l"(p));
                }
            }
            asm volatile("cp.async.wait_group 0;" ::: "memory");
            __syncwarp();
#pragma unroll 1
            for (int x0 = 0; x0 < 32; x0 += 8) {
                uint32_t v[8][4];
#pragma unroll
                for (int x = 0; x < 8; ++x)
#pragma unroll
                    for (int y = 0; y < 4; ++y)
                        asm volatile("ld.shared.u16 %0, [%1];" : "=r"(v[x][y]) : "r"(q_at + prompt_place(w4 * 32 + x0 + x, ch[y] >> 3) + (ch[y] & 7) * 2) : "memory");
                __syncwarp();
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
        // 128 bytes of this warp's rows from shared memory to where each lane's row goes (0: nowhere), whole lines at a time
        const uint32_t line = base + kPOut + (warp - 4) * 4096;
        auto flush = [&](uint64_t to) {
            __syncwarp();
#pragma unroll
            for (int x = 0; x < 32; x += 4) {
                const int row = x + (lane >> 3);
                const uint64_t p = __shfl_sync(0xffffffffu, to, row);
                const uint4 v = lds128(line + row * 128 + (((lane & 7) ^ (row & 7)) << 4));
                if (p) reinterpret_cast<uint4*>(p)[lane & 7] = v;
            }
            __syncwarp();
        };
        int n_run = 0;                // runs of this half so far
        if (n_mine > 0 && (h == 0 || two())) write_q();
        for (int it = 0; it < n_mine;) {
            // ---- a run: tiles [k0, k1) of one entry
            const int k0 = c.k, k1 = min(c.v.n, k0 + n_mine - it), n_tiles = c.v.n;
            const bool here = h == 0 || two();
            const int R = c.s.n * a.group, row = c.rt * kPRows + h * 128 + r;
            const int pos = c.s.base + min(row, R - 1) / a.group;
            const int pos_lo = c.s.base + min(row - r, R - 1) / a.group, pos_hi = c.s.base + min(row - r + 127, R - 1) / a.group;
            const int see_lo = a.window > 0 ? pos - a.window + 1 : 0;
            const int v_np = c.v.np, v_lo = c.v.lo;
            float m = -3.4028235e38f, l = 0.f;
            park();
            for (int k = k0; k < k1; ++k) {
                const int tt = (k < v_np ? k : k - v_np + v_lo) * kPTile, tile = it + k - k0;
                wait(b_s(h, tile), tile >> 1);
                __syncwarp();
                tmem_fence_after();
                if (here) {
                    const bool clear = tt + 127 <= pos_lo && (a.window == 0 || tt > pos_hi - a.window || tt + 128 <= a.n_sink);
                    // 32 tokens at a time, the next ones on their way.  P is formed under the reference there is; where its sum
                    // passes kPLimit (a run's first tokens, hardly ever else) the scores, which are still there, are read again
                    // and the reference goes up to their maximum.
                    uint32_t s[2][32];
                    tmem_ld<32>(tms, s[0]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t (&v)[32] = s[j & 1];
                        tmem_wait_ld(v);
                        if (j < 3) tmem_ld<32>(tms + 32 * (j + 1), s[(j + 1) & 1]);
                        uint32_t p[16];
                        float sum;
                        auto hide = [&]() {          // hidden ones -inf: tokens up to pos are seen, from see_lo on or among the first ones
                            if (clear) return;
                            const int t0 = tt + 32 * j;
                            auto below = [](int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; };
                            const uint32_t see = below(pos - t0 + 1) & (~below(see_lo - t0) | below(a.n_sink - t0));
#pragma unroll
                            for (int e = 0; e < 32; ++e) v[e] = (see >> e) & 1u ? v[e] : 0xff800000u;
                        };
                        auto form = [&]() {          // P of the 32 scores and its sum
                            const F2 mul2 = f2(mul, mul), neg2 = f2(-m, -m);
                            F2 sums[2] = {f2(0.f, 0.f), f2(0.f, 0.f)};
#pragma unroll
                            for (int e = 0; e < 16; ++e) {
                                float x0, x1;
                                f2_split(f2_fma(f2(__uint_as_float(v[2 * e]), __uint_as_float(v[2 * e + 1])), mul2, neg2), x0, x1);
                                x0 = ex2_approx(x0);
                                x1 = ex2_approx(x1);
                                sums[e & 1] = f2_add(sums[e & 1], f2(x0, x1));
                                p[e] = pack_bf16x2_rn(x0, x1);
                            }
                            float a0, a1;
                            f2_split(f2_add(sums[0], sums[1]), a0, a1);
                            sum = a0 + a1;
                        };
                        hide();
                        form();
                        if (__any_sync(0xffffffffu, sum > kPLimit)) {
                            tmem_ld<32>(tms + 32 * j, v);
                            tmem_wait_ld(v);
                            hide();
                            float top = -INFINITY;
#pragma unroll
                            for (int e = 0; e < 16; ++e) top = max3(top, __uint_as_float(v[2 * e]), __uint_as_float(v[2 * e + 1]));
                            top *= mul;
                            // (whole numbers, so that what is there is scaled by a power of two)
                            const float y = fmaxf(m, ceilf(top)), al = ex2_approx(m - y);
                            m = y;
                            l *= al;
                            if (k > k0) {         // O is at rest: S came behind all products before it
#pragma unroll 1
                                for (int x = 0; x < 16; ++x) {
                                    uint32_t o[8];
                                    tmem_ld<8>(tmo + 8 * x, o);
                                    tmem_wait_ld(o);
#pragma unroll
                                    for (int e = 0; e < 8; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * al);
                                    tmem_st<8>(tmo + 8 * x, o);
                                }
                            }
                            const uint32_t al2 = pack_bf16x2_rn(al, al);
                            tmem_wait_st();
#pragma unroll 1
                            for (int x = 0; x < 2 * j; ++x) {          // and P of this tile's tokens before
                                uint32_t o[8];
                                tmem_ld<8>(tms + 8 * x, o);
                                tmem_wait_ld(o);
#pragma unroll
                                for (int e = 0; e < 8; ++e) o[e] = mul_bf16x2(o[e], al2);
                                tmem_st<8>(tms + 8 * x, o);
                            }
                            form();
                        }
                        tmem_st<16>(tms + 16 * j, p);
                        l += sum;
                    }
                    tmem_wait_st();
                }
                tmem_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(b_p(h));
            }
            c = s_at[warp - 4];
            it += k1 - k0;
            // ---- the run's result; pi(Q) of the next run first where it need not wait for it
            const bool whole = k0 == 0 && k1 == n_tiles;
            if (k0 > 0 && k1 == n_tiles) rec = make_int4(c.b, c.rt, c.hk, first_worker);
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
                const float inv = l != 0.f ? (float)(1 << kPDown) / l : 0.f;
                wait(b_o(h), n_run++);
                __syncwarp();
                tmem_fence_after();
                const uint32_t my_line = line + lane * 128;
                const uint64_t to = !wanted ? 0 : whole ? reinterpret_cast<uint64_t>(static_cast<__nv_bfloat16*>(a.out) + out_row * D) : reinterpret_cast<uint64_t>(part);
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
                            sts128(my_line + (((2 * x) ^ (lane & 7)) << 4), __float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
                            sts128(my_line + (((2 * x + 1) ^ (lane & 7)) << 4), __float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7]));
                            continue;
                        }
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] = l != 0.f ? v[e] * inv : 0.f;
                        const uint32_t at = staged ? q_at + prompt_place(r, 4 * j + x) : my_line + (((4 * (j & 1) + x) ^ (lane & 7)) << 4);
                        sts128(at, pack_bf16x2_rn(v[0], v[1]), pack_bf16x2_rn(v[2], v[3]), pack_bf16x2_rn(v[4], v[5]), pack_bf16x2_rn(v[6], v[7]));
                    }
                    if (!whole) flush(to ? to + 128 * j : 0);
                    else if (!staged && (j & 1)) flush(to ? to + 64 * (j - 1) : 0);
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
                        const uint64_t p = __shfl_sync(0xffffffffu, to, x);
                        uint32_t v[4];
#pragma unroll
                        for (int y = 0; y < 4; ++y)
                            asm volatile("ld.shared.u16 %0, [%1];" : "=r"(v[y]) : "r"(q_at + prompt_place(w4 * 32 + x, sl[y] >> 3) + (sl[y] & 7) * 2) : "memory");
                        if (p) reinterpret_cast<uint2*>(p)[lane] = make_uint2(v[0] | v[1] << 16, v[2] | v[3] << 16);
                    }
                    __syncwarp();
                }
            }
            if (next_here && staged) write_q();
        }
        if (tid == 128) a.rec[me] = rec;
    }
    __syncwarp();
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    if (warp == 0) tmem_dealloc(tm, 512);
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
