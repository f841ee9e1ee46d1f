// Attention of a ragged batch of new tokens over a contiguous or paged packed cache, causal, with a sliding window and first
// tokens that stay visible: arguments, what a run of query rows sees, and the split of all tiles over the workers.
//
// The query rows of a (sequence, kv head) are its new tokens times the query heads of the group, token-major.  They are cut into
// row tiles; an entry is a (sequence, row tile, kv head), its items are the cache tiles that any of its rows sees.  All items
// (sequence, row tile, kv head, tile: the last fastest) are cut into one contiguous range per worker (attn.cuh), where an entry
// may count for `extra` items more than it has (what beginning and ending it costs), which come before its first; an entry that
// ends in another worker's range than it begins in leaves partial results, at most two a worker, which ragged_merge joins.
#pragma once
#include "attn.cuh"
#include "pages.cuh"

namespace kvbfp {

struct RaggedArgs {
    kvbfp_format fmt;
    TokenMap map;
    const uint8_t *k_mant, *k_exp, *v_mant, *v_exp;
    const void* q;                 // [n_tokens, Hq, d]
    int q_is_bf16;                 // the output has the same type
    int n_q_heads, group, batch, n_tokens;
    const int32_t* starts;
    const int32_t* lens;
    const int32_t* perm_k;
    const int32_t* inv_perm_v;
    float scale;
    int window, n_sink;
    void* out;
    int few_lo, few_hi;            // this kernel takes sequences of that many query rows per kv head: few_lo < rows <= few_hi
    int rows_tile;                 // rows of a row tile
    int part_rows;                 // rows of a partial
    int extra;                     // items that an entry counts for on top of its tiles
    int workers;
    int4* rec;                     // workspace: per worker the entry that ends in its range's first run and began before it:
                                   // sequence, row tile, kv head, first worker (-1: none)
    int* edge;                     // workspace: does a sequence of this kernel have tokens at negative positions
    float* partials;               // workspace: [2 * workers, part_rows, kAttnPart]
    float out_up;                  // sums of P and V as the kernel carries them -> values
    uint32_t* status;
};

struct RaggedSeq {
    int start, n;      // its rows of q: tokens [start, start + n)
    int len, base;     // cached tokens, position of the first new one (negative: more new tokens than cached ones)
    int clamped;
};
__device__ __forceinline__ RaggedSeq ragged_seq(const RaggedArgs& a, int b) {
    RaggedSeq s;
    s.start = min(max(a.starts[b], 0), a.n_tokens);
    s.n = max(min(max(a.starts[b + 1], 0), a.n_tokens) - s.start, 0);
    const int raw = a.lens[b];
    s.len = min(max(raw, 0), a.map.cap);
    s.clamped = s.len != raw;
    s.base = s.len - s.n;
    return s;
}
__device__ __forceinline__ int ragged_row_tiles(const RaggedArgs& a, const RaggedSeq& s, int rows_tile) {
    const int64_t rows = (int64_t)s.n * a.group;
    return rows > a.few_lo && rows <= a.few_hi ? (int)((rows + rows_tile - 1) / rows_tile) : 0;
}

// Tiles that the rows of row tile rt see: the first tokens' tiles [0, np), then those from `lo` on, n in all.
struct RaggedView {
    int p0, p1;        // positions of the first and last row
    int lo, np, n;
};
__device__ __forceinline__ RaggedView ragged_view(const RaggedArgs& a, const RaggedSeq& s, int rt, int rows_tile, int tile) {
    RaggedView v;
    const int r0 = rt * rows_tile, r1 = min(s.n * a.group, r0 + rows_tile) - 1;
    v.p0 = s.base + r0 / a.group;
    v.p1 = s.base + r1 / a.group;
    const int end = v.p1 + 1;
    const int lo = a.window > 0 ? max(v.p0 - a.window + 1, 0) : 0;
    int t0 = lo / tile, np = a.window > 0 ? (min(a.n_sink, max(end, 0)) + tile - 1) / tile : 0;
    const int t1 = end > 0 ? (end + tile - 1) / tile : 0;
    if (np >= t0) t0 = np = 0;
    v.lo = t0;
    v.np = np;
    v.n = np + max(t1 - t0, 0);
    return v;
}
__device__ __forceinline__ int ragged_token(const RaggedView& v, int k, int tile) { return (k < v.np ? k : k - v.np + v.lo) * tile; }

struct RaggedCursor {      // an item: sequence, row tile, kv head, tile k of n
    int b, rt, nrt, hk, k;
    RaggedSeq s;
    RaggedView v;
};
// To the first item of the next entry (b = batch: none).
__device__ __forceinline__ void ragged_next(const RaggedArgs& a, RaggedCursor& c, int rows_tile, int tile) {
    c.k = 0;
    if (++c.hk < a.fmt.n_kv_heads) return;
    c.hk = 0;
    do {
        if (++c.rt >= c.nrt) {
            c.rt = 0;
            do {
                if (++c.b >= a.batch) return;
                c.s = ragged_seq(a, c.b);
                c.nrt = ragged_row_tiles(a, c.s, rows_tile);
            } while (c.nrt == 0);
        }
        c.v = ragged_view(a, c.s, c.rt, rows_tile, tile);
    } while (c.v.n == 0);
}
// To item `at` of sequence b, which has it (whole warp).  Returns where in its entry that is (below a.extra: before its first
// tile, where the cursor stands then); `before`: the sequence's entries before it.
__device__ __forceinline__ int ragged_seek(const RaggedArgs& a, RaggedCursor& c, int b, int at, int rows_tile, int tile, int& before) {
    const int lane = threadIdx.x & 31, H = a.fmt.n_kv_heads;
    c.b = b;
    c.s = ragged_seq(a, b);
    c.nrt = ragged_row_tiles(a, c.s, rows_tile);
    c.rt = 0;
    before = 0;
    for (int r0 = 0; r0 < c.nrt; r0 += 32) {
        const int n = r0 + lane < c.nrt ? ragged_view(a, c.s, r0 + lane, rows_tile, tile).n : 0;
        int x = n > 0 ? (n + a.extra) * H : 0;
        const int mine = x;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, off);
            if (lane >= off) x += y;
        }
        const uint32_t past = __ballot_sync(0xffffffffu, x > at), some = __ballot_sync(0xffffffffu, n > 0);
        if (past) {
            const int l = __ffs(past) - 1;
            c.rt = r0 + l;
            at -= __shfl_sync(0xffffffffu, x - mine, l);
            before += __popc(some & ((1u << l) - 1u)) * H;
            break;
        }
        at -= __shfl_sync(0xffffffffu, x, 31);
        before += __popc(some) * H;
    }
    c.v = ragged_view(a, c.s, c.rt, rows_tile, tile);
    const int n = c.v.n + a.extra;
    c.hk = at / max(n, 1);
    at -= c.hk * n;
    before += c.hk;
    c.k = max(at - a.extra, 0);
    return at;
}

// Items and entries of every sequence, before it and in all: threads of a block together (THREADS of them).  s_items, s_entries:
// room for 1024 + 1.  Starts that decrease (reported) leave nothing to do: sequences that overlap could be more items than 32 bits
// count.  Afterwards entry b of them holds what comes before sequence b, entry `batch` all.  Lengths outside the cache are reported,
// tokens at negative positions noted for the merge, by the first block.
template <int THREADS>
__device__ __forceinline__ void ragged_count(const RaggedArgs& a, int* s_items, int* s_entries, int (&s_scan)[2][THREADS / 32], int rows_tile, int tile) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, H = a.fmt.n_kv_heads;
    constexpr int kAlone = 8;                                  // row tiles that a thread counts by itself
    bool many = false, back = false, edge = false;
    for (int b = tid; b < a.batch; b += THREADS) {
        const RaggedSeq s = ragged_seq(a, b);
        back |= min(max(a.starts[b + 1], 0), a.n_tokens) < s.start;
        const int nrt = ragged_row_tiles(a, s, rows_tile);
        int x = 0, e = 0;
        if (nrt <= kAlone) {
            for (int r = 0; r < nrt; ++r) {
                const int n = ragged_view(a, s, r, rows_tile, tile).n;
                x += n;
                e += n > 0;
            }
        } else {
            e = -1;
            many = true;
        }
        s_items[b] = (x + max(e, 0) * a.extra) * H;
        s_entries[b] = e * H;
        if (blockIdx.x == 0 && nrt > 0) {
            edge |= s.base < 0;
            if (s.clamped) raise_flag(a.status, KVBFP_FLAG_POSITION);
        }
    }
    if (blockIdx.x == 0) {
        edge = __syncthreads_or(edge);
        if (tid == 0) *a.edge = edge;
    }
    if (__syncthreads_or(many || back)) {
        if (__syncthreads_or(back)) {
            if (back && blockIdx.x == 0) raise_flag(a.status, KVBFP_FLAG_POSITION);
            for (int b = tid; b < a.batch; b += THREADS) s_items[b] = s_entries[b] = 0;
            __syncthreads();
        }
        for (int b = warp; b < a.batch; b += THREADS / 32) {
            if (s_entries[b] >= 0) continue;
            const RaggedSeq s = ragged_seq(a, b);
            const int nrt = ragged_row_tiles(a, s, rows_tile);
            int x = 0, e = 0;
            for (int r = lane; r < nrt; r += 32) {
                const int n = ragged_view(a, s, r, rows_tile, tile).n;
                x += n;
                e += n > 0;
            }
            x = __reduce_add_sync(0xffffffffu, x);
            e = __reduce_add_sync(0xffffffffu, e);
            if (lane == 0) {
                s_items[b] = (x + e * a.extra) * H;
                s_entries[b] = e * H;
            }
        }
        __syncthreads();
    }
    const int per = (a.batch + THREADS - 1) / THREADS;
    int x = 0, e = 0;
    for (int i = 0; i < per; ++i)
        if (tid * per + i < a.batch) {
            x += s_items[tid * per + i];
            e += s_entries[tid * per + i];
        }
    const int mine_x = x, mine_e = e;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, off), z = __shfl_up_sync(0xffffffffu, e, off);
        if (lane >= off) {
            x += y;
            e += z;
        }
    }
    if (lane == 31) {
        s_scan[0][warp] = x;
        s_scan[1][warp] = e;
    }
    __syncthreads();
    x -= mine_x;
    e -= mine_e;
    int total_x = 0, total_e = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) {
        if (w < warp) {
            x += s_scan[0][w];
            e += s_scan[1][w];
        }
        total_x += s_scan[0][w];
        total_e += s_scan[1][w];
    }
    for (int i = 0; i < per; ++i) {
        const int b = tid * per + i;
        if (b >= a.batch) break;
        const int nx = s_items[b], ne = s_entries[b];
        s_items[b] = x;
        s_entries[b] = e;
        x += nx;
        e += ne;
    }
    if (tid == 0) {
        s_items[a.batch] = total_x;
        s_entries[a.batch] = total_e;
    }
    __syncthreads();
}
// The sequence that item `at` belongs to.
__device__ __forceinline__ int ragged_find(const RaggedArgs& a, const int* s_items, int at) {
    int lo = 0, hi = a.batch - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (s_items[mid] <= at) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// ragged_rows: items of eight rows, or of four (by rows_tile), a worker per warp
kvbfp_status launch_ragged_rows4(const RaggedArgs& a, int grid, cudaStream_t s);
kvbfp_status launch_ragged_rows6(const RaggedArgs& a, int grid, cudaStream_t s);
kvbfp_status launch_ragged_rows8(const RaggedArgs& a, int grid, cudaStream_t s);
// ragged_umma: bf16 rows in items of 256, a worker per block, one block per SM
kvbfp_status launch_ragged_umma4(const RaggedArgs& a, int grid, cudaStream_t s);
kvbfp_status launch_ragged_umma6(const RaggedArgs& a, int grid, cudaStream_t s);
kvbfp_status launch_ragged_umma8(const RaggedArgs& a, int grid, cudaStream_t s);

}  // namespace kvbfp
