// Attention of several query rows per kv head over the packed cache (drafted trees, masked / capped / biased scores,
// attention weights): arguments, the visible tiles of a sequence and the split of all tiles over the thread blocks.
#pragma once
#include "common.cuh"

namespace kvbfp {

constexpr int kAttnWarps = 4;          // warps per thread block of attn_rows; every warp is a worker of its own
constexpr int kAttnMaxSms = 160;       // SMs that workspaces are sized for
constexpr int kAttnMaxBatch = 1024;    // sequences
constexpr int kAttnPart = kHeadDim + 4;    // floats of a partial row: o[128], max (log2 units), sum, 2 unused
constexpr int kAttnMaxDraft = 64;      // drafted tokens per sequence (bits of a mask word)

// What of one sequence any query may see, in tiles: the prefix tiles [0, np), then the tiles from `lo` on, n in all.
struct SeqView {
    int ctx;       // cached tokens under the context rule
    int nd;        // drafted rows that exist behind them
    int first, pf; // tokens below `pf` are always visible, others from `first` on (and inside the window)
    int lo, np, n;
    int clamped;   // a length was outside the cache
};
__device__ __forceinline__ int tile_token(const SeqView& s, int k, int tile) { return (k < s.np ? k : k - s.np + s.lo) * tile; }

struct RowInfo {
    int pos;           // position of the query row's token
    float slope;
    uint32_t m0, m1;   // drafted tokens it sees (all clear for rows that do not exist)
};

struct AttnArgs {
    kvbfp_format fmt;
    const uint8_t *k_mant, *k_exp, *v_mant, *v_exp;
    const void* q;                 // [B, T, Hq, d]
    int q_is_bf16;                 // the output has the same type
    int n_q_heads, group;
    int n_draft;                   // T (1 for a single token)
    int tree;                      // 0: the query is the last cached token, no drafted rows
    int rows_tile, n_row_tiles;    // query rows (draft-major, group-minor) per work item and items per (batch, kv head)
    int part_rows;                 // rows of a partial: min(all rows, rows_tile)
    int tile;                      // tokens per tile, the unit of the work split
    const int32_t* ctx_lens;
    const int32_t* draft_lens;     // or NULL: all T
    const uint64_t* tree_mask;     // [B, T] or NULL: a chain
    const int32_t* depth;          // [B, T] or NULL: depth = index
    const int32_t* perm_k;
    const int32_t* inv_perm_v;
    float scale;
    float softcap;
    int window;
    const float* slopes;
    const int32_t* first;
    const int32_t* prefix;
    void* out;
    int* plan;                     // workspace: cumulative tile counts of the sequences, [B + 1]
    SeqView* views;                // workspace: [B]
    int* dpos;                     // workspace of attn_umma: [B, 64] positions of the drafted rows
    RowInfo* rows;                 // workspace of attn_umma: [B * Hkv * n_row_tiles, rows_tile]
    uint4* qfrag;                  // workspace of attn_umma: pi(q) as its operand, [B * Hkv * n_row_tiles]
    float* lse;                    // workspace: [B, Hq] log2-sum-exp2, with mass only (else NULL)
    float* scores;                 // workspace: [B, Hq, max_seq] scores in log2 units, with mass only (else NULL)
    float* mass;                   // [B, Hkv, max_seq] or NULL
    float* partials;               // workspace: [2 * workers, part_rows, kAttnPart]
    int workers;                   // warps (attn_rows) or teams (attn_umma) of the main kernel
    float out_up;                  // sums of P and V as the kernel carries them -> values
    uint32_t* status;
};

__device__ __forceinline__ SeqView seq_view(const AttnArgs& a, int b) {
    SeqView s;
    const int raw = a.ctx_lens[b], S = a.fmt.max_seq;
    s.ctx = min(max(raw, 0), S);
    s.clamped = s.ctx != raw;
    s.nd = 0;
    if (a.tree) {
        int want = a.n_draft;
        if (a.draft_lens) want = min(max(a.draft_lens[b], 0), a.n_draft);
        s.nd = min(want, S - s.ctx);
        s.clamped |= (int)(s.nd != want);
    }
    s.first = a.first ? min(max(a.first[b], 0), s.ctx) : 0;
    s.pf = a.prefix ? min(max(a.prefix[b], 0), s.ctx) : 0;
    int lo = s.first;
    const int nearest = a.tree ? s.ctx : s.ctx - 1;              // the lowest query position
    if (a.window > 0 && nearest - a.window + 1 > lo) lo = min(nearest - a.window + 1, s.ctx);
    const int end = s.ctx + s.nd;
    int t0 = lo / a.tile, t1 = (end + a.tile - 1) / a.tile;
    if (lo >= end) t1 = t0;                                       // nothing but the prefix
    int np = (s.pf + a.tile - 1) / a.tile;
    if (np >= t0) {                                               // the two ranges touch
        t1 = (t1 > t0) ? t1 : np;
        if (t1 < np) t1 = np;
        t0 = 0;
        np = 0;
    }
    s.lo = t0;
    s.np = np;
    s.n = np + t1 - t0;
    return s;
}

// All tiles, ordered by sequence, kv head, row tile, tile, are cut into `workers` contiguous ranges of at least one
// (so workers <= n_items: the merge reads a partial of every worker between a row's first and last).
__host__ __device__ __forceinline__ int worker_start(int w, int n_items, int workers) {
    const uint64_t x = (uint64_t)(uint32_t)n_items * (uint32_t)w;
    return x >> 32 ? (int)(x / (uint32_t)workers) : (int)((uint32_t)x / (uint32_t)workers);       // (a 64-bit division takes some hundred instructions)
}
__host__ __device__ __forceinline__ int worker_of(int x, int n_items, int workers) {
    const uint64_t y = (uint64_t)(uint32_t)(x + 1) * (uint32_t)workers - 1u;
    return y >> 32 ? (int)(y / (uint32_t)n_items) : (int)((uint32_t)y / (uint32_t)n_items);
}

// Tokens per tile of attn_rows, stages of a warp and thread blocks per SM (what registers and shared memory allow; four
// blocks spill, shorter tiles pay for the hand-over: 16 x 32 x 8192 rows 193 us with tiles of 32, 173 us with 64).
__host__ __device__ constexpr int attn_rows_tile(int mant_bits) { return mant_bits == 4 ? 64 : 32; }
__host__ __device__ constexpr int attn_rows_stages(int) { return 2; }
__host__ __device__ constexpr int attn_rows_blocks(bool bf16) { return bf16 ? 3 : 2; }
// attn_rows: up to eight bf16 rows, or fp32 rows in items of eight
kvbfp_status launch_attn_rows4(const AttnArgs& a, int grid, cudaStream_t s);
kvbfp_status launch_attn_rows6(const AttnArgs& a, int grid, cudaStream_t s);
kvbfp_status launch_attn_rows8(const AttnArgs& a, int grid, cudaStream_t s);
// Teams (workers) of a block of attn_umma: three where shared memory holds their converted rows (16 x 32 x up to 8192 4-bit
// rows, 16 tokens: 157 us against 174 with two when it was introduced).
__host__ __device__ constexpr int attn_teams(int mant_bits, int rows_tile) { return mant_bits == 4 && rows_tile <= 32 ? 3 : 2; }
// umma_prep and attn_umma: bf16 queries, tiles of 128 tokens, one thread block per SM
kvbfp_status launch_attn_umma4(const AttnArgs& a, int grid, cudaStream_t s);
kvbfp_status launch_attn_umma6(const AttnArgs& a, int grid, cudaStream_t s);
kvbfp_status launch_attn_umma8(const AttnArgs& a, int grid, cudaStream_t s);

}  // namespace kvbfp
