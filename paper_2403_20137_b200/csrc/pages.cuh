// A paged cache on the device: checks of its description, and where a token's rows lie.
#pragma once
#include "common.cuh"

namespace kvbfp {

constexpr int kMaxPagedBatch = 1024;      // sequences of a page table

// The table and, where `state` asks for them, reference counts and lengths.
inline kvbfp_status check_pages(const kvbfp_pages* p, bool state) {
    if (!p || !p->table || (state && (!p->refs || !p->lens))) return KVBFP_ERR_INVALID_ARG;
    if (p->batch < 1 || p->max_pages < 1 || p->n_pages < 1 || p->page_tokens < 1) return KVBFP_ERR_INVALID_ARG;
    if (p->page_tokens < 16 || p->page_tokens > 1024 || (p->page_tokens & (p->page_tokens - 1))) return KVBFP_ERR_UNSUPPORTED;
    if (p->batch > kMaxPagedBatch) return KVBFP_ERR_UNSUPPORTED;
    if ((int64_t)p->max_pages * p->page_tokens >= (int64_t)1 << 31 || p->n_pages > 1 << 28) return KVBFP_ERR_UNSUPPORTED;
    if (!aligned16(p->table) || (state && (!aligned16(p->refs) || !aligned16(p->lens)))) return KVBFP_ERR_ALIGNMENT;
    return KVBFP_OK;
}

// Where the rows of sequence b's tokens are: a contiguous cache (table NULL) or pages.
struct TokenMap {
    const int32_t* table;      // [batch, max_pages] or NULL
    int max_pages, shift, n_pages;
    int cap;                   // tokens a sequence may have
    int n_heads, rows;         // heads; rows per (page or sequence, head)
};
inline TokenMap token_map(const kvbfp_format& f, const kvbfp_pages* p) {
    TokenMap m = {};
    m.n_heads = f.n_kv_heads;
    m.rows = f.max_seq;
    m.cap = f.max_seq;
    if (p) {
        m.table = p->table;
        m.max_pages = p->max_pages;
        m.n_pages = p->n_pages;
        m.cap = p->max_pages * p->page_tokens;
        while ((1 << m.shift) < p->page_tokens) ++m.shift;
    }
    return m;
}
// The cache behind `p` has to be its pool.
inline kvbfp_status check_pool(const kvbfp_format& f, const kvbfp_pages* p) {
    const kvbfp_status st = check_pages(p, false);
    if (st != KVBFP_OK) return st;
    return f.batch == p->n_pages && f.max_seq == p->page_tokens ? KVBFP_OK : KVBFP_ERR_INVALID_ARG;
}
// Page (or sequence) that holds token t of sequence b, -1 where there is none.
__device__ __forceinline__ int token_page(const TokenMap& m, int b, int t) {
    if (!m.table) return b;
    const int p = m.table[(int64_t)b * m.max_pages + (t >> m.shift)];
    return p < m.n_pages ? p : -1;
}
__device__ __forceinline__ int token_row(const TokenMap& m, int t) { return m.table ? t & ((1 << m.shift) - 1) : t; }

}  // namespace kvbfp
