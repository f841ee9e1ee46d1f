// Pages of a cache: giving them back, sharing them, reserving them, packing them, copying them.
//
// The bookkeeping is a few integers per page and entry, so what it costs is launches and round trips to memory; it stays on
// the device because the lengths do.  Nothing depends on the order of atomics: reference counts only add and subtract, and new
// pages are found by scanning the counts in page order (which also gives every run the same pages).
// Four calls of a step (free, fork, reserve, copy; 8 x 4 branches) take 13.5 us in a graph; packing 16384 pages of 64 tokens x 8
// heads into another pool 198 us, 0.88 of the copy rate.  Reserving scans the counts from the first page on until enough free ones are
// found: where those are the last of 1000, 16384, 131072 pages 4.6, 7.6, 33 us.
#include "pages.cuh"

namespace kvbfp {
namespace {

constexpr int kScanThreads = 1024;

struct Pool {
    int batch, max_pages, n_pages, shift;
    int32_t *table, *refs, *lens;
};
Pool pool_of(const kvbfp_pages& p) {
    Pool a = {p.batch, p.max_pages, p.n_pages, 0, p.table, p.refs, p.lens};
    while ((1 << a.shift) < p.page_tokens) ++a.shift;
    return a;
}
__device__ __forceinline__ int pages_for(const Pool& p, int tokens) { return (int)(((int64_t)tokens + (1 << p.shift) - 1) >> p.shift); }
__device__ __forceinline__ bool is_page(const Pool& p, int x) { return x >= 0 && x < p.n_pages; }

// One block per sequence.
__global__ void __launch_bounds__(128) pages_free(Pool p, const int32_t* lo_in, const int32_t* hi_in) {
    const int b = blockIdx.x;
    pdl_wait();
    pdl_trigger();
    const int len = max(p.lens[b], 0), lo = lo_in ? max(lo_in[b], 0) : 0, hi = hi_in ? hi_in[b] : 0x7fffffff;
    const bool cut = hi >= len;
    // pages [i0, i1): whole ones inside the range, all behind its start where it reaches the end
    const int i0 = pages_for(p, lo), i1 = cut ? p.max_pages : min(max(hi, 0) >> p.shift, p.max_pages);
    int32_t* row = p.table + (int64_t)b * p.max_pages;
    for (int i = i0 + threadIdx.x; i < i1; i += 128) {
        const int x = row[i];
        if (is_page(p, x)) atomicSub(&p.refs[x], 1);
        if (x >= 0) row[i] = -1;
    }
    __syncthreads();
    if (threadIdx.x == 0 && cut && lo < len) p.lens[b] = lo;
}

// One block per pair.
__global__ void __launch_bounds__(128) pages_fork(Pool p, const int32_t* src, const int32_t* dst, int n, uint32_t* status) {
    const int i = blockIdx.x, tid = threadIdx.x;
    pdl_wait();
    pdl_trigger();
    const int s = src[i], d = dst[i];
    if (s < 0) return;
    const bool inside = s < p.batch && d >= 0 && d < p.batch;
    bool bad = !inside;
    for (int j = tid; j < n; j += 128) {
        if (src[j] < 0) continue;
        bad |= dst[j] == s || (j < i && dst[j] == d);
    }
    int32_t* to = p.table + (int64_t)(inside ? d : 0) * p.max_pages;
    const int32_t* from = p.table + (int64_t)(inside ? s : 0) * p.max_pages;
    if (__syncthreads_or(bad)) {          // (no look at a row that another pair may be writing)
        if (tid == 0) raise_flag(status, KVBFP_FLAG_POSITION);
        return;
    }
    bad = p.lens[d] > 0;
    for (int k = tid; k < p.max_pages; k += 128) bad |= to[k] >= 0;
    if (__syncthreads_or(bad)) {
        if (tid == 0) raise_flag(status, KVBFP_FLAG_POSITION);
        return;
    }
    const int len = max(p.lens[s], 0), held = min(pages_for(p, len), p.max_pages);
    for (int k = tid; k < held; k += 128) {
        const int x = from[k];
        if (is_page(p, x)) {
            atomicAdd(&p.refs[x], 1);
            to[k] = x;
        }
    }
    if (tid == 0) p.lens[d] = len;
}

// Sum over the block of what the threads before this one have; `total`: of all of them.  One barrier before the next use.  Sums end
// at kSumEnd: 1024 sequences may ask for 2^37 pages in all, and no pool has more than 2^28.  (A thread's own share is 2^27 at most,
// so what is left of an ended sum without it is above any pool still.)
constexpr int kSumEnd = 1 << 29;
__device__ __forceinline__ int block_before(int mine, int (&s_warp)[32], int& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int x = mine;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, off);
        if (lane >= off) x = min(x + y, kSumEnd);
    }
    if (lane == 31) s_warp[warp] = x;
    __syncthreads();
    int w = s_warp[lane];
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, w, off);
        if (lane >= off) w = min(w + y, kSumEnd);
    }
    total = __shfl_sync(0xffffffffu, w, 31);
    const int before = warp ? __shfl_sync(0xffffffffu, w, (warp + 31) & 31) : 0;
    __syncthreads();
    return before + x - mine;
}
// Reference counts of four neighbouring pages (1 behind the last: not free).
__device__ __forceinline__ int4 refs4(const Pool& p, int at) {
    if (at + 4 <= p.n_pages) return *reinterpret_cast<const int4*>(p.refs + at);
    int4 x = make_int4(1, 1, 1, 1);
    if (at < p.n_pages) x.x = p.refs[at];
    if (at + 1 < p.n_pages) x.y = p.refs[at + 1];
    if (at + 2 < p.n_pages) x.z = p.refs[at + 2];
    return x;
}

// One block, a thread per sequence, then four pages a thread and step until every page asked for is found.
__global__ void __launch_bounds__(kScanThreads) pages_reserve(Pool p, const int32_t* more_in, int32_t* pairs, uint32_t* status) {
    __shared__ int s_warp[32], s_page[kMaxPagedBatch], s_before[kMaxPagedBatch + 1], s_first[kMaxPagedBatch], s_at[kMaxPagedBatch],
        s_new[kMaxPagedBatch];
    const int b = threadIdx.x;
    const bool seq = b < p.batch;
    pdl_wait();
    pdl_trigger();
    int len = 0, more = 0, at = 0, old = -1, shared = 0;
    bool over = false;
    int32_t* row = p.table + (int64_t)(seq ? b : 0) * p.max_pages;
    if (seq) {
        len = max(p.lens[b], 0);
        more = max(more_in[b], 0);
        over = (int64_t)len + more > ((int64_t)p.max_pages << p.shift);
        if ((int64_t)len + more > 0x7fffffff) more = 0;
        if (over) raise_flag(status, KVBFP_FLAG_PAGES);
    }
    // the page that the first new token falls into, where other tokens are in it already
    const bool into = more > 0 && (len & ((1 << p.shift) - 1)) != 0 && (len >> p.shift) < p.max_pages;
    if (into) {
        at = len >> p.shift;
        old = row[at];
        if (!is_page(p, old)) old = -1;
        shared = old >= 0 ? p.refs[old] : 0;
    }
    s_page[b] = shared > 1 ? old : -1;
    __syncthreads();
    bool keeps = false;           // the last of the owners, all of which write the page
    if (shared > 1) {
        int before = 0;
        for (int j = 0; j < b; ++j) before += s_page[j] == old;
        keeps = before >= shared - 1;
    }
    const int first = into && (old < 0 || (shared > 1 && !keeps)) ? 1 : 0;      // a page in the place of entry `at`
    const int held = min(pages_for(p, len), p.max_pages);
    const int need = more > 0 ? first + min(pages_for(p, len + more), p.max_pages) - held : 0;      // (as far as the table goes)
    int total = 0;
    const int before = block_before(need, s_warp, total);
    if (seq) {
        s_before[b] = before;
        s_first[b] = first;
        s_at[b] = first ? at : held;
        s_new[b] = held;
    }
    if (b == 0) s_before[p.batch] = total;
    __syncthreads();
    int found = 0;
    for (int base = 0; base < p.n_pages && found < total; base += 4 * kScanThreads) {
        const int x0 = base + 4 * b;
        const int4 r = refs4(p, x0);
        const bool f[4] = {r.x <= 0, r.y <= 0, r.z <= 0, r.w <= 0};
        int here = 0;
        int rank = found + block_before(f[0] + f[1] + f[2] + f[3], s_warp, here);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (!f[e]) continue;
            if (rank < total) {
                int lo = 0, hi = p.batch - 1;                       // the sequence whose page this is
                while (lo < hi) {
                    const int mid = (lo + hi + 1) >> 1;
                    if (s_before[mid] <= rank) lo = mid; else hi = mid - 1;
                }
                const int k = rank - s_before[lo];
                const int entry = k < s_first[lo] ? s_at[lo] : s_new[lo] + k - s_first[lo];
                p.table[(int64_t)lo * p.max_pages + entry] = x0 + e;
                p.refs[x0 + e] = 1;
            }
            ++rank;
        }
        found += here;
    }
    __syncthreads();
    if (!seq) return;
    int from = -1, to = -1;
    // (a sequence that keeps a page relies on those before it that share the page, so it goes the way they do)
    const bool granted = (need == 0 && !keeps) || before + need <= found;
    if (!granted) {
        raise_flag(status, KVBFP_FLAG_PAGES);
        for (int k = 0; k < need && before + k < found; ++k) {      // what was dealt out to it goes back
            const int entry = k < first ? at : held + k - first;
            p.refs[row[entry]] = 0;
            row[entry] = k < first ? old : -1;
        }
    } else {
        if (first && old >= 0) {
            from = old;
            to = row[at];
            atomicSub(&p.refs[old], 1);
        }
        if (more > 0) p.lens[b] = len + more;
    }
    *reinterpret_cast<int2*>(pairs + 2 * b) = make_int2(from, to);
}

// One block: where each page goes.  remap: new number of every old page, -1 for free ones.
__global__ void __launch_bounds__(kScanThreads) pages_plan(Pool p, int32_t* dst_refs, int dst_pages, int in_place, int32_t* moves,
                                                           int32_t* count, int32_t* remap, int32_t* holes, uint32_t* status) {
    __shared__ int s_warp[32];
    const int tid = threadIdx.x;
    pdl_wait();
    pdl_trigger();
    int used = 0, n_holes = 0, n_moves = 0;
    if (in_place) {
        int mine = 0;
        for (int base = 0; base < p.n_pages; base += 4 * kScanThreads) {
            const int x0 = base + 4 * tid;
            const int4 r = refs4(p, x0);
            mine += (r.x > 0) + (x0 + 1 < p.n_pages && r.y > 0) + (x0 + 2 < p.n_pages && r.z > 0) + (x0 + 3 < p.n_pages && r.w > 0);
            if (x0 >= p.n_pages) mine -= r.x > 0;
        }
        (void)block_before(mine, s_warp, used);
        for (int base = 0; base < used; base += kScanThreads) {        // free numbers below
            const int x = base + tid;
            const bool hole = x < used && p.refs[x] <= 0;
            int here = 0;
            const int k = n_holes + block_before(hole, s_warp, here);
            if (hole) holes[k] = x;
            if (x < used) remap[x] = hole ? -1 : x;
            n_holes += here;
        }
        __syncthreads();
    }
    for (int base = used; base < p.n_pages; base += kScanThreads) {
        const int x = base + tid;
        const int r = x < p.n_pages ? p.refs[x] : 0;
        const bool live = r > 0;
        int here = 0;
        const int k = n_moves + block_before(live, s_warp, here);
        int to = -1;
        if (live) {
            to = in_place ? holes[k] : k;
            if (!in_place && k >= dst_pages) to = -1;
            if (to >= 0) {
                dst_refs[to] = r;
                if (in_place) p.refs[x] = 0;
                *reinterpret_cast<int2*>(moves + 2 * (int64_t)k) = make_int2(x, to);
            }
        }
        if (x < p.n_pages) remap[x] = to;
        n_moves += here;
    }
    if (!in_place) {
        if (n_moves > dst_pages) {
            n_moves = dst_pages;
            if (tid == 0) raise_flag(status, KVBFP_FLAG_PAGES);
        }
        for (int x = n_moves + tid; x < dst_pages; x += kScanThreads) dst_refs[x] = 0;
    }
    for (int k = n_moves + tid; k < p.n_pages; k += kScanThreads) *reinterpret_cast<int2*>(moves + 2 * (int64_t)k) = make_int2(-1, -1);
    if (tid == 0) *count = n_moves;
}

__global__ void __launch_bounds__(256) pages_renumber(Pool p, int32_t* dst_table, int32_t* dst_lens, const int32_t* remap) {
    pdl_wait();
    pdl_trigger();
    const int64_t n = (int64_t)p.batch * p.max_pages, step = (int64_t)gridDim.x * 256, t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    for (int64_t i = t; i < n; i += step) {
        const int x = p.table[i];
        dst_table[i] = is_page(p, x) ? remap[x] : -1;
    }
    if (dst_lens != p.lens)
        for (int64_t i = t; i < p.batch; i += step) dst_lens[i] = p.lens[i];
}

// Pages between pools: 16-byte pieces of the four planes of a page one behind the other, four a thread in flight, a block per
// kCopyPieces of them.  Memory-bound.
constexpr int kCopyPieces = 1024;
struct CopyArgs {
    const uint4* from[4];
    uint4* to[4];
    int64_t mant, exps;        // pieces of a page in a mantissa and an exponent plane
    int src_pages, dst_pages;
    const int32_t* pairs;
    const int32_t* count;
    int n;
    uint32_t* status;
};
__global__ void __launch_bounds__(256) pages_copy(CopyArgs a, int chunks) {
    pdl_wait();
    pdl_trigger();
    const int n = a.count ? min(max(*a.count, 0), a.n) : a.n;
    const int64_t items = (int64_t)n * chunks, total = 2 * (a.mant + a.exps);
    for (int64_t x = blockIdx.x; x < items; x += gridDim.x) {
        const int i = (int)(x / chunks), c = (int)(x - (int64_t)i * chunks);
        const int2 pr = *reinterpret_cast<const int2*>(a.pairs + 2 * (int64_t)i);
        if (pr.x < 0 || pr.y < 0) continue;
        if (pr.x >= a.src_pages || pr.y >= a.dst_pages) {
            if (threadIdx.x == 0 && c == 0) raise_flag(a.status, KVBFP_FLAG_POSITION);
            continue;
        }
        uint4 v[4];
        uint4* to[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            int64_t u = (int64_t)c * kCopyPieces + j * 256 + threadIdx.x;
            to[j] = nullptr;
            if (u < total) {
                const bool v_side = u >= a.mant + a.exps;
                if (v_side) u -= a.mant + a.exps;
                const bool e = u >= a.mant;
                if (e) u -= a.mant;
                const int64_t size = e ? a.exps : a.mant;
                const uint4* src = v_side ? (e ? a.from[3] : a.from[2]) : (e ? a.from[1] : a.from[0]);
                uint4* dst = v_side ? (e ? a.to[3] : a.to[2]) : (e ? a.to[1] : a.to[0]);
                v[j] = src[pr.x * size + u];
                to[j] = dst + pr.y * size + u;
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (to[j]) *to[j] = v[j];
    }
}

}  // namespace
}  // namespace kvbfp

extern "C" kvbfp_status kvbfp_pages_free(const kvbfp_pages* pool, const int32_t* lo, const int32_t* hi, void* stream) {
    using namespace kvbfp;
    const kvbfp_status st = check_pages(pool, true);
    if (st != KVBFP_OK) return st;
    KVBFP_CUDA(launch_pdl(pages_free, dim3(pool->batch), dim3(128), 0, (cudaStream_t)stream, pool_of(*pool), lo, hi));
    KVBFP_LAUNCH_CHECK("pages_free");
    return KVBFP_OK;
}

extern "C" kvbfp_status kvbfp_pages_fork(const kvbfp_pages* pool, const int32_t* src, const int32_t* dst, int32_t n,
                                         void* stream) {
    using namespace kvbfp;
    kvbfp_status st = check_pages(pool, true);
    if (st != KVBFP_OK) return st;
    if (n < 0 || (n > 0 && (!src || !dst))) return KVBFP_ERR_INVALID_ARG;
    if (n > 65535) return KVBFP_ERR_UNSUPPORTED;
    if (n == 0) return KVBFP_OK;
    uint32_t* status = nullptr;
    st = status_word(&status);
    if (st != KVBFP_OK) return st;
    KVBFP_CUDA(launch_pdl(pages_fork, dim3(n), dim3(128), 0, (cudaStream_t)stream, pool_of(*pool), src, dst, n, status));
    KVBFP_LAUNCH_CHECK("pages_fork");
    return KVBFP_OK;
}

extern "C" kvbfp_status kvbfp_pages_reserve(const kvbfp_pages* pool, const int32_t* more, int32_t* pairs, void* stream) {
    using namespace kvbfp;
    kvbfp_status st = check_pages(pool, true);
    if (st != KVBFP_OK) return st;
    if (!more || !pairs) return KVBFP_ERR_INVALID_ARG;
    if (!aligned16(pairs)) return KVBFP_ERR_ALIGNMENT;
    uint32_t* status = nullptr;
    st = status_word(&status);
    if (st != KVBFP_OK) return st;
    KVBFP_CUDA(launch_pdl(pages_reserve, dim3(1), dim3(kScanThreads), 0, (cudaStream_t)stream, pool_of(*pool), more, pairs, status));
    KVBFP_LAUNCH_CHECK("pages_reserve");
    return KVBFP_OK;
}

extern "C" size_t kvbfp_pages_workspace_bytes(const kvbfp_pages* pool) {
    if (kvbfp::check_pages(pool, true) != KVBFP_OK) return 0;
    return ((size_t)pool->n_pages * 4 + 255) / 256 * 256 * 2;
}

extern "C" kvbfp_status kvbfp_pages_compact(const kvbfp_pages* pool, const kvbfp_pages* dst, int32_t* moves, int32_t* count,
                                            void* workspace, size_t workspace_bytes, void* stream) {
    using namespace kvbfp;
    kvbfp_status st = check_pages(pool, true);
    if (st == KVBFP_OK) st = check_pages(dst, true);
    if (st != KVBFP_OK) return st;
    if (!moves || !count) return KVBFP_ERR_INVALID_ARG;
    if (pool->batch != dst->batch || pool->max_pages != dst->max_pages || pool->page_tokens != dst->page_tokens) return KVBFP_ERR_INVALID_ARG;
    const bool in_place = pool->table == dst->table;
    if ((pool->refs == dst->refs) != in_place || (pool->lens == dst->lens) != in_place) return KVBFP_ERR_INVALID_ARG;
    if (in_place && pool->n_pages != dst->n_pages) return KVBFP_ERR_INVALID_ARG;
    if (!aligned16(moves) || !aligned16(workspace)) return KVBFP_ERR_ALIGNMENT;
    if (!workspace || workspace_bytes < kvbfp_pages_workspace_bytes(pool)) return KVBFP_ERR_WORKSPACE;
    if (!in_place) {        // different pools must not overlap
        const void* p[] = {pool->table, pool->refs, pool->lens};
        const void* q[] = {dst->table, dst->refs, dst->lens};
        const size_t np[] = {(size_t)pool->batch * pool->max_pages * 4, (size_t)pool->n_pages * 4, (size_t)pool->batch * 4};
        const size_t nq[] = {np[0], (size_t)dst->n_pages * 4, np[2]};
        for (int i = 0; i < 9; ++i) {
            const uintptr_t x = (uintptr_t)p[i / 3], y = (uintptr_t)q[i % 3];
            if (x < y + nq[i % 3] && y < x + np[i / 3]) return KVBFP_ERR_INVALID_ARG;
        }
    }
    uint32_t* status = nullptr;
    st = status_word(&status);
    if (st != KVBFP_OK) return st;
    int n_sm = 0;
    st = sm_count(&n_sm);
    if (st != KVBFP_OK) return st;
    int32_t* remap = static_cast<int32_t*>(workspace);
    int32_t* holes = remap + ((size_t)pool->n_pages * 4 + 255) / 256 * 64;
    const Pool p = pool_of(*pool);
    cudaStream_t s = (cudaStream_t)stream;
    KVBFP_CUDA(launch_pdl(pages_plan, dim3(1), dim3(kScanThreads), 0, s, p, dst->refs, (int)dst->n_pages, (int)in_place, moves,
                          count, remap, holes, status));
    KVBFP_LAUNCH_CHECK("pages_plan");
    const int64_t blocks = ((int64_t)p.batch * p.max_pages + 255) / 256;
    KVBFP_CUDA(launch_pdl(pages_renumber, dim3((unsigned)(blocks < 8 * n_sm ? blocks : 8 * n_sm)), dim3(256), 0, s, p, dst->table,
                          dst->lens, (const int32_t*)remap));
    KVBFP_LAUNCH_CHECK("pages_renumber");
    return KVBFP_OK;
}

extern "C" kvbfp_status kvbfp_pages_copy(const kvbfp_cache* src, const kvbfp_cache* dst, const int32_t* pairs, int32_t n,
                                         const int32_t* count, void* stream) {
    using namespace kvbfp;
    if (!src || !dst) return KVBFP_ERR_INVALID_ARG;
    kvbfp_status st = check_format(&src->fmt);
    if (st == KVBFP_OK) st = check_format(&dst->fmt);
    if (st != KVBFP_OK) return st;
    const kvbfp_format &f = src->fmt, &d = dst->fmt;
    if (f.n_kv_heads != d.n_kv_heads || f.max_seq != d.max_seq || f.block != d.block || f.mant_bits != d.mant_bits) return KVBFP_ERR_INVALID_ARG;
    if (n < 0 || (n > 0 && !pairs)) return KVBFP_ERR_INVALID_ARG;
    const uint8_t* from[4] = {src->k_mant, src->k_exp, src->v_mant, src->v_exp};
    uint8_t* to[4] = {dst->k_mant, dst->k_exp, dst->v_mant, dst->v_exp};
    const int64_t rows = (int64_t)f.n_kv_heads * f.max_seq;
    const size_t size[4] = {rows * row_m_bytes(f), rows * row_e_bytes(f), rows * row_m_bytes(f), rows * row_e_bytes(f)};
    int same = 0;
    for (int i = 0; i < 4; ++i) {
        if (!from[i] || !to[i]) return KVBFP_ERR_INVALID_ARG;
        if (!aligned16(from[i]) || !aligned16(to[i])) return KVBFP_ERR_ALIGNMENT;
        same += from[i] == to[i];
    }
    if (!aligned16(pairs)) return KVBFP_ERR_ALIGNMENT;
    if (same != 0 && (same != 4 || f.batch != d.batch)) return KVBFP_ERR_INVALID_ARG;
    for (int x = 0; x < 16 && same == 0; ++x) {        // different pools must not overlap, whichever planes
        const uintptr_t s = (uintptr_t)from[x >> 2], t = (uintptr_t)to[x & 3];
        if (s < t + size[x & 3] * d.batch && t < s + size[x >> 2] * f.batch) return KVBFP_ERR_INVALID_ARG;
    }
    if (n == 0) return KVBFP_OK;
    CopyArgs a = {};
    for (int i = 0; i < 4; ++i) {
        a.from[i] = reinterpret_cast<const uint4*>(from[i]);
        a.to[i] = reinterpret_cast<uint4*>(to[i]);
    }
    a.mant = (int64_t)(size[0] / 16);
    a.exps = (int64_t)(size[1] / 16);
    a.src_pages = f.batch;
    a.dst_pages = d.batch;
    a.pairs = pairs;
    a.count = count;
    a.n = n;
    st = status_word(&a.status);
    if (st != KVBFP_OK) return st;
    int n_sm = 0;
    st = sm_count(&n_sm);
    if (st != KVBFP_OK) return st;
    const int64_t chunks = (2 * (a.mant + a.exps) + kCopyPieces - 1) / kCopyPieces;
    if (chunks > 0x7fffffff) return KVBFP_ERR_UNSUPPORTED;
    const int64_t want = chunks * n, most = (int64_t)n_sm * 8 * 4;
    KVBFP_CUDA(launch_pdl(pages_copy, dim3((unsigned)(want < most ? want : most)), dim3(256), 0, (cudaStream_t)stream, a, (int)chunks));
    KVBFP_LAUNCH_CHECK("pages_copy");
    return KVBFP_OK;
}
