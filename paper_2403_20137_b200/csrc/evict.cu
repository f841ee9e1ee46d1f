// Dropping and moving cached rows: eviction by accumulated attention weight, and the gather of listed rows (the
// accepted branch of a drafted tree) in all four planes of the packed cache.
#include <cooperative_groups.h>

#include "common.cuh"

namespace kvbfp {
namespace {

constexpr int kSelThreads = 512, kSelWarps = kSelThreads / 32;
constexpr int kSelKeys = 16;                 // keys a thread keeps in registers
constexpr int kSelBins = 2048, kSelCluster = 8;
constexpr int kSelCopy = 1024 + 8;           // bins of a copy of the first digit's histogram, eight banks apart from the next

// Weights in the order of unsigned integers: -0 as 0, NaN below everything.
__device__ __forceinline__ uint32_t mass_key(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    if ((u & 0x7fffffffu) > 0x7f800000u) return 0u;
    return (u >> 31) ? ~u : (u | 0x80000000u);
}

// The rows to keep of one (sequence, kv head), in position order, by a block or (CS > 1) a cluster of blocks that share
// the region.  The heaviest `need` of the middle region are found by radix selection: three digits of 10, 11 and 11 bits,
// a histogram each in shared memory (the first, where most weights fall into a few bins, in four copies by lane: 95 -> 87
// us for 16 x 32 x 8192 rows with the move), the cluster's summed through distributed shared memory; of equals to the
// threshold the lowest positions are kept.  Counting is by integer atomics: the result does not depend on their order.  Each warp owns a contiguous piece of the region, so one scan over the warps' counts
// places every kept row.  A thread keeps its keys in registers where they fit (CACHED: up to 8192 rows a block; with
// three blocks an SM some of them spill: 40 registers, 148 bytes) and reads them again otherwise.  What bounds it is the chain of passes, not the bytes (4 per row).
template <int CS, bool CACHED>
__global__ void __launch_bounds__(kSelThreads, CS == 1 ? 3 : 1) evict_select(const float* mass, const int32_t* seq_lens, int max_seq, int n_heads,
                                                            int budget, int n_sink, int n_recent, int32_t* kept, uint32_t* status) {
    __shared__ __align__(16) uint32_t hist0[4 * kSelCopy], hist[2][kSelBins];
    __shared__ uint32_t s_scan[kSelWarps], s_digit, s_need;
    __shared__ int s_gt[kSelWarps], s_eq[kSelWarps], s_tot[2];
    namespace cg = cooperative_groups;
    const int pair = blockIdx.x / CS, rank = blockIdx.x % CS, b = pair / n_heads, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    for (int i = tid; i < 4 * kSelCopy; i += kSelThreads) hist0[i] = 0;
    for (int i = tid; i < 2 * kSelBins; i += kSelThreads) (&hist[0][0])[i] = 0;
    __syncthreads();
    pdl_wait();
    pdl_trigger();
    const int raw = seq_lens[b], len = min(max(raw, 0), max_seq);
    if (raw != len && tid == 0 && rank == 0) raise_flag(status, KVBFP_FLAG_POSITION);
    int32_t* out = kept + (int64_t)pair * budget;
    if (len <= budget) {                                          // (alike in the whole cluster)
        for (int i = rank * kSelThreads + tid; i < budget; i += CS * kSelThreads) out[i] = i < len ? i : -1;
        return;
    }
    const int m0 = n_sink, m1 = len - n_recent;                   // the middle region; m1 - m0 > need
    uint32_t need = (uint32_t)(budget - n_sink - n_recent);
    for (int i = rank * kSelThreads + tid; i < n_sink; i += CS * kSelThreads) out[i] = i;
    for (int i = rank * kSelThreads + tid; i < n_recent; i += CS * kSelThreads) out[budget - n_recent + i] = m1 + i;
    if (need == 0) return;
    const float* x = mass + (int64_t)pair * max_seq;
    // this warp's piece [w0, w1): the region in CS * kSelWarps pieces of whole 32s
    const int per = ((m1 - m0 + CS * kSelWarps - 1) / (CS * kSelWarps) + 31) & ~31;
    const int w0 = min(m0 + (rank * kSelWarps + warp) * per, m1), w1 = min(w0 + per, m1);
    uint32_t keys[CACHED ? kSelKeys : 1];
    if (CACHED) {
#pragma unroll
        for (int j = 0; j < kSelKeys; ++j) {
            const int i = w0 + 32 * j + lane;
            keys[CACHED ? j : 0] = i < w1 ? mass_key(x[i]) : 0u;
        }
    }
    // runs f(position, key, in the piece) over the warp's piece, whole warps at a time
    auto each = [&](auto f) {
        if (CACHED) {
#pragma unroll
            for (int j = 0; j < kSelKeys; ++j)
                if (w0 + 32 * j < w1) f(w0 + 32 * j + lane, keys[CACHED ? j : 0], w0 + 32 * j + lane < w1);
        } else {
#pragma unroll 8
            for (int i = w0 + lane; i - lane < w1; i += 32) f(i, i < w1 ? mass_key(x[i]) : 0u, i < w1);
        }
    };
    uint32_t thr = 0;
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 22 : pass == 1 ? 11 : 0, above_bit = pass == 1 ? 22 : 11;
        const uint32_t mask = pass == 0 ? 1023u : 2047u;
        uint32_t* h = pass == 0 ? hist0 + (lane & 3) * kSelCopy : hist[pass > 0 ? pass - 1 : 0];
        each([&](int, uint32_t key, bool in) {
            const bool take = in && (pass == 0 || (key >> above_bit) == (thr >> above_bit));
            const uint32_t bin = (key >> shift) & mask;
            if (pass == 2) {       // the lowest digits of rounded weights are all alike: one addition then
                const uint32_t who = __ballot_sync(0xffffffffu, take);
                if (who == 0) return;
                const uint32_t lead = __shfl_sync(0xffffffffu, bin, __ffs(who) - 1);
                if (__all_sync(0xffffffffu, !take || bin == lead)) {
                    if (lane == __ffs(who) - 1) atomicAdd(&h[lead], (uint32_t)__popc(who));
                    return;
                }
            }
            if (take) atomicAdd(&h[bin], 1u);
        });
        if (pass == 0) {           // the copies into the first
            __syncthreads();
            for (int i = tid; i < 1024; i += kSelThreads) hist0[i] += hist0[kSelCopy + i] + hist0[2 * kSelCopy + i] + hist0[3 * kSelCopy + i];
        }
        if (CS > 1) cg::this_cluster().sync(); else __syncthreads();
        // thread t holds the last four bins but 4 t (first digit: two), from the top
        uint32_t c[4] = {0u, 0u, 0u, 0u}, sum = 0;
        const uint32_t* first = pass == 0 ? hist0 : hist[pass > 0 ? pass - 1 : 0];
#pragma unroll
        for (int r = 0; r < CS; ++r) {
            const uint32_t* hr = CS > 1 ? cg::this_cluster().map_shared_rank(first, r) : first;
            if (pass == 0) {
                const uint2 v = reinterpret_cast<const uint2*>(hr)[511 - tid];
                c[0] += v.y; c[1] += v.x;
            } else {
                const uint4 v = reinterpret_cast<const uint4*>(hr)[511 - tid];
                c[0] += v.w; c[1] += v.z; c[2] += v.y; c[3] += v.x;
            }
        }
        sum = c[0] + c[1] + c[2] + c[3];
        uint32_t incl = sum;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const uint32_t y = __shfl_up_sync(0xffffffffu, incl, off);
            if (lane >= off) incl += y;
        }
        if (lane == 31) s_scan[warp] = incl;
        __syncthreads();
        uint32_t above = incl - sum;
        for (int w = 0; w < warp; ++w) above += s_scan[w];
#pragma unroll
        for (int j = 0; j < (pass == 0 ? 2 : 4); ++j) {
            if (above < need && above + c[j] >= need) {
                s_digit = (uint32_t)(pass == 0 ? 1023 - 2 * tid - j : kSelBins - 1 - 4 * tid - j);
                s_need = need - above;
            }
            above += c[j];
        }
        __syncthreads();
        thr |= s_digit << shift;
        need = s_need;                     // of the rows that share the digits so far
    }
    // need = rows equal to the threshold that are kept
    int gt = 0, eq = 0;
    each([&](int, uint32_t key, bool in) {
        gt += in && key > thr;
        eq += in && key == thr;
    });
    gt = __reduce_add_sync(0xffffffffu, gt);
    eq = __reduce_add_sync(0xffffffffu, eq);
    if (lane == 0) { s_gt[warp] = gt; s_eq[warp] = eq; }
    __syncthreads();
    int gt0 = 0, eq0 = 0;
    for (int w = 0; w < warp; ++w) { gt0 += s_gt[w]; eq0 += s_eq[w]; }
    if (CS > 1) {
        if (tid == kSelThreads - 1) { s_tot[0] = gt0 + gt; s_tot[1] = eq0 + eq; }       // (a lane of the last warp)
        cg::this_cluster().sync();
        for (int r = 0; r < rank; ++r) {
            const int* t = cg::this_cluster().map_shared_rank(s_tot, r);
            gt0 += t[0];
            eq0 += t[1];
        }
    }
    const int quota = (int)need;
    each([&](int i, uint32_t key, bool in) {
        const bool is_gt = in && key > thr, is_eq = in && key == thr;
        const uint32_t bg = __ballot_sync(0xffffffffu, is_gt), be = __ballot_sync(0xffffffffu, is_eq);
        const uint32_t below = (1u << lane) - 1u;
        const int eq_rank = eq0 + __popc(be & below);
        if (is_gt || (is_eq && eq_rank < quota)) out[n_sink + gt0 + __popc(bg & below) + min(eq_rank, quota)] = i;
        gt0 += __popc(bg);
        eq0 += __popc(be);
    });
    if (CS > 1) cg::this_cluster().sync();            // nobody reads a block's shared memory after it has gone
}

template <int CS, bool CACHED>
kvbfp_status launch_select(const float* mass, const int32_t* seq_lens, const kvbfp_format& f, int budget, int n_sink, int n_recent,
                           int32_t* kept, uint32_t* status, cudaStream_t s) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(f.batch * f.n_kv_heads * CS));
    cfg.blockDim = dim3(kSelThreads);
    cfg.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = CS;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = CS > 1 ? 2 : 1;
    KVBFP_CUDA(cudaLaunchKernelEx(&cfg, evict_select<CS, CACHED>, mass, seq_lens, (int)f.max_seq, (int)f.n_kv_heads, budget, n_sink,
                                  n_recent, kept, status));
    KVBFP_LAUNCH_CHECK("evict_select");
    return KVBFP_OK;
}

struct MoveArgs {
    kvbfp_format src, dst;              // same batch, heads and row format
    const uint8_t* from[4];             // k_mant, k_exp, v_mant, v_exp
    uint8_t* to[4];
    const int32_t* index;               // [batch, heads or 1, n_index]
    int index_heads, n_index;
    const int32_t* count;               // [batch] or NULL: up to the first negative index
    const int32_t* src_base;            // [batch] or NULL: 0
    const int32_t* dst_base;
    const float* mass;                  // [batch, heads, src.max_seq] or NULL
    float* to_mass;                     // [batch, heads, dst.max_seq], zero behind the moved rows
    int32_t* new_lens;                  // eviction: [batch], the number of kept rows
    uint32_t* status;
};

constexpr int kMoveThreads = 256, kMoveRows = 128;

// A piece of a scattered row: no more than 64 bytes around it need come from DRAM.
__device__ __forceinline__ uint4 ld_row(const void* p) {
    uint4 x;
    asm volatile("ld.global.L1::no_allocate.L2::64B.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "l"(p) : "memory");
    return x;
}

// Rows src_base + index[i] -> dst_base + i of all planes, kMoveRows at a time through registers.  A block per (chunk,
// pair) where the caches differ; in place one block per pair walks the chunks upwards: every row of a chunk is read
// before any is written, and as no source lies below its destination (others are refused) later chunks read only rows
// behind the written ones.
template <bool IN_PLACE, int PIECES>      // 16-byte pieces of a mantissa row: 4, 6, 8
__global__ void __launch_bounds__(kMoveThreads) move_rows(const MoveArgs a) {
    constexpr int PER = kMoveRows * PIECES / kMoveThreads;      // pieces per thread and plane
    __shared__ int src_row[kMoveRows];
    pdl_wait();
    pdl_trigger();
    const int H = a.src.n_kv_heads, pair = blockIdx.x, b = pair / H, h = pair - b * H, tid = threadIdx.x;
    const int row_e = kHeadDim / a.src.block;
    const int32_t* idx = a.index + ((int64_t)b * a.index_heads + (a.index_heads == 1 ? 0 : h)) * a.n_index;
    const int n = a.count ? min(max(a.count[b], 0), a.n_index) : a.n_index;
    const int sb = a.src_base ? a.src_base[b] : 0, db = a.dst_base ? a.dst_base[b] : 0;
    const int64_t src0 = (int64_t)pair * a.src.max_seq, dst0 = (int64_t)pair * a.dst.max_seq;
    for (int c = IN_PLACE ? 0 : blockIdx.y; c * kMoveRows < n; c += IN_PLACE ? 1 : gridDim.y) {
        __syncthreads();
        if (tid < kMoveRows) {
            const int i = c * kMoveRows + tid;
            int r = -1;
            if (i < n) {
                const int v = idx[i];
                const int64_t s = (int64_t)sb + v, d = (int64_t)db + i;
                if (v >= 0) {
                    if (s >= 0 && s < a.src.max_seq && d >= 0 && d < a.dst.max_seq && !(IN_PLACE && s < d)) r = (IN_PLACE && s == d) ? -1 : (int)s;
                    else raise_flag(a.status, KVBFP_FLAG_POSITION);
                } else if (a.count) {
                    raise_flag(a.status, KVBFP_FLAG_POSITION);
                }
            }
            src_row[tid] = r;
        }
        __syncthreads();
        uint4 km[PER], vm[PER];
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int x = tid + j * kMoveThreads, r = src_row[x / PIECES];
            if (r >= 0) {
                const int64_t at = (src0 + r) * (PIECES * 16) + (x % PIECES) * 16;
                km[j] = ld_row(a.from[0] + at);
                vm[j] = ld_row(a.from[2] + at);
            }
        }
        // exponent bytes: a thread per (row, plane)
        const int er = tid & (kMoveRows - 1), ep = 1 + 2 * (tid / kMoveRows);
        const int es = src_row[er];
        uint2 eb = make_uint2(0u, 0u);
        if (es >= 0) {
            const uint8_t* p = a.from[ep] + (src0 + es) * row_e;
            if (row_e == 8) eb = *reinterpret_cast<const uint2*>(p);
            else if (row_e == 4) eb.x = *reinterpret_cast<const uint32_t*>(p);
            else if (row_e == 2) eb.x = *reinterpret_cast<const uint16_t*>(p);
            else eb.x = *p;
        }
        float w = 0.f;
        if (a.mass && tid < kMoveRows && src_row[tid] >= 0) w = a.mass[src0 + src_row[tid]];
        if (IN_PLACE) __syncthreads();
        const int64_t d0 = dst0 + db + (int64_t)c * kMoveRows;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int x = tid + j * kMoveThreads, r = x / PIECES;
            if (src_row[r] >= 0) {
                const int64_t at = (d0 + r) * (PIECES * 16) + (x % PIECES) * 16;
                *reinterpret_cast<uint4*>(a.to[0] + at) = km[j];
                *reinterpret_cast<uint4*>(a.to[2] + at) = vm[j];
            }
        }
        if (es >= 0) {
            uint8_t* p = a.to[ep] + (d0 + er) * row_e;
            if (row_e == 8) *reinterpret_cast<uint2*>(p) = eb;
            else if (row_e == 4) *reinterpret_cast<uint32_t*>(p) = eb.x;
            else if (row_e == 2) *reinterpret_cast<uint16_t*>(p) = (uint16_t)eb.x;
            else *p = (uint8_t)eb.x;
        }
        if (a.mass && tid < kMoveRows && src_row[tid] >= 0) a.to_mass[d0 + tid] = w;
    }
    if (a.new_lens && (IN_PLACE || blockIdx.y == 0)) {
        // behind the moved rows: weights zero, so that rows appended there start from nothing
        __shared__ int s_kept;
        if (tid == 0) s_kept = 0;
        __syncthreads();
        int mine = 0;
        for (int i = tid; i < a.n_index; i += kMoveThreads) mine += idx[i] >= 0;
        if (mine) atomicAdd(&s_kept, mine);
        __syncthreads();
        const int kept = s_kept;
        for (int i = kept + tid; i < a.dst.max_seq; i += kMoveThreads) a.to_mass[dst0 + i] = 0.f;
        if (h == 0 && tid == 0) a.new_lens[b] = kept;
    }
}

kvbfp_status launch_move(const MoveArgs& a, cudaStream_t s) {
    const int64_t pairs = (int64_t)a.src.batch * a.src.n_kv_heads;
    const bool in_place = a.to[0] == a.from[0];
    const int chunks = (a.n_index + kMoveRows - 1) / kMoveRows;
    const dim3 grid((unsigned)pairs, in_place ? 1u : (unsigned)(chunks < 65535 ? chunks : 65535));
    const int pieces = a.src.mant_bits;      // 16-byte pieces: 128 p / 8 / 16 = p
    cudaError_t e;
    if (in_place)
        e = pieces == 4 ? launch_pdl(move_rows<true, 4>, grid, dim3(kMoveThreads), 0, s, a)
            : pieces == 6 ? launch_pdl(move_rows<true, 6>, grid, dim3(kMoveThreads), 0, s, a)
                          : launch_pdl(move_rows<true, 8>, grid, dim3(kMoveThreads), 0, s, a);
    else
        e = pieces == 4 ? launch_pdl(move_rows<false, 4>, grid, dim3(kMoveThreads), 0, s, a)
            : pieces == 6 ? launch_pdl(move_rows<false, 6>, grid, dim3(kMoveThreads), 0, s, a)
                          : launch_pdl(move_rows<false, 8>, grid, dim3(kMoveThreads), 0, s, a);
    KVBFP_CUDA(e);
    KVBFP_LAUNCH_CHECK("move_rows");
    return KVBFP_OK;
}

// Fills the caches of `a`; in place means the same four planes, anything else has to be apart.
kvbfp_status set_caches(const kvbfp_cache* src, const kvbfp_cache* dst, MoveArgs* a) {
    if (!src || !dst) return KVBFP_ERR_INVALID_ARG;
    kvbfp_status st = check_format(&src->fmt);
    if (st == KVBFP_OK) st = check_format(&dst->fmt);
    if (st != KVBFP_OK) return st;
    const kvbfp_format &f = src->fmt, &d = dst->fmt;
    if (f.batch != d.batch || f.n_kv_heads != d.n_kv_heads || f.block != d.block || f.mant_bits != d.mant_bits)
        return KVBFP_ERR_INVALID_ARG;
    if ((int64_t)f.batch * f.n_kv_heads >= (int64_t)1 << 28) return KVBFP_ERR_UNSUPPORTED;
    a->src = f;
    a->dst = d;
    const uint8_t* from[4] = {src->k_mant, src->k_exp, src->v_mant, src->v_exp};
    uint8_t* to[4] = {dst->k_mant, dst->k_exp, dst->v_mant, dst->v_exp};
    int same = 0;
    for (int i = 0; i < 4; ++i) {
        if (!from[i] || !to[i]) return KVBFP_ERR_INVALID_ARG;
        if (!aligned16(from[i]) || !aligned16(to[i])) return KVBFP_ERR_ALIGNMENT;
        a->from[i] = from[i];
        a->to[i] = to[i];
        same += from[i] == to[i];
    }
    if (same != 0 && (same != 4 || f.max_seq != d.max_seq)) return KVBFP_ERR_INVALID_ARG;
    const size_t pairs = (size_t)f.batch * f.n_kv_heads;
    for (int x = 0; x < 16 && same == 0; ++x) {        // different caches must not overlap, whichever planes
        const int i = x >> 2, j = x & 3;
        const size_t row_i = (i & 1) ? row_e_bytes(f) : row_m_bytes(f), row_j = (j & 1) ? row_e_bytes(f) : row_m_bytes(f);
        const uintptr_t s = (uintptr_t)from[i], t = (uintptr_t)to[j];
        if (s < t + pairs * d.max_seq * row_j && t < s + pairs * f.max_seq * row_i) return KVBFP_ERR_INVALID_ARG;
    }
    return KVBFP_OK;
}

}  // namespace
}  // namespace kvbfp

extern "C" kvbfp_status kvbfp_gather_rows(const kvbfp_cache* src, const kvbfp_cache* dst, const int32_t* index,
                                          int32_t index_heads, int32_t n_index, const int32_t* count,
                                          const int32_t* src_base, const int32_t* dst_base, void* stream) {
    using namespace kvbfp;
    MoveArgs a = {};
    if (!index || !count || n_index < 1) return KVBFP_ERR_INVALID_ARG;
    if (n_index > 1 << 30) return KVBFP_ERR_UNSUPPORTED;      // (move_rows counts in 32 bits, a chunk past the end)
    kvbfp_status st = set_caches(src, dst, &a);
    if (st != KVBFP_OK) return st;
    if (index_heads != 1 && index_heads != src->fmt.n_kv_heads) return KVBFP_ERR_INVALID_ARG;
    a.index = index; a.index_heads = index_heads; a.n_index = n_index; a.count = count;
    a.src_base = src_base; a.dst_base = dst_base;
    st = status_word(&a.status);
    if (st != KVBFP_OK) return st;
    return launch_move(a, (cudaStream_t)stream);
}

extern "C" kvbfp_status kvbfp_evict(const kvbfp_cache* src, const int32_t* seq_lens, const float* mass, int32_t budget,
                                    int32_t n_sink, int32_t n_recent, const kvbfp_cache* dst, float* dst_mass,
                                    int32_t* new_lens, int32_t* kept, void* stream) {
    using namespace kvbfp;
    MoveArgs a = {};
    if (!seq_lens || !mass || !dst_mass || !new_lens || !kept) return KVBFP_ERR_INVALID_ARG;
    if (budget < 1 || n_sink < 0 || n_recent < 0 || n_sink > budget || n_recent > budget - n_sink)
        return KVBFP_ERR_INVALID_ARG;
    kvbfp_status st = set_caches(src, dst, &a);
    if (st != KVBFP_OK) return st;
    if (budget > dst->fmt.max_seq) return KVBFP_ERR_CAPACITY;
    if (!aligned16(mass) || !aligned16(dst_mass) || !aligned16(kept)) return KVBFP_ERR_ALIGNMENT;
    if ((dst_mass == mass) != (a.from[0] == a.to[0])) return KVBFP_ERR_INVALID_ARG;
    const size_t pairs = (size_t)src->fmt.batch * src->fmt.n_kv_heads;
    const uintptr_t x = (uintptr_t)mass, y = (uintptr_t)dst_mass;
    if (x != y && x < y + pairs * dst->fmt.max_seq * 4 && y < x + pairs * src->fmt.max_seq * 4) return KVBFP_ERR_INVALID_ARG;
    st = status_word(&a.status);
    if (st != KVBFP_OK) return st;
    cudaStream_t s = (cudaStream_t)stream;
    // A cluster per pair where the pairs alone leave most of the GPU idle and a block would have several rows per thread
    // (8 x 65536 rows: 58 us with a block each); keys in registers where the longest sequence allowed fits.
    const kvbfp_format& f = src->fmt;
    int n_sm = 0;
    st = sm_count(&n_sm);
    if (st != KVBFP_OK) return st;
    const bool wide = (int64_t)f.batch * f.n_kv_heads * kSelCluster <= 2 * n_sm && f.max_seq > kSelThreads * 4;
    const bool cached = (int64_t)f.max_seq - n_sink - n_recent <= (int64_t)kSelThreads * kSelKeys * (wide ? kSelCluster : 1);
    auto select = wide ? (cached ? launch_select<kSelCluster, true> : launch_select<kSelCluster, false>)
                       : (cached ? launch_select<1, true> : launch_select<1, false>);
    st = select(mass, seq_lens, f, budget, n_sink, n_recent, kept, a.status, s);
    if (st != KVBFP_OK) return st;
    a.index = kept; a.index_heads = src->fmt.n_kv_heads; a.n_index = budget;
    a.mass = mass; a.to_mass = dst_mass; a.new_lens = new_lens;
    return launch_move(a, s);
}
