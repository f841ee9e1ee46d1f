// From the projections to the cache in one pass: norm of every query and key head, rotation, and the cast and write of
// kvbfp_append, for a ragged batch of new tokens, into a contiguous cache or pages.
//
//   y = x / sqrt(mean(x^2) + eps) * w ;  (y_a, y_b) -> (y_a cos - y_b sin, y_a sin + y_b cos), angle = position * theta[pair]
//
// A warp takes two neighbouring tokens, sixteen lanes each, and walks heads: queries, keys, values.  A lane holds four
// rotation pairs of its token's rows, so that sine and cosine are formed once per token (four a lane, in registers) and serve
// all heads, and no pair crosses lanes.  Rows come through a ring of shared-memory stages per warp that asynchronous copies
// fill some heads ahead.  Keys pass through shared memory once more for the permutation, then a lane owns eight stored slots and
// casts them as kvbfp_append does (sixteen lanes to a row).
//
// Codes of keys.  Values next to a rounding border fall on the side that fp32 errors pick, which would make the cache depend on
// the order of operations.  The error of a value is bounded by kErr times the magnitude of its pair; a row with a value (or
// block maximum) that close to a border is formed and cast again in fp64, four rows in a thousand (4 bits) to one in twenty (8
// bits).  So the codes are those of the formula.
//
// What bounds it: memory for whole prompts.  Bytes of a token: 2 (Hq + Hkv) es 128 ... read and written once.
#include <atomic>

#include "pages.cuh"
#include "ptx.cuh"
#include "umma.cuh"

namespace kvbfp {
namespace {

constexpr int kWWarps = 8;            // warps of a block, each on its own
__host__ __device__ constexpr int write_ring(int type_bytes) { return type_bytes == 2 ? 4 : 3; }      // heads in flight (48 KB a block)

struct WriteArgs {
    const void* src[3];               // q, k, v
    int64_t stride[3];                // elements from token to token
    void* q_out;
    uint8_t* mant[2];
    uint8_t* exp8[2];
    const int32_t* perm[2];
    const float* weight[2];           // of q, k
    const double* theta;
    const int32_t* starts;
    const int32_t* lens;
    TokenMap map;
    int heads[3];                     // of q, k, v; 0: not there
    int batch, n_tokens, head_chunk;
    float eps;
    uint32_t* status;
};

// fp32 error of a normalised and rotated value, relative to the sum of its pair's magnitudes (in units of 2^-24): the norm's
// factor and its two products 3, sine and cosine of an angle rounded once 4 (the angle is 3.14 at most: half a step is 2; the
// functions are good to 2), the product and the sum 2; rounded up.
constexpr float kErr = 10.f / 16777216.f;

// Squares summed in fp64: their sum's square root inverted to fp32's last bit by one step of Newton's from an fp32 start.
__device__ __forceinline__ float inv_rms64(double ss, float eps) {
    const double m = ss * (1.0 / kHeadDim) + (double)eps;
    const double i0 = (double)rsqrtf((float)m);
    const double i1 = i0 * (1.5 - 0.5 * m * i0 * i0);
    // outside fp32's range (or nothing to invert) the start is no start: the long way
    return (float)((m > 1e-30 && m < 1e30) ? i1 : 1.0 / sqrt(m));
}

template <int P, int N>
struct Cast {
    static constexpr int QMAX = (1 << (P - 1)) - 1, EXC = 1 << (P - 1), LANES = N / 8;
    static constexpr float MAGIC = 12582912.f + (float)EXC;            // 1.5 * 2^23 + 2^(p-1)
    static constexpr uint32_t MAGIC_BITS = 0x4B400000u;
};
// Writes a lane's eight fields (0 .. 2^P - 1) and, by the first lane of each block, the exponent byte.
template <int P, int N>
__device__ __forceinline__ void put_row(const uint32_t (&f)[8], int e8, uint8_t* mrow, uint8_t* erow, int sub) {
    if (P == 4) {
        uint32_t w = f[7];
#pragma unroll
        for (int i = 6; i >= 0; --i) w = w * 16u + f[i];
        reinterpret_cast<uint32_t*>(mrow)[sub] = w;
    } else if (P == 6) {
        uint64_t w = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) w |= (uint64_t)f[i] << (6 * i);
        uint16_t* o = reinterpret_cast<uint16_t*>(mrow + sub * 6);
        o[0] = (uint16_t)w;
        o[1] = (uint16_t)(w >> 16);
        o[2] = (uint16_t)(w >> 32);
    } else {
        uint32_t lo = 0, hi = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            lo |= f[i] << (8 * i);
            hi |= f[i + 4] << (8 * i);
        }
        reinterpret_cast<uint2*>(mrow)[sub] = make_uint2(lo, hi);
    }
    if ((sub % Cast<P, N>::LANES) == 0) erow[sub / Cast<P, N>::LANES] = (uint8_t)e8;
}
// Eight slots of a lane to fields; err: bound of each value's error.  True if a value or the block's maximum lies within its
// error of a border.
template <int P, int N, bool GUARD>
__device__ __forceinline__ bool cast32(const float (&v)[8], const float (&err)[8], uint32_t (&f)[8], int& e8, bool& finite) {
    using C = Cast<P, N>;
    uint32_t amax = 0;
    float worst = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        amax = max(amax, __float_as_uint(v[i]) & 0x7fffffffu);
        if (GUARD) worst = fmaxf(worst, err[i]);
    }
#pragma unroll
    for (int off = 1; off < C::LANES; off <<= 1) {
        amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, off));
        if (GUARD) worst = fmaxf(worst, __shfl_xor_sync(0xffffffffu, worst, off));
    }
    e8 = (int)(amax >> 23);
    finite = e8 != 255;
    if (!finite) e8 = 254;
    const int k = 127 - e8 + (P - 2), k1 = k >> 1, k2 = k - k1;
    const float s1 = pow2i(k1), s2 = pow2i(k2);
    bool near = false;
    if (GUARD) {
        const float top = __uint_as_float(amax);
        near = worst > 0.f && (__float_as_uint(top + worst) >> 23 != amax >> 23 || __float_as_uint(fmaxf(top - worst, 0.f)) >> 23 != amax >> 23);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float x = v[i] * s1;
        float r = fmaf(x, s2, C::MAGIC);                                              // to nearest, ties to even
        if (GUARD) near |= fabsf(fmaf(x, s2, C::MAGIC - r)) > 0.5f - err[i] * s1 * s2;
        r = fminf(fmaxf(r, C::MAGIC - (float)C::QMAX), C::MAGIC + (float)C::QMAX);    // NaN falls to the lower bound
        f[i] = __float_as_uint(r) - C::MAGIC_BITS;
    }
    return near;
}
// The same of values in fp64.
template <int P, int N>
__device__ __forceinline__ void cast64(const double (&v)[8], uint32_t (&f)[8], int& e8) {
    using C = Cast<P, N>;
    double amax = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = fmax(amax, fabs(v[i]));
#pragma unroll
    for (int off = 1; off < C::LANES; off <<= 1) amax = fmax(amax, __shfl_xor_sync(0xffffffffu, amax, off));
    const int e = (int)((uint64_t)__double_as_longlong(amax) >> 52) - 1023 + 127;
    e8 = min(max(e, 0), 254);
    const double up = __longlong_as_double((long long)(127 - e8 + (P - 2) + 1023) << 52);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const double r = fmin(fmax(rint(v[i] * up), -(double)C::QMAX), (double)C::QMAX);
        f[i] = (uint32_t)((int)r + C::EXC);
    }
}

// Four pairs of a key row in fp64 (a call: few rows come here).
__device__ __noinline__ void turn64(const float (&a)[4], const float (&b)[4], const float* wa, const float* wb, double inv,
                                    const double* theta, int pos, double (&ya)[4], double (&yb)[4]) {
#pragma unroll 1
    for (int j = 0; j < 4; ++j) {
        const double xa = (double)a[j] * inv * (wa ? (double)wa[j] : 1.0), xb = (double)b[j] * inv * (wb ? (double)wb[j] : 1.0);
        double sn = 0.0, cs = 1.0;
        if (theta) sincos((double)pos * theta[j], &sn, &cs);
        ya[j] = xa * cs - xb * sn;
        yb[j] = xa * sn + xb * cs;
    }
}

// HALF: pairs (i, i + 64), else (2i, 2i + 1).  A lane's pairs are 4 sub .. 4 sub + 3 in both.
template <bool HALF>
__device__ __forceinline__ int chan_a(int sub, int j) { return HALF ? 4 * sub + j : 8 * sub + 2 * j; }
template <bool HALF>
__device__ __forceinline__ int chan_b(int sub, int j) { return HALF ? 64 + 4 * sub + j : 8 * sub + 2 * j + 1; }

template <typename T, bool HALF>
__device__ __forceinline__ void read_pairs(const uint8_t* row, int sub, float (&a)[4], float (&b)[4]) {
    if (sizeof(T) == 2) {
        if (HALF) {
            const uint2 x = *reinterpret_cast<const uint2*>(row + 8 * sub), y = *reinterpret_cast<const uint2*>(row + 128 + 8 * sub);
            a[0] = __uint_as_float(x.x << 16); a[1] = __uint_as_float(x.x & 0xffff0000u);
            a[2] = __uint_as_float(x.y << 16); a[3] = __uint_as_float(x.y & 0xffff0000u);
            b[0] = __uint_as_float(y.x << 16); b[1] = __uint_as_float(y.x & 0xffff0000u);
            b[2] = __uint_as_float(y.y << 16); b[3] = __uint_as_float(y.y & 0xffff0000u);
        } else {
            const uint4 x = *reinterpret_cast<const uint4*>(row + 16 * sub);
            const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) { a[j] = __uint_as_float(w[j] << 16); b[j] = __uint_as_float(w[j] & 0xffff0000u); }
        }
    } else {
        const float4 x = *reinterpret_cast<const float4*>(row + (HALF ? 16 * sub : 32 * sub));
        const float4 y = *reinterpret_cast<const float4*>(row + (HALF ? 256 + 16 * sub : 32 * sub + 16));
        if (HALF) {
            a[0] = x.x; a[1] = x.y; a[2] = x.z; a[3] = x.w; b[0] = y.x; b[1] = y.y; b[2] = y.z; b[3] = y.w;
        } else {
            a[0] = x.x; b[0] = x.y; a[1] = x.z; b[1] = x.w; a[2] = y.x; b[2] = y.y; a[3] = y.z; b[3] = y.w;
        }
    }
}
template <typename T, bool HALF>
__device__ __forceinline__ void write_pairs(T* row, int sub, const float (&a)[4], const float (&b)[4]) {
    if (sizeof(T) == 2) {
        uint8_t* to = reinterpret_cast<uint8_t*>(row);
        if (HALF) {
            *reinterpret_cast<uint2*>(to + 8 * sub) = make_uint2(pack_bf16x2_rn(a[0], a[1]), pack_bf16x2_rn(a[2], a[3]));
            *reinterpret_cast<uint2*>(to + 128 + 8 * sub) = make_uint2(pack_bf16x2_rn(b[0], b[1]), pack_bf16x2_rn(b[2], b[3]));
        } else {
            *reinterpret_cast<uint4*>(to + 16 * sub) = make_uint4(pack_bf16x2_rn(a[0], b[0]), pack_bf16x2_rn(a[1], b[1]),
                                                                  pack_bf16x2_rn(a[2], b[2]), pack_bf16x2_rn(a[3], b[3]));
        }
    } else {
        float* to = reinterpret_cast<float*>(row);
        if (HALF) {
            *reinterpret_cast<float4*>(to + 4 * sub) = make_float4(a[0], a[1], a[2], a[3]);
            *reinterpret_cast<float4*>(to + 64 + 4 * sub) = make_float4(b[0], b[1], b[2], b[3]);
        } else {
            *reinterpret_cast<float4*>(to + 8 * sub) = make_float4(a[0], b[0], a[1], b[1]);
            *reinterpret_cast<float4*>(to + 8 * sub + 4) = make_float4(a[2], b[2], a[3], b[3]);
        }
    }
}

template <int P, int N, typename T, bool HALF>
__global__ void __launch_bounds__(kWWarps * 32) norm_rope_append(const WriteArgs a) {
    constexpr int D = kHeadDim, ROW_M = D * P / 8, ROW_E = D / N, ROW_IN = D * (int)sizeof(T), RING = write_ring(sizeof(T));
    constexpr int PARK = 2 * D + 4;             // floats of a parked row (value and error bound, or fp64 values), off the other's banks
    __shared__ __align__(16) uint8_t ring[kWWarps][RING][2][ROW_IN];
    __shared__ __align__(16) float park[kWWarps][2][PARK];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane & 15, grp = lane >> 4;
    pdl_wait();
    pdl_trigger();
    // the warp's unit: two tokens, a run of heads
    const int n_heads = a.heads[0] + a.heads[1] + a.heads[2];
    const int h0 = blockIdx.y * a.head_chunk, h1 = min(n_heads, h0 + a.head_chunk);
    const int tok = 2 * (blockIdx.x * kWWarps + warp) + grp;
    const int first = min(max(a.starts[0], 0), a.n_tokens), end = min(max(a.starts[a.batch], 0), a.n_tokens);
    const bool live = tok < end && tok >= first;
    if (__all_sync(0xffffffffu, !live)) return;

    auto source = [&](int h) -> const T* {
        int s = 0;
        if (h >= a.heads[0]) {
            s = 1;
            h -= a.heads[0];
            if (h >= a.heads[1]) {
                s = 2;
                h -= a.heads[1];
            }
        }
        const T* base = static_cast<const T*>(s == 0 ? a.src[0] : s == 1 ? a.src[1] : a.src[2]);
        const int64_t stride = s == 0 ? a.stride[0] : s == 1 ? a.stride[1] : a.stride[2];
        return base + (int64_t)tok * stride + h * D;
    };
    const uint32_t my_ring = smem_u32(&ring[warp][0][grp][0]);
    auto issue = [&](int h) {
        if (h < h1 && live) {
            const uint4* p = reinterpret_cast<const uint4*>(source(h)) + sub;
            const uint32_t dst = my_ring + ((h - h0) % RING) * (2 * ROW_IN) + 16 * sub;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(p) : "memory");
            if (sizeof(T) == 4) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + 256), "l"(p + 16) : "memory");
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < RING; ++i) issue(h0 + i);

    // ---- sequence and position: the last sequence that starts at or before the token
    int b = 0;
    {
        const int t0 = __shfl_sync(0xffffffffu, tok, 0), t1 = __shfl_sync(0xffffffffu, tok, 16);
        int n0 = 0, n1 = 0;
        for (int i = 0; i < a.batch; i += 32) {
            const int s = i + lane < a.batch ? a.starts[i + lane] : 0x7fffffff;
            n0 += __popc(__ballot_sync(0xffffffffu, s <= t0));
            n1 += __popc(__ballot_sync(0xffffffffu, s <= t1));
        }
        b = min(max((grp ? n1 : n0) - 1, 0), a.batch - 1);
    }
    const int len = a.lens[b], pos = len - min(max(a.starts[b + 1], 0), a.n_tokens) + tok;
    int64_t row0 = 0;             // row of head 0; heads follow map.rows rows on
    bool stored = live && pos >= 0 && pos < a.map.cap;
    if (stored) {
        const int pg = token_page(a.map, b, pos);
        stored = pg >= 0;
        row0 = (int64_t)max(pg, 0) * a.map.n_heads * a.map.rows + token_row(a.map, pos);
    }
    if (live && !stored && sub == 0 && blockIdx.y == 0 && a.heads[1]) raise_flag(a.status, KVBFP_FLAG_POSITION);

    float cs[4], sn[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        cs[j] = 1.f;
        sn[j] = 0.f;
        if (a.theta && h0 < a.heads[0] + a.heads[1]) sincos_reduced((double)pos * a.theta[4 * sub + j], &sn[j], &cs[j]);
    }
    float wa[4], wb[4];
    auto weights = [&](const float* w) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            wa[j] = w ? w[chan_a<HALF>(sub, j)] : 1.f;
            wb[j] = w ? w[chan_b<HALF>(sub, j)] : 1.f;
        }
    };
    weights(h0 < a.heads[0] ? a.weight[0] : a.weight[1]);
    float* mine = &park[warp][grp][0];

    for (int h = h0; h < h1; ++h) {
        asm volatile("cp.async.wait_group %0;" ::"n"(RING - 1) : "memory");
        __syncwarp();
        const uint8_t* row = &ring[warp][(h - h0) % RING][grp][0];
        const int kind = h < a.heads[0] ? 0 : h < a.heads[0] + a.heads[1] ? 1 : 2;
        const int head = h - (kind == 0 ? 0 : kind == 1 ? a.heads[0] : a.heads[0] + a.heads[1]);
        if (h == a.heads[0] && h != h0) weights(a.weight[1]);
        float xa[4], xb[4];
        if (kind == 0) {
            read_pairs<T, HALF>(row, sub, xa, xb);
            __syncwarp();
            issue(h + RING);
            if (a.weight[0]) {
                float ss = 0.f;
#pragma unroll
                for (int j = 0; j < 4; ++j) ss = fmaf(xa[j], xa[j], fmaf(xb[j], xb[j], ss));
#pragma unroll
                for (int off = 8; off; off >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, off);
                const float inv = rsqrtf(fmaf(ss, 1.f / D, a.eps));
#pragma unroll
                for (int j = 0; j < 4; ++j) { xa[j] = xa[j] * inv * wa[j]; xb[j] = xb[j] * inv * wb[j]; }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float y = fmaf(xa[j], cs[j], -(xb[j] * sn[j]));
                xb[j] = fmaf(xb[j], cs[j], xa[j] * sn[j]);
                xa[j] = y;
            }
            if (live) write_pairs<T, HALF>(static_cast<T*>(a.q_out) + ((int64_t)tok * a.heads[0] + head) * D, sub, xa, xb);
            continue;
        }
        uint8_t* mrow = a.mant[kind - 1] + (row0 + (int64_t)head * a.map.rows) * ROW_M;
        uint8_t* erow = a.exp8[kind - 1] + (row0 + (int64_t)head * a.map.rows) * ROW_E;
        const int32_t* perm = kind == 1 ? a.perm[0] : a.perm[1];
        int at[8];
        if (perm) {
            const int4* pp = reinterpret_cast<const int4*>(perm + head * D + sub * 8);
            const int4 p0 = __ldg(pp), p1 = __ldg(pp + 1);
            at[0] = p0.x & (D - 1); at[1] = p0.y & (D - 1); at[2] = p0.z & (D - 1); at[3] = p0.w & (D - 1);
            at[4] = p1.x & (D - 1); at[5] = p1.y & (D - 1); at[6] = p1.z & (D - 1); at[7] = p1.w & (D - 1);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) at[i] = sub * 8 + i;
        }
        float v[8], err[8];
        uint32_t f[8];
        int e8;
        bool finite;
        if (kind == 2) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                v[i] = sizeof(T) == 2 ? __uint_as_float((uint32_t)reinterpret_cast<const unsigned short*>(row)[at[i]] << 16)
                                      : reinterpret_cast<const float*>(row)[at[i]];
            __syncwarp();
            issue(h + RING);
            (void)cast32<P, N, false>(v, v, f, e8, finite);
        } else {
            read_pairs<T, HALF>(row, sub, xa, xb);
            __syncwarp();
            issue(h + RING);
            double ss = 0.0;
            float inv = 1.f;
            if (a.weight[1]) {
#pragma unroll
                for (int j = 0; j < 4; ++j) ss = fma((double)xa[j], (double)xa[j], fma((double)xb[j], (double)xb[j], ss));
#pragma unroll
                for (int off = 8; off; off >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, off);
                inv = inv_rms64(ss, a.eps);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float ya = xa[j] * inv * wa[j], yb = xb[j] * inv * wb[j];
                const float e = (a.weight[1] || a.theta) ? kErr * (fabsf(ya) + fabsf(yb)) : 0.f;
                *reinterpret_cast<float2*>(mine + 2 * chan_a<HALF>(sub, j)) = make_float2(fmaf(ya, cs[j], -(yb * sn[j])), e);
                *reinterpret_cast<float2*>(mine + 2 * chan_b<HALF>(sub, j)) = make_float2(fmaf(yb, cs[j], ya * sn[j]), e);
            }
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float2 x = *reinterpret_cast<const float2*>(mine + 2 * at[i]);
                v[i] = x.x;
                err[i] = x.y;
            }
            __syncwarp();
            const bool near = cast32<P, N, true>(v, err, f, e8, finite);
            if (__any_sync(0xffffffffu, near && finite && stored)) {
                double ya[4], yb[4], inv64 = 1.0;
                if (a.weight[1]) inv64 = 1.0 / sqrt(ss * (1.0 / D) + (double)a.eps);
                turn64(xa, xb, a.weight[1] ? wa : nullptr, a.weight[1] ? wb : nullptr, inv64, a.theta ? a.theta + 4 * sub : nullptr, pos, ya, yb);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    *reinterpret_cast<double*>(mine + 2 * chan_a<HALF>(sub, j)) = ya[j];
                    *reinterpret_cast<double*>(mine + 2 * chan_b<HALF>(sub, j)) = yb[j];
                }
                __syncwarp();
                double w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = *reinterpret_cast<const double*>(mine + 2 * at[i]);
                __syncwarp();
                uint32_t f64[8];
                int e64;
                cast64<P, N>(w, f64, e64);
                if (finite) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) f[i] = f64[i];
                    e8 = e64;
                }
            }
        }
        if (live && !finite) raise_flag(a.status, KVBFP_FLAG_NONFINITE);
        if (stored) put_row<P, N>(f, e8, mrow, erow, sub);
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
}

template <int P, int N, typename T, bool HALF>
kvbfp_status launch_write(WriteArgs a, cudaStream_t s) {
    int n_sm = 0;
    const kvbfp_status st = sm_count(&n_sm);
    if (st != KVBFP_OK) return st;
    const int n_heads = a.heads[0] + a.heads[1] + a.heads[2];
    const int64_t pairs = ((int64_t)a.n_tokens + 1) / 2, gx = (pairs + kWWarps - 1) / kWWarps;
    // few tokens: heads spread over the blocks too, down to one head a warp
    int64_t chunks = (int64_t)n_sm * 4 / gx;
    if (chunks < 1) chunks = 1;
    if (chunks > n_heads) chunks = n_heads;
    a.head_chunk = (int)((n_heads + chunks - 1) / chunks);
    const dim3 grid((unsigned)gx, (unsigned)((n_heads + a.head_chunk - 1) / a.head_chunk));
    KVBFP_CUDA(launch_pdl(norm_rope_append<P, N, T, HALF>, grid, dim3(kWWarps * 32), 0, s, a));
    KVBFP_LAUNCH_CHECK("norm_rope_append");
    return KVBFP_OK;
}

template <int P, int N>
kvbfp_status launch_type(const WriteArgs& a, bool bf16, bool half, cudaStream_t s) {
    if (bf16) return half ? launch_write<P, N, __nv_bfloat16, true>(a, s) : launch_write<P, N, __nv_bfloat16, false>(a, s);
    return half ? launch_write<P, N, float, true>(a, s) : launch_write<P, N, float, false>(a, s);
}
template <int P>
kvbfp_status launch_block(int n, const WriteArgs& a, bool bf16, bool half, cudaStream_t s) {
    switch (n) {
        case 16: return launch_type<P, 16>(a, bf16, half, s);
        case 32: return launch_type<P, 32>(a, bf16, half, s);
        case 64: return launch_type<P, 64>(a, bf16, half, s);
        case 128: return launch_type<P, 128>(a, bf16, half, s);
    }
    return KVBFP_ERR_UNSUPPORTED;
}

}  // namespace
}  // namespace kvbfp

extern "C" kvbfp_status kvbfp_norm_rope_append(const kvbfp_cache* cache, const kvbfp_pages* pages, const void* q, int64_t q_stride,
                                               const void* k, int64_t k_stride, const void* v, int64_t v_stride, kvbfp_dtype dt,
                                               int32_t n_q_heads, int32_t n_tokens, const int32_t* starts, const int32_t* seq_lens,
                                               const float* q_weight, const float* k_weight, float eps, const double* theta,
                                               int32_t half_split, const int32_t* perm_k, const int32_t* perm_v, void* q_out,
                                               void* stream) {
    using namespace kvbfp;
    if (!cache) return KVBFP_ERR_INVALID_ARG;
    const kvbfp_format& f = cache->fmt;
    kvbfp_status st = check_format(&f);
    if (st == KVBFP_OK && pages) st = check_pool(f, pages);
    if (st != KVBFP_OK) return st;
    if ((!q && !k) || (k == nullptr) != (v == nullptr) || (q == nullptr) != (q_out == nullptr) || !starts || !seq_lens) return KVBFP_ERR_INVALID_ARG;
    if (k && (!cache->k_mant || !cache->k_exp || !cache->v_mant || !cache->v_exp)) return KVBFP_ERR_INVALID_ARG;
    if (dt != KVBFP_F32 && dt != KVBFP_BF16) return KVBFP_ERR_INVALID_ARG;
    if (n_tokens < 0 || !(eps >= 0.f) || eps > 3e38f) return KVBFP_ERR_INVALID_ARG;
    if (q && n_q_heads < 1) return KVBFP_ERR_INVALID_ARG;
    if (n_q_heads > 4096 || f.n_kv_heads > 4096 || n_tokens > 1 << 26) return KVBFP_ERR_UNSUPPORTED;
    const size_t es = dt == KVBFP_F32 ? 4 : 2;
    const int64_t kv_width = (int64_t)f.n_kv_heads * kHeadDim, q_width = (int64_t)n_q_heads * kHeadDim;
    const void* ptrs[] = {q, k, v, q_out, cache->k_mant, cache->k_exp, cache->v_mant, cache->v_exp, perm_k, perm_v};
    for (const void* p : ptrs)
        if (p && !aligned16(p)) return KVBFP_ERR_ALIGNMENT;
    if (((uintptr_t)theta & 7) || ((uintptr_t)q_weight & 3) || ((uintptr_t)k_weight & 3)) return KVBFP_ERR_ALIGNMENT;
    const void* src[3] = {q, k, v};
    const int64_t stride[3] = {q_stride, k_stride, v_stride};
    for (int i = 0; i < 3; ++i) {
        if (!src[i]) continue;
        if (stride[i] < (i ? kv_width : q_width) || stride[i] > (int64_t)1 << 40) return KVBFP_ERR_INVALID_ARG;
        if (stride[i] * es % 16) return KVBFP_ERR_ALIGNMENT;
    }
    if (n_tokens == 0) return KVBFP_OK;
    if (q) {        // the output is apart from what is read, or q itself
        const uintptr_t o = (uintptr_t)q_out, oe = o + (size_t)n_tokens * q_width * es;
        for (int i = 0; i < 3; ++i) {
            if (!src[i]) continue;
            const uintptr_t x = (uintptr_t)src[i], xe = x + ((size_t)(n_tokens - 1) * stride[i] + (i ? kv_width : q_width)) * es;
            if (x < oe && o < xe && !(i == 0 && x == o && stride[0] == q_width)) return KVBFP_ERR_INVALID_ARG;
        }
    }
    WriteArgs a = {};
    for (int i = 0; i < 3; ++i) {
        a.src[i] = src[i];
        a.stride[i] = stride[i];
    }
    a.q_out = q_out;
    a.mant[0] = cache->k_mant; a.mant[1] = cache->v_mant;
    a.exp8[0] = cache->k_exp; a.exp8[1] = cache->v_exp;
    a.perm[0] = perm_k; a.perm[1] = perm_v;
    a.weight[0] = q_weight; a.weight[1] = k_weight;
    a.theta = theta;
    a.starts = starts; a.lens = seq_lens;
    a.map = token_map(f, pages);
    a.heads[0] = q ? n_q_heads : 0;
    a.heads[1] = a.heads[2] = k ? f.n_kv_heads : 0;
    a.batch = pages ? pages->batch : f.batch;
    a.n_tokens = n_tokens;
    a.eps = eps;
    st = status_word(&a.status);
    if (st != KVBFP_OK) return st;
    cudaStream_t s = (cudaStream_t)stream;
    const bool bf16 = dt == KVBFP_BF16, half = half_split != 0;
    switch (f.mant_bits) {
        case 4: return launch_block<4>(f.block, a, bf16, half, s);
        case 6: return launch_block<6>(f.block, a, bf16, half, s);
        case 8: return launch_block<8>(f.block, a, bf16, half, s);
    }
    return KVBFP_ERR_UNSUPPORTED;
}
