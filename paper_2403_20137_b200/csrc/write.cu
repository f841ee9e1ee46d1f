// From the projections to the cache in one pass: norm of every query and key head, rotation, and the cast and write of
// kvbfp_append, for a ragged batch of new tokens, into a contiguous cache or pages.
//
//   y = x / sqrt(mean(x^2) + eps) * w ;  (y_a, y_b) -> (y_a cos - y_b sin, y_a sin + y_b cos), angle = position * theta[pair]
//
// A warp takes two neighbouring tokens, sixteen lanes each, and walks heads: queries, keys, values.  A lane holds four
// rotation pairs of its token's rows, so that sine and cosine are formed once per token (four a lane, in registers, times the
// norm's weights) and serve all heads, and no pair crosses lanes.  The rows of the next heads are on their way while the ones
// before are worked on (they pass through registers only: a ring of shared-memory stages cost more instructions than its
// asynchronous copies hid).  Keys, and values with a permutation, are parked in shared memory and picked up slot by slot; then a
// lane owns eight stored slots and casts them as kvbfp_append does (sixteen lanes to a row).
//
// Codes of keys.  Values next to a rounding border fall on the side that fp32 errors pick, which would make the cache depend on
// the order of operations.  The error of a value is bounded by kErr times the magnitude of its pair (and kErrLow); a row with a value (or
// block maximum) that close to a border is formed and cast again in fp64.  (By arithmetic about one row of random keys in 800
// at 4 bits, in 50 at 8: 128 slots, twice a bound of some 5e-6 of the distance of borders, or 16 times that.)  So the codes are
// those of the formula.
//
// What bounds it: instructions (issue slots 60 % busy while blocks run, 54 % over the launch), most of them in the casts, and the
// parking of keys (shared-memory data pipe 58 %; memory 44 %).  Four ragged prompts of up to 8192 tokens, 32 query and 8 kv heads, 4
// bits, two runs of heads a token: 121 us, floor 71.
#include <atomic>

#include "pages.cuh"
#include "ptx.cuh"
#include "umma.cuh"

namespace kvbfp {
namespace {

constexpr int kWWarps = 8;            // warps of a block, each on its own

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
// factor 9 (squares summed in ten roundings, halved by the square root; the function itself 4), its product 1, sine and cosine of
// an angle rounded once 4 (the angle is 3.14 at most: half a step is 2; the functions are good to 2), their product with the
// weight 1, the product and the sum 2; rows beyond 2^126, whose factor is a subnormal number, 4 more; rounded up.  kErrLow: what
// results in the subnormal range add, half a step of 2^-149 each: two products and their sum, and where the weights are that small
// two entries of the table, times normalised values of 11.4 at most (the square root of 128).
constexpr float kErr = 22.f / 16777216.f, kErrLow = 0x1p-145f;

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
// Eight bf16 numbers of a lane, in pairs, cast and written as pairs (as in append_rows: everything the cast does to a bf16
// number stays inside bf16).  4 bits: pair j is slots j and j + 4, 6 bits: 2 j and 2 j + 1.  Returns whether all are finite.
template <int P, int N>
__device__ __forceinline__ bool cast_bf16(uint32_t (&f)[4], bool stored, uint8_t* mrow, uint8_t* erow, int sub) {
    using C = Cast<P, N>;
    auto top2 = [](uint32_t a, uint32_t b) { uint32_t d; asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b)); return d; };
    uint32_t m = top2(top2(f[0] & 0x7fff7fffu, f[1] & 0x7fff7fffu), top2(f[2] & 0x7fff7fffu, f[3] & 0x7fff7fffu));
#pragma unroll
    for (int off = 1; off < C::LANES; off <<= 1) m = top2(m, __shfl_xor_sync(0xffffffffu, m, off));
    int e8 = (int)(max(m & 0xffffu, m >> 16) >> 7);
    const bool finite = e8 != 255;
    if (!finite) e8 = 254;
    const int k = 127 - e8 + (P - 2), k1 = k >> 1, k2 = k - k1;
    constexpr uint32_t BASE = 0x43404340u;                       // bf16 192.0 twice
    constexpr uint32_t MAGIC = BASE + C::EXC * 0x10001u, LO = MAGIC - C::QMAX * 0x10001u, HI = MAGIC + C::QMAX * 0x10001u;
    const uint32_t s1 = ((uint32_t)(k1 + 127) << 7) * 0x10001u, s2 = ((uint32_t)(k2 + 127) << 7) * 0x10001u;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        f[j] = fma_bf16x2(mul_bf16x2(f[j], s1), s2, MAGIC);
        asm("max.bf16x2 %0, %0, %1;" : "+r"(f[j]) : "r"(LO));    // (a NaN falls to the lower bound)
        asm("min.bf16x2 %0, %0, %1;" : "+r"(f[j]) : "r"(HI));
    }
    if (!stored) return finite;
    if (P == 4) {
        reinterpret_cast<uint32_t*>(mrow)[sub] = ((f[3] * 16u + f[2]) * 16u + f[1]) * 16u + f[0] - BASE * 0x1111u;
    } else {
        uint32_t t[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t c = f[j] - BASE;
            t[j] = (c | (c >> 10)) & 0xfffu;
        }
        const uint32_t lo = t[0] + (t[1] << 12) + (t[2] << 24), hi = (t[2] >> 8) + (t[3] << 4);
        uint16_t* o = reinterpret_cast<uint16_t*>(mrow + sub * 6);
        o[0] = (uint16_t)lo;
        o[1] = (uint16_t)(lo >> 16);
        o[2] = (uint16_t)hi;
    }
    if ((sub % C::LANES) == 0) erow[sub / C::LANES] = (uint8_t)e8;
    return finite;
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
__device__ __noinline__ void turn64(const float (&a)[4], const float (&b)[4], const float (&wa)[4], const float (&wb)[4], double inv,
                                    const double* theta, int pos, double (&ya)[4], double (&yb)[4]) {
#pragma unroll 1
    for (int j = 0; j < 4; ++j) {
        const double xa = (double)a[j] * inv * (double)wa[j], xb = (double)b[j] * inv * (double)wb[j];
        double sn = 0.0, cs = 1.0;
        if (theta) sincos((double)pos * theta[j], &sn, &cs);
        ya[j] = xa * cs - xb * sn;
        yb[j] = xa * sn + xb * cs;
    }
}

// 1 / sqrt(mean(x^2) + eps) of a row that sixteen lanes hold (the whole warp calls).
__device__ __forceinline__ float inv_rms(const F2 (&xa)[2], const F2 (&xb)[2], float eps) {
    auto squares = [&](F2 a0, F2 a1, F2 b0, F2 b1) {
        float s0, s1;
        f2_split(f2_fma(a0, a0, f2_fma(a1, a1, f2_fma(b0, b0, f2_mul(b1, b1)))), s0, s1);
        float ss = s0 + s1;
#pragma unroll
        for (int off = 8; off; off >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, off);
        return ss;
    };
    float ss = squares(xa[0], xa[1], xb[0], xb[1]), mean = fmaf(ss, 1.f / kHeadDim, eps), up = 1.f;
    if (__any_sync(0xffffffffu, !(mean >= 1e-30f && ss <= 1e37f))) {      // squares leave the range of fp32, or lose bits below it
        up = !(ss <= 1e37f) ? 0x1p-100f : mean >= 1e-30f ? 1.f : 0x1p100f;
        const F2 s2 = f2(up, up);
        ss = squares(f2_mul(xa[0], s2), f2_mul(xa[1], s2), f2_mul(xb[0], s2), f2_mul(xb[1], s2));
        mean = fmaf(ss, 1.f / kHeadDim, eps * up * up);
    }
    return up * rsqrtf(mean);
}

// HALF: pairs (i, i + 64), else (2i, 2i + 1).  A lane's pairs are 4 sub .. 4 sub + 3 in both.
template <bool HALF>
__device__ __forceinline__ int chan_a(int sub, int j) { return HALF ? 4 * sub + j : 8 * sub + 2 * j; }
template <bool HALF>
__device__ __forceinline__ int chan_b(int sub, int j) { return HALF ? 64 + 4 * sub + j : 8 * sub + 2 * j + 1; }

// A lane's share of a row: two runs of four channels (HALF) or eight channels, and the pairs in it.
template <typename T>
struct Share {
    uint32_t w[2 * sizeof(T)];
};
template <typename T, bool HALF>
__device__ __forceinline__ Share<T> load_share(const T* row, int sub) {
    Share<T> x;
    const uint8_t* p = reinterpret_cast<const uint8_t*>(row);
    if (sizeof(T) == 2) {
        if (HALF) {
            const uint2 a = *reinterpret_cast<const uint2*>(p + 8 * sub), b = *reinterpret_cast<const uint2*>(p + 128 + 8 * sub);
            x.w[0] = a.x; x.w[1] = a.y; x.w[2] = b.x; x.w[3] = b.y;
        } else {
            const uint4 a = *reinterpret_cast<const uint4*>(p + 16 * sub);
            x.w[0] = a.x; x.w[1] = a.y; x.w[2] = a.z; x.w[3] = a.w;
        }
    } else {
        const uint4 a = *reinterpret_cast<const uint4*>(p + (HALF ? 16 * sub : 32 * sub)), b = *reinterpret_cast<const uint4*>(p + (HALF ? 256 + 16 * sub : 32 * sub + 16));
        x.w[0] = a.x; x.w[1] = a.y; x.w[2] = a.z; x.w[3] = a.w;
        x.w[(4) % (2 * sizeof(T))] = b.x; x.w[5 % (2 * sizeof(T))] = b.y; x.w[6 % (2 * sizeof(T))] = b.z; x.w[7 % (2 * sizeof(T))] = b.w;
    }
    return x;
}
// The eight numbers of a share in memory order.
template <typename T>
__device__ __forceinline__ void share_values(const Share<T>& x, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
        v[i] = sizeof(T) == 4 ? __uint_as_float(x.w[i % (2 * sizeof(T))]) : (i & 1) ? __uint_as_float(x.w[i / 2] & 0xffff0000u) : __uint_as_float(x.w[i / 2] << 16);
}
// Its pairs, two by two: a[j] = pairs 2 j and 2 j + 1.
template <typename T, bool HALF>
__device__ __forceinline__ void share_pairs(const Share<T>& x, F2 (&a)[2], F2 (&b)[2]) {
    float v[8];
    share_values<T>(x, v);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        a[j] = HALF ? f2(v[2 * j], v[2 * j + 1]) : f2(v[4 * j], v[4 * j + 2]);
        b[j] = HALF ? f2(v[4 + 2 * j], v[4 + 2 * j + 1]) : f2(v[4 * j + 1], v[4 * j + 3]);
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

__device__ __forceinline__ int clamped_start(const WriteArgs& a, int b) { return min(max(a.starts[b], 0), a.n_tokens); }

template <int P, int N, typename T, bool HALF>
__global__ void __launch_bounds__(kWWarps * 32, 3) norm_rope_append(const WriteArgs a) {
    constexpr int D = kHeadDim, ROW_M = D * P / 8, ROW_E = D / N;
    constexpr int QB = sizeof(T) == 2 ? 4 : 2, KB = 2;          // query (key, value) rows of a lane under way
    constexpr int PARK = 2 * D + 8;             // floats of a parked row (value and error bound, or fp64 values), off the other's banks
    __shared__ __align__(16) float park[kWWarps][2][PARK];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane & 15, grp = lane >> 4;
    pdl_wait();
    pdl_trigger();
    // the warp's unit: two tokens, a run of heads
    const int hq = a.heads[0], hk = a.heads[1], n_heads = hq + 2 * hk;
    const int h0 = blockIdx.y * a.head_chunk, h1 = min(n_heads, h0 + a.head_chunk);
    const int tok = 2 * (blockIdx.x * kWWarps + warp) + grp;
    const int first = clamped_start(a, 0), end = clamped_start(a, a.batch);
    const bool live = tok < end && tok >= first;
    // Starts that decrease leave nothing to do: which sequence a token belongs to is not known.
    if (__all_sync(0xffffffffu, !live)) {
        if (blockIdx.x + blockIdx.y + warp > 0) return;
        bool back = false;
        for (int i = lane; i < a.batch; i += 32) back |= clamped_start(a, i + 1) < clamped_start(a, i);
        if (back) raise_flag(a.status, KVBFP_FLAG_POSITION);
        return;
    }

    // heads of each kind in the run, and its first rows on their way
    const int q0 = min(h0, hq), q1 = min(h1, hq), k0 = min(max(h0 - hq, 0), hk), k1 = min(max(h1 - hq, 0), hk);
    const int v0 = max(h0 - hq - hk, 0), v1 = max(h1 - hq - hk, 0);
    const int at = live ? tok : max(first, min(tok, end - 1));           // (a token that exists: read, but not used)
    const T* q_in = static_cast<const T*>(a.src[0]) + (int64_t)at * a.stride[0] + q0 * D;
    const T* k_in = static_cast<const T*>(a.src[1]) + (int64_t)at * a.stride[1] + k0 * D;
    const T* v_in = static_cast<const T*>(a.src[2]) + (int64_t)at * a.stride[2] + v0 * D;
    Share<T> qx[QB];
#pragma unroll
    for (int i = 0; i < QB; ++i)
        if (q0 + i < q1) qx[i] = load_share<T, HALF>(q_in + i * D, sub);

    // ---- sequence and position: the last sequence that starts at or before the token
    int b = 0;
    {
        const int t0 = __shfl_sync(0xffffffffu, tok, 0), t1 = __shfl_sync(0xffffffffu, tok, 16);
        int n0 = 0, n1 = 0;
        bool back = false;
        for (int i = 0; i < a.batch; i += 32) {
            const int s = i + lane < a.batch ? clamped_start(a, i + lane) : 0x7fffffff;
            if (i + lane < a.batch) back |= clamped_start(a, i + lane + 1) < s;
            n0 += __popc(__ballot_sync(0xffffffffu, s <= t0));
            n1 += __popc(__ballot_sync(0xffffffffu, s <= t1));
        }
        if (__any_sync(0xffffffffu, back)) {
            if (lane == 0) raise_flag(a.status, KVBFP_FLAG_POSITION);
            return;
        }
        b = min(max((grp ? n1 : n0) - 1, 0), a.batch - 1);
    }
    const int len = a.lens[b], pos = len - clamped_start(a, b + 1) + tok;
    int64_t row0 = 0;             // row of head 0; heads follow map.rows rows on
    bool stored = live && pos >= 0 && pos < a.map.cap;
    if (stored) {
        const int pg = token_page(a.map, b, pos);
        stored = pg >= 0;
        row0 = (int64_t)max(pg, 0) * a.map.n_heads * a.map.rows + token_row(a.map, pos);
    }
    if (live && !stored && sub == 0 && blockIdx.y == 0 && hk) raise_flag(a.status, KVBFP_FLAG_POSITION);

    F2 cs[2], sn[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        float c[2] = {1.f, 1.f}, n[2] = {0.f, 0.f};
#pragma unroll
        for (int e = 0; e < 2; ++e)
            if (a.theta && h0 < hq + hk) sincos_reduced((double)pos * a.theta[4 * sub + 2 * j + e], &n[e], &c[e]);
        cs[j] = f2(c[0], c[1]);
        sn[j] = f2(n[0], n[1]);
    }
    // rotation with the norm's weights in it: y_a = x_a ac - x_b bs, y_b = x_b bc + x_a as
    F2 wa[2], wb[2], ac[2], as[2], bc[2], bs[2];
    auto tables = [&](const float* w) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            wa[j] = wb[j] = f2(1.f, 1.f);
            if (w) {
                wa[j] = f2(w[chan_a<HALF>(sub, 2 * j)], w[chan_a<HALF>(sub, 2 * j + 1)]);
                wb[j] = f2(w[chan_b<HALF>(sub, 2 * j)], w[chan_b<HALF>(sub, 2 * j + 1)]);
            }
            ac[j] = f2_mul(wa[j], cs[j]);
            as[j] = f2_mul(wa[j], sn[j]);
            bc[j] = f2_mul(wb[j], cs[j]);
            bs[j] = f2_mul(wb[j], f2_mul(sn[j], f2(-1.f, -1.f)));
        }
    };
    // ---- queries
    if (q0 < q1) {
        tables(a.weight[0]);
        T* out = static_cast<T*>(a.q_out) + ((int64_t)tok * hq + q0) * D;
        for (int h = q0; h < q1; h += QB) {
            Share<T> next[QB];
            q_in += QB * D;
#pragma unroll
            for (int i = 0; i < QB; ++i)
                if (h + QB + i < q1) next[i] = load_share<T, HALF>(q_in + i * D, sub);
#pragma unroll
            for (int i = 0; i < QB; ++i) {
                if (h + i >= q1) break;
                F2 xa[2], xb[2];
                share_pairs<T, HALF>(qx[i], xa, xb);
                if (a.weight[0]) {
                    const float inv = inv_rms(xa, xb, a.eps);
                    const F2 inv2 = f2(inv, inv);
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        xa[j] = f2_mul(xa[j], inv2);
                        xb[j] = f2_mul(xb[j], inv2);
                    }
                }
                float ya[4], yb[4];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    f2_split(f2_fma(xa[j], ac[j], f2_mul(xb[j], bs[j])), ya[2 * j], ya[2 * j + 1]);
                    f2_split(f2_fma(xb[j], bc[j], f2_mul(xa[j], as[j])), yb[2 * j], yb[2 * j + 1]);
                }
                if (live) write_pairs<T, HALF>(out + i * D, sub, ya, yb);
            }
            out += QB * D;
#pragma unroll
            for (int i = 0; i < QB; ++i) qx[i] = next[i];
        }
    }
    float* mine = &park[warp][grp][0];
    // where this lane's eight slots of head `head` find their channels
    auto slots = [&](const int32_t* perm, int head, int (&at)[8]) {
        const int4* pp = reinterpret_cast<const int4*>(perm + head * D + sub * 8);
        const int4 p0 = __ldg(pp), p1 = __ldg(pp + 1);
        at[0] = p0.x & (D - 1); at[1] = p0.y & (D - 1); at[2] = p0.z & (D - 1); at[3] = p0.w & (D - 1);
        at[4] = p1.x & (D - 1); at[5] = p1.y & (D - 1); at[6] = p1.z & (D - 1); at[7] = p1.w & (D - 1);
    };
    // ---- keys
    if (k0 < k1) {
        tables(a.weight[1]);
        const bool moved = a.weight[1] || a.theta;
        Share<T> kx[KB];
#pragma unroll
        for (int i = 0; i < KB; ++i)
            if (k0 + i < k1) kx[i] = load_share<T, HALF>(k_in + i * D, sub);
        for (int h = k0; h < k1; h += KB) {
            Share<T> next[KB];
            k_in += KB * D;
#pragma unroll
            for (int i = 0; i < KB; ++i)
                if (h + KB + i < k1) next[i] = load_share<T, HALF>(k_in + i * D, sub);
#pragma unroll
            for (int i = 0; i < KB; ++i) {
                if (h + i >= k1) break;
                int at[8];
                if (a.perm[0]) {
                    slots(a.perm[0], h + i, at);
                } else {
#pragma unroll
                    for (int x = 0; x < 8; ++x) at[x] = sub * 8 + x;
                }
                F2 xa[2], xb[2];
                share_pairs<T, HALF>(kx[i], xa, xb);
                const float inv = a.weight[1] ? inv_rms(xa, xb, a.eps) : 1.f;
                const F2 inv2 = f2(inv, inv);
                float y[2][4], err[4];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const F2 na = f2_mul(xa[j], inv2), nb = f2_mul(xb[j], inv2);
                    f2_split(f2_fma(na, ac[j], f2_mul(nb, bs[j])), y[0][2 * j], y[0][2 * j + 1]);
                    f2_split(f2_fma(nb, bc[j], f2_mul(na, as[j])), y[1][2 * j], y[1][2 * j + 1]);
                    float ma[2], mb[2];
                    f2_split(f2_mul(na, wa[j]), ma[0], ma[1]);
                    f2_split(f2_mul(nb, wb[j]), mb[0], mb[1]);
#pragma unroll
                    for (int e = 0; e < 2; ++e) err[2 * j + e] = moved ? fmaf(kErr, fabsf(ma[e]) + fabsf(mb[e]), kErrLow) : 0.f;
                }
                // (value, bound) of each channel
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    if (HALF) {
                        *reinterpret_cast<float4*>(mine + 2 * chan_a<HALF>(sub, 2 * j)) = make_float4(y[0][2 * j], err[2 * j], y[0][2 * j + 1], err[2 * j + 1]);
                        *reinterpret_cast<float4*>(mine + 2 * chan_b<HALF>(sub, 2 * j)) = make_float4(y[1][2 * j], err[2 * j], y[1][2 * j + 1], err[2 * j + 1]);
                    } else {
#pragma unroll
                        for (int e = 0; e < 2; ++e)
                            *reinterpret_cast<float4*>(mine + 2 * chan_a<HALF>(sub, 2 * j + e)) = make_float4(y[0][2 * j + e], err[2 * j + e], y[1][2 * j + e], err[2 * j + e]);
                    }
                }
                __syncwarp();
                float v[8], ev[8];
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    const float2 z = *reinterpret_cast<const float2*>(mine + 2 * at[x]);
                    v[x] = z.x;
                    ev[x] = z.y;
                }
                __syncwarp();
                uint32_t f[8];
                int e8;
                bool finite;
                const bool near = cast32<P, N, true>(v, ev, f, e8, finite);
                if (__any_sync(0xffffffffu, near && finite && stored)) {
                    double za[4], zb[4], inv64 = 1.0;
                    float pa[4], pb[4], qa[4], qb[4];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        f2_split(xa[j], pa[2 * j], pa[2 * j + 1]);
                        f2_split(xb[j], pb[2 * j], pb[2 * j + 1]);
                        f2_split(wa[j], qa[2 * j], qa[2 * j + 1]);
                        f2_split(wb[j], qb[2 * j], qb[2 * j + 1]);
                    }
                    if (a.weight[1]) {
                        double ss = 0.0;
#pragma unroll
                        for (int j = 0; j < 4; ++j) ss = fma((double)pa[j], (double)pa[j], fma((double)pb[j], (double)pb[j], ss));
#pragma unroll
                        for (int off = 8; off; off >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, off);
                        inv64 = 1.0 / sqrt(ss * (1.0 / D) + (double)a.eps);
                    }
                    turn64(pa, pb, qa, qb, inv64, a.theta ? a.theta + 4 * sub : nullptr, pos, za, zb);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        *reinterpret_cast<double*>(mine + 2 * chan_a<HALF>(sub, j)) = za[j];
                        *reinterpret_cast<double*>(mine + 2 * chan_b<HALF>(sub, j)) = zb[j];
                    }
                    __syncwarp();
                    double w[8];
#pragma unroll
                    for (int x = 0; x < 8; ++x) w[x] = *reinterpret_cast<const double*>(mine + 2 * at[x]);
                    __syncwarp();
                    uint32_t f64[8];
                    int e64;
                    cast64<P, N>(w, f64, e64);
                    if (finite) {
#pragma unroll
                        for (int x = 0; x < 8; ++x) f[x] = f64[x];
                        e8 = e64;
                    }
                }
                if (live && !finite) raise_flag(a.status, KVBFP_FLAG_NONFINITE);
                const int64_t row = row0 + (int64_t)(h + i) * a.map.rows;
                if (stored) put_row<P, N>(f, e8, a.mant[0] + row * ROW_M, a.exp8[0] + row * ROW_E, sub);
            }
#pragma unroll
            for (int i = 0; i < KB; ++i) kx[i] = next[i];
        }
    }
    // ---- values
    if (v0 < v1) {
        Share<T> vx[KB];
#pragma unroll
        for (int i = 0; i < KB; ++i)
            if (v0 + i < v1) vx[i] = load_share<T, false>(v_in + i * D, sub);
        for (int h = v0; h < v1; h += KB) {
            Share<T> next[KB];
            v_in += KB * D;
#pragma unroll
            for (int i = 0; i < KB; ++i)
                if (h + KB + i < v1) next[i] = load_share<T, false>(v_in + i * D, sub);
#pragma unroll
            for (int i = 0; i < KB; ++i) {
                if (h + i >= v1) break;
                const int64_t row = row0 + (int64_t)(h + i) * a.map.rows;
                uint8_t *mrow = a.mant[1] + row * ROW_M, *erow = a.exp8[1] + row * ROW_E;
                bool finite;
                int at[8];
                if (a.perm[1]) slots(a.perm[1], h + i, at);
                if (sizeof(T) == 2 && P != 8) {
                    uint32_t f[4];
                    if (a.perm[1]) {
                        *reinterpret_cast<uint4*>(mine + 4 * sub) = make_uint4(vx[i].w[0], vx[i].w[1], vx[i].w[2], vx[i].w[3]);
                        __syncwarp();
                        uint32_t e[8];
#pragma unroll
                        for (int x = 0; x < 8; ++x) e[x] = reinterpret_cast<const unsigned short*>(mine)[at[x]];
                        __syncwarp();
#pragma unroll
                        for (int x = 0; x < 4; ++x) f[x] = P == 4 ? prmt(e[x], e[x + 4], 0x5410u) : prmt(e[2 * x], e[2 * x + 1], 0x5410u);
                    } else {
#pragma unroll
                        for (int x = 0; x < 4; ++x) f[x] = P == 4 ? prmt(vx[i].w[x >> 1], vx[i].w[2 + (x >> 1)], (x & 1) ? 0x7632u : 0x5410u) : vx[i].w[x];
                    }
                    finite = cast_bf16<P == 8 ? 4 : P, N>(f, stored, mrow, erow, sub);
                } else {
                    float v[8];
                    share_values<T>(vx[i], v);
                    if (a.perm[1]) {
                        *reinterpret_cast<float4*>(mine + 8 * sub) = make_float4(v[0], v[1], v[2], v[3]);
                        *reinterpret_cast<float4*>(mine + 8 * sub + 4) = make_float4(v[4], v[5], v[6], v[7]);
                        __syncwarp();
#pragma unroll
                        for (int x = 0; x < 8; ++x) v[x] = mine[at[x]];
                        __syncwarp();
                    }
                    uint32_t f[8];
                    int e8;
                    (void)cast32<P, N, false>(v, v, f, e8, finite);
                    if (stored) put_row<P, N>(f, e8, mrow, erow, sub);
                }
                if (live && !finite) raise_flag(a.status, KVBFP_FLAG_NONFINITE);
            }
#pragma unroll
            for (int i = 0; i < KB; ++i) vx[i] = next[i];
        }
    }
}

template <int P, int N, typename T, bool HALF>
kvbfp_status launch_write(WriteArgs a, cudaStream_t s) {
    int n_sm = 0;
    const kvbfp_status st = sm_count(&n_sm);
    if (st != KVBFP_OK) return st;
    const int n_heads = a.heads[0] + a.heads[1] + a.heads[2];
    const int64_t pairs = ((int64_t)a.n_tokens + 1) / 2, gx = (pairs + kWWarps - 1) / kWWarps;
    // few tokens: heads spread over the blocks too, down to one head a warp.  Up to four rounds of three blocks an SM in halves, whose
    // last round is shorter (3 and 4 prompts 95.8 -> 93.1, 122.8 -> 120.5 us); later what a warp begins with costs more (6 and 14
    // prompts 163.2 -> 165.1, 324 -> 345 us).
    int64_t chunks = (int64_t)n_sm * 4 / gx;
    if (chunks < 2) chunks = gx < (int64_t)n_sm * 12 ? 2 : 1;
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
    if (!starts || !seq_lens) return KVBFP_ERR_INVALID_ARG;
    // (arrays of no tokens may well have no address)
    if (n_tokens != 0 && ((!q && !k) || (k == nullptr) != (v == nullptr) || (q == nullptr) != (q_out == nullptr))) return KVBFP_ERR_INVALID_ARG;
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
