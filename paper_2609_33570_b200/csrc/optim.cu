// OptimizerStep of the actor update: the global gradient norm and the AdamW step over all tensors of a table, one launch
// for the whole table.  Moments are fp32, or 8 bits in the library's block format (E4M3FN codes, one fp32 scale per 64).
//
// Both are streams of a few bytes and a few operations per element: HBM is the bound.  A warp owns a tile of 1024
// consecutive elements of one tensor and finds that tensor by a 32-ary search over the table's `first` column (two
// dependent loads for a thousand tensors), so tensors of any size share one launch without a map of tiles.
// Measured: the norm of 900 M bf16 gradients 267 us (6.7 TB/s); their step with 8-bit moments 1690 us (10.25 bytes an element,
// 5.5 TB/s: some 40 operations per element fill two thirds of the issue slots; asynchronous copies of the next 512 elements into shared memory
// changed nothing); a step with fp32 moments and master copies over 11.2 GB 1807 us (6.2 TB/s).
#include "common.cuh"

#include <cmath>

namespace hilore {

constexpr int kTile = HILORE_PARAM_TILE; // elements of a warp's tile
constexpr int kOptThreads = 256, kOptWarps = kOptThreads / 32;
constexpr int kNormMaxGrid = 2048; // partial sums in the workspace
constexpr float kE4m3Max = 448.0f;

__device__ __forceinline__ float load_one(const void *p, int32_t dtype, int64_t i)
{
    return dtype == HILORE_BF16 ? __uint_as_float((uint32_t)static_cast<const uint16_t *>(p)[i] << 16) : static_cast<const float *>(p)[i];
}

__device__ __forceinline__ void store_one(void *p, int32_t dtype, int64_t i, float v)
{
    if (dtype == HILORE_BF16) static_cast<uint16_t *>(p)[i] = (uint16_t)cvt_bf16x2(0.0f, v);
    else static_cast<float *>(p)[i] = v;
}

__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// N consecutive values (8 or 16) in vectors, kept as loaded: bf16 pairs or fp32.
template <int DTYPE, int N> struct Raw {
    static constexpr int W = DTYPE == HILORE_BF16 ? N / 2 : N;
    uint32_t w[W];
    __device__ __forceinline__ void load(const void *p, int64_t i)
    {
        if (W == 4) {
            const uint4 q = ld_global_128_stream(static_cast<const uint16_t *>(p) + i);
            w[0] = q.x, w[1] = q.y, w[2] = q.z, w[3] = q.w;
        } else {
#pragma unroll
            for (int k = 0; k < W / 8; ++k) {
                uint32_t t[8];
                ld_global_256(static_cast<const char *>(p) + i * (DTYPE == HILORE_BF16 ? 2 : 4) + 32 * k, t);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    w[8 * k + j] = t[j];
            }
        }
    }
    __device__ __forceinline__ float get(int k) const
    {
        if (DTYPE == HILORE_F32) return __uint_as_float(w[k]);
        return k & 1 ? bf16_hi(w[k >> 1]) : bf16_lo(w[k >> 1]);
    }
    __device__ __forceinline__ uint64_t pair(int k) const { return f32x2_pack(get(k), get(k + 1)); }
    __device__ __forceinline__ void set2(int k, float x0, float x1) // k even
    {
        if (DTYPE == HILORE_F32) {
            w[k] = __float_as_uint(x0);
            w[k + 1] = __float_as_uint(x1);
        } else {
            w[k >> 1] = cvt_bf16x2(x1, x0);
        }
    }
    __device__ __forceinline__ void store(void *p, int64_t i) const
    {
        if (W == 4) {
            *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(p) + i) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
#pragma unroll
            for (int k = 0; k < W / 8; ++k) {
                uint32_t t[8];
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    t[j] = w[8 * k + j];
                st_global_256(static_cast<char *>(p) + i * (DTYPE == HILORE_BF16 ? 2 : 4) + 32 * k, t);
            }
        }
    }
};

// Index of the tensor that owns `tile`: the last entry whose first tile is not beyond it.  Called by whole warps.
__device__ __forceinline__ int owner_of(const hilore_param *params, int n_params, int64_t tile)
{
    const int lane = threadIdx.x & 31;
    int lo = 0, hi = n_params;
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) >> 5;
        const int at = lo + lane * step;
        const bool below = at < hi && __ldg(&params[at].first) <= tile;
        const int n = __popc(__ballot_sync(0xFFFFFFFFu, below)); // the entries are in order: lanes 0 .. n - 1
        lo += (n - 1) * step;
        hi = min(lo + step, hi);
    }
    return lo;
}

// A warp's way through consecutive tiles: the entry that owns the current one, looked up only when the tile leaves it.  The
// entry lives in shared memory: its seven pointers would take a quarter of the registers.
struct Walk {
    const hilore_param *params;
    int n_params;
    int64_t begin, end; // tiles of entry `e`
    hilore_param *e;    // the warp's copy
    __device__ __forceinline__ Walk(const hilore_param *p, int n, hilore_param *copies)
        : params(p), n_params(n), begin(0), end(0), e(copies + (threadIdx.x >> 5))
    {
    }
    __device__ __forceinline__ bool at(int64_t tile) // true where the entry is a new one
    {
        if (tile < end)
            return false;
        const uint32_t *from = reinterpret_cast<const uint32_t *>(params + owner_of(params, n_params, tile));
        __syncwarp();
        for (int i = threadIdx.x & 31; i < (int)(sizeof(hilore_param) / 4); i += 32)
            reinterpret_cast<uint32_t *>(e)[i] = __ldg(from + i);
        __syncwarp();
        begin = e->first;
        end = begin + (e->n + kTile - 1) / kTile;
        return true;
    }
};

// Tiles of a warp: up to eight in a row, so that the look-up (two to three dependent loads) is paid once in 8192 elements,
// fewer while that would leave SMs without two rounds of full occupancy.
static int tiles_per_warp(int64_t tiles)
{
    int64_t k = tiles / ((int64_t)sm_count() * 64);
    return k < 1 ? 1 : k > 8 ? 8 : (int)k;
}

// ------------------------------------------------------------------------------------------------------------------- norm
// Squares in fp32 over the 32 elements of a lane's tile, fp64 beyond; a lane whose fp32 sum overflows, or is so small that squares have
// lost bits to 2^-149 (at 2^-100 all 32 lose 2^-45 of it at most), redoes its elements in fp64; zeros alone do not.  Partial sums in
// fixed slots: the result does not depend on scheduling.
template <int DTYPE> __device__ __forceinline__ double tile_squares(const void *g, int64_t base, int64_t n, bool vec)
{
    constexpr float kExact = 7.888609052e-31f; // 2^-100
    const int lane = threadIdx.x & 31;
    float s = 0.0f;
    uint32_t any = 0; // bits of the magnitudes, for a small sum
    if (vec && base + kTile <= n) {
        Raw<DTYPE, 8> x[kTile / 256];
#pragma unroll
        for (int k = 0; k < kTile / 256; ++k)
            x[k].load(g, base + k * 256 + lane * 8);
#pragma unroll
        for (int k = 0; k < kTile / 256; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                s = fmaf(x[k].get(i), x[k].get(i), s);
        if (s < kExact) {
#pragma unroll
            for (int k = 0; k < kTile / 256; ++k)
#pragma unroll
                for (int i = 0; i < Raw<DTYPE, 8>::W; ++i)
                    any |= x[k].w[i] & (DTYPE == HILORE_BF16 ? 0x7FFF7FFFu : 0x7FFFFFFFu);
        }
    } else {
        for (int64_t i = base + lane; i < min(n, base + kTile); i += 32) {
            const float x = load_one(g, DTYPE, i);
            s = fmaf(x, x, s);
            any |= __float_as_uint(x) & 0x7FFFFFFFu;
        }
    }
    double d = (double)s;
    if (!(s < INFINITY) || (s < kExact && any)) {
        d = 0.0;
        const bool dealt = vec && base + kTile <= n; // which elements were this lane's
        for (int k = 0; k < kTile / 32; ++k) {
            const int64_t i = base + (dealt ? (k >> 3) * 256 + lane * 8 + (k & 7) : k * 32 + lane);
            const double x = i < n ? (double)load_one(g, DTYPE, i) : 0.0;
            d += x * x;
        }
    }
    return d;
}

__global__ void __launch_bounds__(kOptThreads, 4) grad_norm_kernel(const hilore_param *params, int n_params, int64_t n_tiles, int per_warp, double *partial)
{
    const int lane = threadIdx.x & 31;
    double sum = 0.0;
    grid_dependency_wait();
    grid_dependency_release();
    __shared__ hilore_param copies[kOptWarps];
    Walk walk(params, n_params, copies);
    const int64_t stride = (int64_t)gridDim.x * kOptWarps * per_warp;
    for (int64_t t0 = ((int64_t)blockIdx.x * kOptWarps + (threadIdx.x >> 5)) * per_warp; t0 < n_tiles; t0 += stride)
        for (int64_t tile = t0; tile < min(t0 + per_warp, n_tiles); ++tile) {
            walk.at(tile);
            const int64_t base = (tile - walk.begin) * kTile;
            const hilore_param &e = *walk.e;
            const bool vec = (reinterpret_cast<uintptr_t>(e.g) & 31) == 0;
            sum += e.g_dtype == HILORE_BF16 ? tile_squares<HILORE_BF16>(e.g, base, e.n, vec) : tile_squares<HILORE_F32>(e.g, base, e.n, vec);
        }
    __shared__ double sm[kOptWarps];
    sum = warp_sum(sum);
    if (lane == 0) sm[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kOptWarps; ++w)
            sum += sm[w];
        partial[blockIdx.x] = sum;
    }
}

__global__ void __launch_bounds__(kOptThreads) grad_norm_final_kernel(const double *partial, int n, double max_norm, float *norm, float *scale)
{
    __shared__ double sm[kOptWarps];
    double sum = 0.0;
    grid_dependency_wait();
    grid_dependency_release();
    for (int i = threadIdx.x; i < n; i += kOptThreads)
        sum += partial[i];
    sum = warp_sum(sum);
    if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kOptWarps; ++w)
            sum += sm[w];
        const double r = sqrt(sum);
        if (norm) *norm = (float)r;
        if (scale) *scale = r < (double)INFINITY ? (float)fmin(1.0, max_norm / (r + 1e-6)) : NAN;
    }
}

// ------------------------------------------------------------------------------------------------------------------ AdamW
struct AdamArgs {
    double beta1, beta2;
    float b1, omb1, b2, omb2, eps, one; // omb = 1 - beta, rounded once; one = 1
    float lr, inv_bc1, rsqrt_bc2;  // 1 / (1 - beta1^t), 1 / sqrt(1 - beta2^t) where t is known on the host
    const float *lr_dev, *grad_scale;
    const int64_t *step_dev;
};

// What one element's update takes, in registers.
struct AdamStep {
    float gscale, b1, omb1, b2, omb2, eps, rsqrt_bc2, one;
    float step, lrwd; // lr / (1 - beta1^t), lr * weight decay of the entry
};

__device__ __forceinline__ uint64_t both(float x) { return f32x2_pack(x, x); }

// Two elements at a time, in packed fp32 pairs.  The moments take every operation rounded by itself in the order of the
// formula: with 8-bit states the last bit decides the codes of values near a tie, and a code of the next step's largest value
// moves the scale of 64 elements; contracted operations would make them depend on the compiler.  The sums are written as
// products with a one that the compiler does not know: a packed product and a packed sum come out as one fused operation even where
// both name their rounding (a fifth of the scales of a large table then differed in the last bit).
__device__ __forceinline__ void next_moments(const AdamStep &h, uint64_t g, uint64_t &m, uint64_t &v)
{
    const uint64_t x = f32x2_mul(g, both(h.gscale));
    m = f32x2_fma(f32x2_mul(both(h.b1), m), both(h.one), f32x2_mul(both(h.omb1), x));
    v = f32x2_fma(f32x2_mul(both(h.b2), v), both(h.one), f32x2_mul(f32x2_mul(both(h.omb2), x), x));
}

// The same with minus v for the 8-bit states, which flush what is below 2^-126 on the way; `h` has b2 and omb2 negated.
__device__ __forceinline__ void next_moments_negated(const AdamStep &h, uint64_t g, uint64_t &m, uint64_t &v)
{
    const uint64_t x = f32x2_mul(g, both(h.gscale));
    m = f32x2_fma(f32x2_mul(both(h.b1), m), both(h.one), f32x2_mul(both(h.omb1), x));
    const uint64_t a = f32x2_mul(both(h.b2), v), b = f32x2_mul(f32x2_mul(both(h.omb2), x), x);
    asm("fma.rn.ftz.f32x2 %0, %1, %2, %3;" : "=l"(v) : "l"(a), "l"(both(h.one)), "l"(b));
}

__device__ __forceinline__ float rcp_approx(float x)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// p - lr (wd p + m^ / (sqrt(v^) + eps)) from the new moment m and root r = sqrt(v): the 32-bit states' form, and the packed one of
// the 8-bit states, whose quotient is within three units in the last place (a denominator is zero or above 2^-63).
__device__ __forceinline__ float next_param(const AdamStep &h, float p, float m, float r)
{
    return p - fmaf(h.lrwd, p, h.step * __fdiv_rn(m, fmaf(r, h.rsqrt_bc2, h.eps)));
}
__device__ __forceinline__ uint64_t next_param2(const AdamStep &h, uint64_t p, uint64_t m, uint64_t r)
{
    float d0, d1;
    f32x2_unpack(f32x2_fma(r, both(h.rsqrt_bc2), both(h.eps)), d0, d1);
    const uint64_t q = f32x2_mul(f32x2_mul(m, both(h.step)), f32x2_pack(rcp_approx(d0), rcp_approx(d1)));
    return f32x2_sub(p, f32x2_fma(both(h.lrwd), p, q));
}

// Square roots of a pair of v from minus v (zero, or at least 2^-126 in size): Newton's step r - (r^2 - v) / (2 r) from
// r = v * rsqrt(v), the residual formed exactly by a fused operation down to v = 2^-102: an error of 2^-43 is left before the final
// rounding, and of all numbers from there on none was found rounded to the wrong neighbour.  Below, where the residual loses bits to
// 2^-149, 1.8 of 201 million are (one in ten at 2^-126).  Every path of the 8-bit states takes its roots
// here: a tensor's results do not depend on its alignment.  Two roots at a time in packed operations without a branch.
__device__ __forceinline__ uint64_t root2(uint64_t minus_v)
{
    constexpr float kMost = 9.223372036854775808e18f; // 2^63, of 2^-126; of zero this instead of Inf
    float v0, v1, y0, y1;
    f32x2_unpack(minus_v, v0, v1);
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y0) : "f"(-v0));
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y1) : "f"(-v1));
    const uint64_t y = f32x2_pack(fmaxf(-y0, -kMost), fmaxf(-y1, -kMost)); // minus 1 / sqrt(v)
    const uint64_t r = f32x2_mul(minus_v, y);
    return f32x2_fma(f32x2_fma(r, r, minus_v), f32x2_mul(y, both(0.5f)), r);
}

// The same where v may be Inf or NaN, which are their own roots.
__device__ __forceinline__ uint64_t root2_any(uint64_t minus_v)
{
    float v0, v1, r0, r1;
    f32x2_unpack(minus_v, v0, v1);
    f32x2_unpack(root2(minus_v), r0, r1);
    return f32x2_pack(fabsf(v0) < INFINITY ? r0 : fabsf(v0), fabsf(v1) < INFINITY ? r1 : fabsf(v1));
}

__device__ __forceinline__ uint64_t decode2(uint32_t codes, float s) // two codes in the low half
{
    const uint32_t h = cvt_e4m3x2_to_f16x2(codes);
    return f32x2_mul(f32x2_pack(f16_lo_to_f32(h), f16_hi_to_f32(h)), both(s));
}

// Largest magnitude of a block of 64: 16 values of each of the four lanes of a quad; Inf and NaN count as Inf.
__device__ __forceinline__ float quad_max(const uint64_t (&x)[8])
{
    float a = 0.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        float x0, x1;
        f32x2_unpack(x[k], x0, x1);
        a = max_nan(a, max_nan(fabsf(x0), fabsf(x1)));
    }
    a = a < INFINITY ? a : INFINITY;
    a = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, 1));
    return fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, 2));
}

// The same over the finite values alone.
__device__ __forceinline__ float quad_max_finite(const uint64_t (&x)[8])
{
    float a = 0.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        float x0, x1;
        f32x2_unpack(x[k], x0, x1);
        a = fabsf(x0) < INFINITY ? fmaxf(a, fabsf(x0)) : a;
        a = fabsf(x1) < INFINITY ? fmaxf(a, fabsf(x1)) : a;
    }
    a = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, 1));
    return fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, 2));
}

// And of two values of each lane of a warp.
__device__ __forceinline__ float warp_max_finite(float x0, float x1)
{
    float a = fabsf(x0) < INFINITY ? fabsf(x0) : 0.0f;
    a = fabsf(x1) < INFINITY ? fmaxf(a, fabsf(x1)) : a;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        a = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, o));
    return a;
}

// Scale of a block whose largest magnitude is `top`, and its inverse.  A block of zeros, without a finite value, or too small
// for 448 / top takes scale 1.
struct BlockScale {
    float scale, inv;
    bool fits; // not one of those
};
__device__ __forceinline__ BlockScale block_scale(float top)
{
    BlockScale s{__fmul_rn(top, 1.0f / kE4m3Max), __fmul_rn(kE4m3Max, __frcp_rn(top)), true};
    if (!(s.inv < INFINITY)) {
        s.scale = s.inv = 1.0f;
        s.fits = false;
    }
    return s;
}

// Codes of 16 values of a block.  ROOT: the values are square roots of v, of which a positive one is never rounded to zero (it
// would turn the next step's division into one by eps) but takes the smallest code; lanes without a zero code, the usual
// ones, skip the test of their values.
template <bool ROOT> __device__ __forceinline__ void encode16(const uint64_t (&x)[8], const BlockScale &s, uint32_t (&w)[4])
{
    uint32_t zeros = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float q[4];
        f32x2_unpack(f32x2_mul(x[2 * k], both(s.inv)), q[0], q[1]);
        f32x2_unpack(f32x2_mul(x[2 * k + 1], both(s.inv)), q[2], q[3]);
        w[k] = cvt_e4m3x4(q[0], q[1], q[2], q[3]);
        if (ROOT) zeros |= (w[k] - 0x01010101u) & ~w[k];
    }
    if (ROOT && (zeros & 0x80808080u) && s.fits) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            float x0, x1;
            f32x2_unpack(x[k], x0, x1);
            const int at = 16 * (k & 1);
            if (x0 > 0.0f && !(w[k >> 1] >> at & 0xFFu)) w[k >> 1] |= 1u << at;
            if (x1 > 0.0f && !(w[k >> 1] >> (at + 8) & 0xFFu)) w[k >> 1] |= 1u << (at + 8);
        }
    }
}

// ---- whole tiles: vectors, types known at compile time ----
template <int P, int G, bool MASTER> __device__ __forceinline__ void run_f32(const hilore_param &e, const AdamStep &h, int64_t base, int len)
{
    const int lane = threadIdx.x & 31;
#pragma unroll 1
    for (int k = 0; k < len; k += 256) {
        const int64_t i = base + k + lane * 8;
        Raw<G, 8> g;
        Raw<HILORE_F32, 8> m, v;
        Raw<MASTER ? HILORE_F32 : P, 8> p;
        g.load(e.g, i);
        m.load(e.m, i);
        v.load(e.v, i);
        p.load(MASTER ? (const void *)e.master : e.p, i);
        Raw<P, 8> out;
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            uint64_t mm = m.pair(j), vv = v.pair(j);
            next_moments(h, g.pair(j), mm, vv);
            float m0, m1, v0, v1;
            f32x2_unpack(mm, m0, m1);
            f32x2_unpack(vv, v0, v1);
            const float p0 = next_param(h, p.get(j), m0, __fsqrt_rn(v0)), p1 = next_param(h, p.get(j + 1), m1, __fsqrt_rn(v1));
            m.set2(j, m0, m1);
            v.set2(j, v0, v1);
            if (MASTER) p.set2(j, p0, p1);
            out.set2(j, p0, p1);
        }
        m.store(e.m, i);
        v.store(e.v, i);
        if (MASTER) p.store(e.master, i);
        out.store(e.p, i);
    }
}

// The four lanes of a quad own one block of 64.  The moments of this step enter the update in fp32, before they are rounded
// to codes; v holds the codes of sqrt(v), as the square root halves the range that the codes have to span.
template <int P, int G, bool MASTER>
__device__ __forceinline__ void run_e4m3(const hilore_param &e, const AdamStep &h, int64_t base, int len)
{
    const int lane = threadIdx.x & 31;
#pragma unroll 1
    for (int t = 0; t < len; t += 512) {
        const int64_t i = base + t + lane * 16;
        Raw<G, 16> g;
        Raw<MASTER ? HILORE_F32 : P, 16> p;
        const uint4 mc = ld_global_128_stream(static_cast<const uint8_t *>(e.m) + i), rc = ld_global_128_stream(static_cast<const uint8_t *>(e.v) + i);
        const float ms = e.m_scale[i >> 6], rs = e.v_scale[i >> 6];
        g.load(e.g, i);
        p.load(MASTER ? (const void *)e.master : e.p, i);
        const uint32_t mw[4] = {mc.x, mc.y, mc.z, mc.w}, rw[4] = {rc.x, rc.y, rc.z, rc.w};
        uint64_t m[8], r[8]; // r: v until its root is taken
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            m[k] = decode2(mw[k >> 1] >> (16 * (k & 1)), ms);
            r[k] = decode2(rw[k >> 1] >> (16 * (k & 1)), rs);
            r[k] = f32x2_mul(r[k], r[k]);
            next_moments_negated(h, g.pair(2 * k), m[k], r[k]);
        }
        float am = quad_max(m), ar = quad_max(r); // of v: the root is monotone
        const bool odd = __any_sync(0xFFFFFFFFu, fmaxf(am, ar) == INFINITY);
        if (odd) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                r[k] = root2_any(r[k]);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                r[k] = root2(r[k]);
        }
        Raw<P, 16> out;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            float p0, p1;
            f32x2_unpack(next_param2(h, p.pair(2 * k), m[k], r[k]), p0, p1);
            if (MASTER) p.set2(2 * k, p0, p1);
            out.set2(2 * k, p0, p1);
        }
        if (MASTER) p.store(e.master, i);
        out.store(e.p, i);
        if (odd) {
            am = quad_max_finite(m);
            ar = quad_max_finite(r);
        } else {
            float unused;
            f32x2_unpack(root2(both(-ar)), ar, unused);
        }
        const BlockScale sm = block_scale(am), sr = block_scale(ar);
        uint32_t w[4];
        encode16<false>(m, sm, w);
        *reinterpret_cast<uint4 *>(static_cast<uint8_t *>(e.m) + i) = make_uint4(w[0], w[1], w[2], w[3]);
        encode16<true>(r, sr, w);
        *reinterpret_cast<uint4 *>(static_cast<uint8_t *>(e.v) + i) = make_uint4(w[0], w[1], w[2], w[3]);
        if ((lane & 3) == 0) {
            e.m_scale[i >> 6] = sm.scale;
            e.v_scale[i >> 6] = sr.scale;
        }
    }
}

// ---- the last tile of a tensor and tensors off the vectors' alignment: the same arithmetic on single elements, two of
// every block of 64 in each lane, so that a warp's accesses are next to each other ----
template <int DTYPE> __device__ __forceinline__ uint32_t load_bits(const void *p, int64_t i) // nothing waits for it here
{
    return DTYPE == HILORE_BF16 ? (uint32_t)static_cast<const uint16_t *>(p)[i] : static_cast<const uint32_t *>(p)[i];
}
template <int DTYPE> __device__ __forceinline__ float from_bits(uint32_t w) { return __uint_as_float(DTYPE == HILORE_BF16 ? w << 16 : w); }

template <bool CODED, int P, int G, bool MASTER> __device__ __noinline__ void tile_ragged(const hilore_param *entry, const AdamStep h, int64_t base, int len)
{
    constexpr int B = 4; // blocks in flight
    constexpr int Q = MASTER ? HILORE_F32 : P;
    const int lane = threadIdx.x & 31;
    const int64_t n = entry->n;
    void *const out = entry->p;
    float *const master = entry->master;
    void *const from = MASTER ? (void *)master : out;
    const void *const grad = entry->g;
    uint8_t *const mc = static_cast<uint8_t *>(entry->m), *const rc = static_cast<uint8_t *>(entry->v);
    float *const m32 = static_cast<float *>(entry->m), *const v32 = static_cast<float *>(entry->v);
    float *const m_scale = entry->m_scale, *const v_scale = entry->v_scale;
    for (int64_t b0 = base; b0 < min(n, base + len); b0 += 64 * B) {
        uint32_t g[B][2], p[B][2], m[B][2], v[B][2];
        float ms[B], rs[B];
#pragma unroll
        for (int k = 0; k < B; ++k) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int64_t i = b0 + 64 * k + 32 * u + lane;
                g[k][u] = p[k][u] = m[k][u] = v[k][u] = 0;
                if (i < n) {
                    g[k][u] = load_bits<G>(grad, i);
                    p[k][u] = load_bits<Q>(from, i);
                    m[k][u] = CODED ? mc[i] : __float_as_uint(m32[i]);
                    v[k][u] = CODED ? rc[i] : __float_as_uint(v32[i]);
                }
            }
            const bool some = CODED && b0 + 64 * k < n;
            ms[k] = some ? m_scale[(b0 >> 6) + k] : 0.0f;
            rs[k] = some ? v_scale[(b0 >> 6) + k] : 0.0f;
        }
#pragma unroll
        for (int k = 0; k < B; ++k) {
            const int64_t i0 = b0 + 64 * k + lane;
            uint64_t mm = u32x2_pack(m[k][0], m[k][1]), vv = u32x2_pack(v[k][0], v[k][1]);
            if (CODED) {
                mm = decode2(m[k][0] | m[k][1] << 8, ms[k]);
                vv = decode2(v[k][0] | v[k][1] << 8, rs[k]);
                vv = f32x2_mul(vv, vv);
            }
            const uint64_t gg = f32x2_pack(from_bits<G>(g[k][0]), from_bits<G>(g[k][1]));
            if (CODED) next_moments_negated(h, gg, mm, vv);
            else next_moments(h, gg, mm, vv);
            float m1[2], v1[2], r[2], q[2];
            f32x2_unpack(mm, m1[0], m1[1]);
            f32x2_unpack(vv, v1[0], v1[1]);
            if (CODED) {
                f32x2_unpack(root2_any(vv), r[0], r[1]);
            } else {
                r[0] = __fsqrt_rn(v1[0]);
                r[1] = __fsqrt_rn(v1[1]);
            }
            const float p0 = from_bits<Q>(p[k][0]), p1 = from_bits<Q>(p[k][1]);
            if (CODED) {
                f32x2_unpack(next_param2(h, f32x2_pack(p0, p1), mm, f32x2_pack(r[0], r[1])), q[0], q[1]);
            } else {
                q[0] = next_param(h, p0, m1[0], r[0]);
                q[1] = next_param(h, p1, m1[1], r[1]);
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int64_t i = i0 + 32 * u;
                if (i >= n)
                    continue;
                if (!CODED) {
                    m32[i] = m1[u];
                    v32[i] = v1[u];
                }
                if (MASTER) master[i] = q[u];
                store_one(out, P, i, q[u]);
            }
            if (!CODED)
                continue;
            const BlockScale sm = block_scale(warp_max_finite(m1[0], m1[1])), sr = block_scale(warp_max_finite(r[0], r[1]));
            const uint32_t cm = cvt_e4m3x2(__fmul_rn(m1[1], sm.inv), __fmul_rn(m1[0], sm.inv));
            r[0] = __fmul_rn(r[0], sr.inv);
            r[1] = __fmul_rn(r[1], sr.inv);
            uint32_t cr = cvt_e4m3x2(r[1], r[0]);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if (sr.fits && r[u] > 0.0f && !(cr >> (8 * u) & 0xFFu)) cr |= 1u << (8 * u);
                if (i0 + 32 * u < n) {
                    mc[i0 + 32 * u] = (uint8_t)(cm >> (8 * u));
                    rc[i0 + 32 * u] = (uint8_t)(cr >> (8 * u));
                }
            }
            if (lane == 0 && b0 + 64 * k < n) {
                m_scale[(b0 >> 6) + k] = sm.scale;
                v_scale[(b0 >> 6) + k] = sr.scale;
            }
        }
    }
}

// Kinds of tables: KIND = state * 6 + gradient type * 3 + (0: bf16, 1: fp32, 2: bf16 with a master copy); kMixed: entries of
// several kinds, told apart at run time.
constexpr int kMixed = 12;
static int kind_of(const hilore_param &e) { return e.state * 6 + e.g_dtype * 3 + (e.master ? 2 : e.p_dtype); }

// Elements [base, base + len): whole tiles (or halves of one) in vectors, or single elements.
template <int KIND>
__device__ __forceinline__ void run_of_kind(const hilore_param &e, const AdamStep &h, int64_t base, int len, bool whole)
{
    constexpr int G = KIND / 3 % 2, PK = KIND % 3;
    constexpr int P = PK == 1 ? HILORE_F32 : HILORE_BF16;
    if (!whole) tile_ragged<KIND / 6 == HILORE_STATE_E4M3FN, P, G, PK == 2>(&e, h, base, len);
    else if (KIND / 6 == HILORE_STATE_F32) run_f32<P, G, PK == 2>(e, h, base, len);
    else run_e4m3<P, G, PK == 2>(e, h, base, len);
}

// Registers: 64 for 32-bit states, 80 for 8-bit ones (900 M bf16 elements 1690 us, 1750 with 64).
// SPLIT: warps per tile; two where there are few tiles, for the latency.
template <int KIND, int SPLIT>
__global__ void __launch_bounds__(kOptThreads, KIND == kMixed ? 2 : KIND <= 5 ? 4 : 3) adamw_kernel(const hilore_param *params, int n_params, int64_t n_tiles, int per_warp, AdamArgs a)
{
    // From the last tile to the first: a norm taken just before has left the end of the gradients in L2.
    const int64_t w = (int64_t)(gridDim.x - 1 - blockIdx.x) * kOptWarps + (threadIdx.x >> 5), t0 = w / SPLIT * per_warp;
    const int skip = (int)(w % SPLIT) * (kTile / SPLIT);
    grid_dependency_wait();
    if (t0 >= n_tiles)
        return;
    AdamStep h;
    h.gscale = a.grad_scale ? *a.grad_scale : 1.0f;
    __shared__ hilore_param copies[kOptWarps];
    Walk walk(params, n_params, copies);
    const hilore_param &e = *walk.e;
    if (SPLIT > 1) walk.at(t0); // while the scale is on its way
    if (!(fabsf(h.gscale) < INFINITY)) // the gradients are not finite: parameters and moments stay as they are
        return;
    const float lr = a.lr_dev ? *a.lr_dev : a.lr;
    float inv_bc1 = a.inv_bc1;
    h.rsqrt_bc2 = a.rsqrt_bc2;
    if (a.step_dev) {
        const double t = (double)*a.step_dev;
        inv_bc1 = (float)(1.0 / -expm1(t * log(a.beta1)));
        h.rsqrt_bc2 = (float)rsqrt(-expm1(t * log(a.beta2)));
    }
    h.b1 = a.b1, h.omb1 = a.omb1, h.eps = a.eps, h.one = a.one;
    h.step = lr * inv_bc1;
    bool vec = false;
    const int64_t t1 = min(t0 + per_warp, n_tiles);
    for (int64_t tile = t0; tile < t1;) {
        if (walk.at(tile) || (SPLIT > 1 && tile == t0)) {
            const uintptr_t wide = reinterpret_cast<uintptr_t>(e.p) | reinterpret_cast<uintptr_t>(e.g) | reinterpret_cast<uintptr_t>(e.master);
            const uintptr_t st = reinterpret_cast<uintptr_t>(e.m) | reinterpret_cast<uintptr_t>(e.v);
            vec = (wide & 31) == 0 && (st & (e.state == HILORE_STATE_F32 ? 31 : 15)) == 0;
            h.lrwd = lr * e.weight_decay;
            const bool coded = (KIND < kMixed ? KIND / 6 : e.state) == HILORE_STATE_E4M3FN;
            h.b2 = coded ? -a.b2 : a.b2;
            h.omb2 = coded ? -a.omb2 : a.omb2;
        }
        const int64_t base = (tile - walk.begin) * kTile;
        const int tiles = vec ? (int)min((e.n - base) / kTile, t1 - tile) : 0; // whole ones of this entry
        const int len = SPLIT > 1 ? kTile / SPLIT : max(tiles, 1) * kTile;
        tile += max(tiles, 1);
        if (KIND < kMixed) {
            run_of_kind<KIND == kMixed ? 0 : KIND>(e, h, base + skip, len, tiles > 0);
        } else {
            switch (e.state * 6 + e.g_dtype * 3 + (e.master ? 2 : e.p_dtype)) {
            case 0: run_of_kind<0>(e, h, base + skip, len, tiles > 0); break;
            case 1: run_of_kind<1>(e, h, base + skip, len, tiles > 0); break;
            case 2: run_of_kind<2>(e, h, base + skip, len, tiles > 0); break;
            case 3: run_of_kind<3>(e, h, base + skip, len, tiles > 0); break;
            case 4: run_of_kind<4>(e, h, base + skip, len, tiles > 0); break;
            case 5: run_of_kind<5>(e, h, base + skip, len, tiles > 0); break;
            case 6: run_of_kind<6>(e, h, base + skip, len, tiles > 0); break;
            case 7: run_of_kind<7>(e, h, base + skip, len, tiles > 0); break;
            case 8: run_of_kind<8>(e, h, base + skip, len, tiles > 0); break;
            case 9: run_of_kind<9>(e, h, base + skip, len, tiles > 0); break;
            case 10: run_of_kind<10>(e, h, base + skip, len, tiles > 0); break;
            default: run_of_kind<11>(e, h, base + skip, len, tiles > 0); break;
            }
        }
    }
}

// Checks a table, counts its tiles and finds its kind; `for_step`: everything, not the gradients alone.
static int check_params(const hilore_param *dev, const hilore_param *host, int32_t n, bool for_step, int64_t &tiles, int &kind)
{
    tiles = 0;
    kind = -1;
    if (n < 0)
        return HILORE_INVALID_ARG;
    if (n == 0)
        return HILORE_OK;
    if (!dev || !host)
        return HILORE_INVALID_ARG;
    if (!aligned(dev, 8))
        return HILORE_ALIGN;
    int status = HILORE_OK;
    for (int32_t i = 0; i < n && status == HILORE_OK; ++i) {
        const hilore_param &e = host[i];
        if (e.n < 0 || (e.g_dtype != HILORE_BF16 && e.g_dtype != HILORE_F32) || (e.n > 0 && !e.g))
            return HILORE_INVALID_ARG;
        if (e.n > ((int64_t)1 << 46) || e.first != tiles)
            return HILORE_SHAPE;
        if (!aligned(e.g, e.g_dtype == HILORE_BF16 ? 2 : 4))
            return HILORE_ALIGN;
        tiles += (e.n + kTile - 1) / kTile;
        if (!for_step)
            continue;
        if ((e.p_dtype != HILORE_BF16 && e.p_dtype != HILORE_F32) || (e.state != HILORE_STATE_F32 && e.state != HILORE_STATE_E4M3FN))
            return HILORE_INVALID_ARG;
        const bool coded = e.state == HILORE_STATE_E4M3FN;
        if (e.n > 0 && (!e.p || !e.m || !e.v || (coded && (!e.m_scale || !e.v_scale))))
            return HILORE_INVALID_ARG;
        if (e.master && e.p_dtype != HILORE_BF16)
            return HILORE_INVALID_ARG;
        if (!aligned(e.p, e.p_dtype == HILORE_BF16 ? 2 : 4) || !aligned(e.master, 4) || !aligned(e.m_scale, 4) || !aligned(e.v_scale, 4))
            return HILORE_ALIGN;
        if (!coded && (!aligned(e.m, 4) || !aligned(e.v, 4)))
            return HILORE_ALIGN;
        if (e.n > 0) kind = kind < 0 || kind == kind_of(e) ? kind_of(e) : kMixed;
    }
    return status;
}

} // namespace hilore

using namespace hilore;

extern "C" size_t hilore_grad_norm_workspace_bytes(void) { return (size_t)kNormMaxGrid * sizeof(double); }

extern "C" int hilore_grad_norm(const hilore_param *params_dev, const hilore_param *params_host, int32_t n_params, double max_norm, float *norm,
                                float *scale, void *workspace, size_t workspace_bytes, void *stream)
{
    int64_t tiles = 0;
    int kind = 0;
    if (!(max_norm >= 0.0) || !workspace || (!norm && !scale))
        return HILORE_INVALID_ARG;
    const int bad = check_params(params_dev, params_host, n_params, false, tiles, kind);
    if (bad)
        return bad;
    if (!aligned(norm, 4) || !aligned(scale, 4) || !aligned(workspace, 16))
        return HILORE_ALIGN;
    if (workspace_bytes < hilore_grad_norm_workspace_bytes())
        return HILORE_WORKSPACE;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int64_t grid = (int64_t)sm_count() * ctas_per_sm(grad_norm_kernel, kOptThreads, 0, 4);
    const int per_warp = tiles_per_warp(tiles);
    const int64_t share = (int64_t)kOptWarps * per_warp;
    if (grid > kNormMaxGrid) grid = kNormMaxGrid;
    if (grid > (tiles + share - 1) / share) grid = (tiles + share - 1) / share;
    double *partial = static_cast<double *>(workspace);
    if (grid > 0 && launch_dependent(grad_norm_kernel, dim3((unsigned)grid), dim3(kOptThreads), 0, st, params_dev, n_params, tiles, per_warp, partial) != cudaSuccess)
        return HILORE_CUDA;
    if (launch_dependent(grad_norm_final_kernel, dim3(1), dim3(kOptThreads), 0, st, partial, (int)grid, max_norm, norm, scale) != cudaSuccess)
        return HILORE_CUDA;
    return cudaGetLastError() == cudaSuccess ? HILORE_OK : HILORE_CUDA;
}

extern "C" int hilore_adamw_step(const hilore_param *params_dev, const hilore_param *params_host, int32_t n_params, double lr, const float *lr_dev,
                                 double beta1, double beta2, double eps, int64_t step, const int64_t *step_dev, const float *grad_scale,
                                 void *stream)
{
    int64_t tiles = 0;
    int kind = 0;
    if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps >= 0.0) || !std::isfinite(lr))
        return HILORE_INVALID_ARG;
    if (!step_dev && step < 1)
        return HILORE_INVALID_ARG;
    const int bad = check_params(params_dev, params_host, n_params, true, tiles, kind);
    if (bad)
        return bad;
    if (!aligned(lr_dev, 4) || !aligned(step_dev, 8) || !aligned(grad_scale, 4))
        return HILORE_ALIGN;
    if (tiles == 0)
        return HILORE_OK;
    const int per_warp = tiles_per_warp(tiles);
    const int split = tiles <= 8 * (int64_t)sm_count() ? 2 : 1;
    const int64_t share = (int64_t)kOptWarps * per_warp, grid = (tiles * split + share - 1) / share;
    if (grid > 0x7FFFFFFF)
        return HILORE_SHAPE;
    AdamArgs a{};
    a.beta1 = beta1;
    a.beta2 = beta2;
    a.b1 = (float)beta1;
    a.omb1 = (float)(1.0 - beta1);
    a.b2 = (float)beta2;
    a.omb2 = (float)(1.0 - beta2);
    a.one = 1.0f;
    a.eps = (float)eps;
    a.lr = (float)lr;
    if (!step_dev) {
        a.inv_bc1 = (float)(1.0 / (1.0 - std::pow(beta1, (double)step)));
        a.rsqrt_bc2 = (float)(1.0 / std::sqrt(1.0 - std::pow(beta2, (double)step)));
    }
    a.lr_dev = lr_dev;
    a.grad_scale = grad_scale;
    a.step_dev = step_dev;
#define HILORE_KINDS(S)                                                                                                                         \
    {adamw_kernel<0, S>, adamw_kernel<1, S>, adamw_kernel<2, S>, adamw_kernel<3, S>,  adamw_kernel<4, S>,  adamw_kernel<5, S>,                   \
     adamw_kernel<6, S>, adamw_kernel<7, S>, adamw_kernel<8, S>, adamw_kernel<9, S>, adamw_kernel<10, S>, adamw_kernel<11, S>, adamw_kernel<kMixed, S>}
    static void (*const kernels[2][kMixed + 1])(const hilore_param *, int, int64_t, int, AdamArgs) = {HILORE_KINDS(1), HILORE_KINDS(2)};
#undef HILORE_KINDS
    if (launch_dependent(kernels[split - 1][kind], dim3((unsigned)grid), dim3(kOptThreads), 0, static_cast<cudaStream_t>(stream), params_dev, n_params, tiles, per_warp, a) !=
        cudaSuccess)
        return HILORE_CUDA;
    return cudaGetLastError() == cudaSuccess ? HILORE_OK : HILORE_CUDA;
}
