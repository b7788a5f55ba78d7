// OptimizerStep of the actor update: the global gradient norm and the AdamW step over all tensors of a table, one launch
// for the whole table.  Moments are fp32, or 8 bits in the library's block format (E4M3FN codes, one fp32 scale per 64).
//
// Both are streams of a few bytes and a few operations per element: HBM is the bound.  A warp owns a tile of 1024
// consecutive elements of one tensor and finds that tensor by a 32-ary search over the table's `first` column (two
// dependent loads for a thousand tensors), so tensors of any size share one launch without a map of tiles.
#include "common.cuh"

#include <cmath>

namespace hilore {

constexpr int kTile = HILORE_PARAM_TILE; // elements of a warp's tile
constexpr int kOptThreads = 256, kOptWarps = kOptThreads / 32;
constexpr int kNormMaxGrid = 2048; // partial sums in the workspace
constexpr float kE4m3Max = 448.0f, kE4m3Min = 0.001953125f; // largest and smallest positive value

__device__ __forceinline__ float load_one(const void *p, int32_t dtype, int64_t i)
{
    return dtype == HILORE_BF16 ? __uint_as_float((uint32_t)static_cast<const uint16_t *>(p)[i] << 16) : static_cast<const float *>(p)[i];
}

__device__ __forceinline__ void store_one(void *p, int32_t dtype, int64_t i, float v)
{
    if (dtype == HILORE_BF16) static_cast<uint16_t *>(p)[i] = (uint16_t)cvt_bf16x2(0.0f, v);
    else static_cast<float *>(p)[i] = v;
}

// Eight consecutive values from element i on (a multiple of 8), `n` of them real; vectors where the tensor allows it.
__device__ __forceinline__ void load8(const void *p, int32_t dtype, int64_t i, int n, bool vec, float (&x)[8])
{
    if (vec && n == 8) {
        if (dtype == HILORE_BF16) {
            const uint4 w = ld_global_128_stream(static_cast<const uint16_t *>(p) + i);
            const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                x[2 * k] = bf16_lo(u[k]);
                x[2 * k + 1] = bf16_hi(u[k]);
            }
        } else {
            uint32_t w[8];
            ld_global_256(static_cast<const float *>(p) + i, w);
#pragma unroll
            for (int k = 0; k < 8; ++k)
                x[k] = __uint_as_float(w[k]);
        }
        return;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
        x[k] = k < n ? load_one(p, dtype, i + k) : 0.0f;
}

__device__ __forceinline__ void store8(void *p, int32_t dtype, int64_t i, int n, bool vec, const float (&x)[8])
{
    if (vec && n == 8) {
        if (dtype == HILORE_BF16) {
            uint4 w;
            w.x = cvt_bf16x2(x[1], x[0]);
            w.y = cvt_bf16x2(x[3], x[2]);
            w.z = cvt_bf16x2(x[5], x[4]);
            w.w = cvt_bf16x2(x[7], x[6]);
            *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(p) + i) = w;
        } else {
            uint32_t w[8];
#pragma unroll
            for (int k = 0; k < 8; ++k)
                w[k] = __float_as_uint(x[k]);
            st_global_256(static_cast<float *>(p) + i, w);
        }
        return;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (k < n) store_one(p, dtype, i + k, x[k]);
}

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

// ------------------------------------------------------------------------------------------------------------------- norm
// Squares in fp32 over the 32 elements of a lane's tile, fp64 beyond; a lane whose fp32 sum leaves the range redoes its
// elements in fp64.  Partial sums in fixed slots: the result does not depend on scheduling.
__global__ void __launch_bounds__(kOptThreads) grad_norm_kernel(const hilore_param *params, int n_params, int64_t n_tiles, double *partial)
{
    const int lane = threadIdx.x & 31;
    double sum = 0.0;
    for (int64_t tile = (int64_t)blockIdx.x * kOptWarps + (threadIdx.x >> 5); tile < n_tiles; tile += (int64_t)gridDim.x * kOptWarps) {
        const hilore_param &e = params[owner_of(params, n_params, tile)];
        const void *g = e.g;
        const int32_t dtype = e.g_dtype;
        const int64_t base = (tile - e.first) * kTile, n = e.n;
        const bool vec = (reinterpret_cast<uintptr_t>(g) & 31) == 0;
        float x[kTile / 256][8], s = 0.0f;
#pragma unroll
        for (int k = 0; k < kTile / 256; ++k) {
            const int64_t i = base + k * 256 + lane * 8;
            load8(g, dtype, i, (int)max((int64_t)0, min((int64_t)8, n - i)), vec, x[k]);
        }
#pragma unroll
        for (int k = 0; k < kTile / 256; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                s = fmaf(x[k][i], x[k][i], s);
        if (s < INFINITY) {
            sum += (double)s;
        } else {
#pragma unroll
            for (int k = 0; k < kTile / 256; ++k)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    sum += (double)x[k][i] * (double)x[k][i];
        }
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
    float b1, omb1, b2, omb2, eps; // omb = 1 - beta, rounded once
    float lr, inv_bc1, rsqrt_bc2;  // 1 / (1 - beta1^t), 1 / sqrt(1 - beta2^t) where t is known on the host
    const float *lr_dev, *grad_scale;
    const int64_t *step_dev;
};

struct AdamStep {
    float lr, step, rsqrt_bc2; // step = lr / (1 - beta1^t)
};

// The moments, every operation rounded by itself in the order of the formula.  With 8-bit states the last bit decides the
// codes of values near a tie, and a code of the next step's largest value moves the scale of 64 elements: contracted
// operations would make them depend on the compiler.
__device__ __forceinline__ float next_m(const AdamArgs &a, float m, float g) { return __fadd_rn(__fmul_rn(a.b1, m), __fmul_rn(a.omb1, g)); }
__device__ __forceinline__ float next_v(const AdamArgs &a, float v, float g)
{
    return __fadd_rn(__fmul_rn(a.b2, v), __fmul_rn(__fmul_rn(a.omb2, g), g));
}

// One step of a 32-bit lane of eight elements.
__device__ __forceinline__ void adam_f32(const hilore_param &e, const AdamArgs &a, const AdamStep &h, float gscale, int64_t i, int n, bool vec)
{
    float g[8], m[8], v[8], p[8];
    load8(e.g, e.g_dtype, i, n, vec, g);
    load8(e.m, HILORE_F32, i, n, vec, m);
    load8(e.v, HILORE_F32, i, n, vec, v);
    if (e.master) load8(e.master, HILORE_F32, i, n, vec, p);
    else load8(e.p, e.p_dtype, i, n, vec, p);
    const float lrwd = h.lr * e.weight_decay;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const float x = __fmul_rn(g[k], gscale);
        m[k] = next_m(a, m[k], x);
        v[k] = next_v(a, v[k], x);
        const float den = fmaf(__fsqrt_rn(v[k]), h.rsqrt_bc2, a.eps);
        p[k] -= fmaf(lrwd, p[k], h.step * __fdiv_rn(m[k], den));
    }
    store8(e.m, HILORE_F32, i, n, vec, m);
    store8(e.v, HILORE_F32, i, n, vec, v);
    if (e.master) store8(e.master, HILORE_F32, i, n, vec, p);
    store8(e.p, e.p_dtype, i, n, vec, p);
}

__device__ __forceinline__ void load_codes(const uint8_t *c, int64_t i, int n, bool vec, float s, float (&x)[16])
{
    uint32_t w[4] = {0, 0, 0, 0};
    if (vec && n == 16) {
        const uint4 q = ld_global_128_stream(c + i);
        w[0] = q.x, w[1] = q.y, w[2] = q.z, w[3] = q.w;
    } else {
#pragma unroll
        for (int k = 0; k < 16; ++k)
            if (k < n) w[k >> 2] |= (uint32_t)c[i + k] << (8 * (k & 3));
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t lo = cvt_e4m3x2_to_f16x2(w[k]), hi = cvt_e4m3x2_to_f16x2(w[k] >> 16);
        x[4 * k] = f16_lo_to_f32(lo) * s;
        x[4 * k + 1] = f16_hi_to_f32(lo) * s;
        x[4 * k + 2] = f16_lo_to_f32(hi) * s;
        x[4 * k + 3] = f16_hi_to_f32(hi) * s;
    }
}

__device__ __forceinline__ void store_codes(uint8_t *c, int64_t i, int n, bool vec, const float (&q)[16])
{
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
        w[k] = cvt_e4m3x4(q[4 * k], q[4 * k + 1], q[4 * k + 2], q[4 * k + 3]);
    if (vec && n == 16) {
        *reinterpret_cast<uint4 *>(c + i) = make_uint4(w[0], w[1], w[2], w[3]);
        return;
    }
#pragma unroll
    for (int k = 0; k < 16; ++k)
        if (k < n) c[i + k] = (uint8_t)(w[k >> 2] >> (8 * (k & 3)));
}

// Largest finite magnitude of a block of 64: 16 values of each of the four lanes of a quad.
__device__ __forceinline__ float block_max(const float (&x)[16])
{
    float a = 0.0f;
#pragma unroll
    for (int k = 0; k < 16; ++k)
        a = fmaxf(a, fabsf(x[k]));
    a = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, 1));
    a = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, 2));
    if (__any_sync(0xFFFFFFFFu, a == INFINITY)) { // fmaxf passes over NaN but not over Inf
        a = 0.0f;
#pragma unroll
        for (int k = 0; k < 16; ++k)
            a = fabsf(x[k]) < INFINITY ? fmaxf(a, fabsf(x[k])) : a;
        a = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, 1));
        a = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, 2));
    }
    return a;
}

__device__ __forceinline__ void load16(const void *p, int32_t dtype, int64_t i, int n, bool vec, float (&x)[16])
{
    float lo[8], hi[8];
    load8(p, dtype, i, min(n, 8), vec, lo);
    load8(p, dtype, i + 8, max(n - 8, 0), vec, hi);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        x[k] = lo[k];
        x[8 + k] = hi[k];
    }
}

__device__ __forceinline__ void store16(void *p, int32_t dtype, int64_t i, int n, bool vec, const float (&x)[16])
{
    float lo[8], hi[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        lo[k] = x[k];
        hi[k] = x[8 + k];
    }
    store8(p, dtype, i, min(n, 8), vec, lo);
    store8(p, dtype, i + 8, max(n - 8, 0), vec, hi);
}

// One step of a lane of sixteen elements with 8-bit moments.  The four lanes of a quad own one block of 64; the moments of
// this step enter the update in fp32, before they are rounded to codes.  v holds the codes of sqrt(v): the square root
// halves the range that the codes have to span, and a positive root is never rounded to zero (it would turn the next
// step's division into one by eps), it takes the smallest code instead.
__device__ __forceinline__ void adam_e4m3(const hilore_param &e, const AdamArgs &a, const AdamStep &h, float gscale, int64_t i, int n, bool vec)
{
    const int lane = threadIdx.x & 31;
    float g[16], m[16], r[16], p[16];
    const bool some = n > 0;
    uint8_t *mc = static_cast<uint8_t *>(e.m), *vc = static_cast<uint8_t *>(e.v);
    load16(e.g, e.g_dtype, i, n, vec, g);
    load_codes(mc, i, n, vec, some ? e.m_scale[i >> 6] : 0.0f, m);
    load_codes(vc, i, n, vec, some ? e.v_scale[i >> 6] : 0.0f, r);
    if (e.master) load16(e.master, HILORE_F32, i, n, vec, p);
    else load16(e.p, e.p_dtype, i, n, vec, p);
    const float lrwd = h.lr * e.weight_decay;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        const float x = __fmul_rn(g[k], gscale);
        m[k] = next_m(a, m[k], x);
        r[k] = __fsqrt_rn(next_v(a, __fmul_rn(r[k], r[k]), x));
        const float den = fmaf(r[k], h.rsqrt_bc2, a.eps);
        p[k] -= fmaf(lrwd, p[k], h.step * __fdividef(m[k], den));
    }
    if (e.master) store16(e.master, HILORE_F32, i, n, vec, p);
    store16(e.p, e.p_dtype, i, n, vec, p);
    const float am = block_max(m), ar = block_max(r);
    float ms = __fmul_rn(am, 1.0f / kE4m3Max), mi = __fmul_rn(kE4m3Max, __frcp_rn(am));
    float rs = __fmul_rn(ar, 1.0f / kE4m3Max), ri = __fmul_rn(kE4m3Max, __frcp_rn(ar));
    if (!(mi < INFINITY)) ms = mi = 1.0f; // nothing finite but zeros, or too small to be scaled
    float least = kE4m3Min;
    if (!(ri < INFINITY)) {
        rs = ri = 1.0f;
        least = 0.0f;
    }
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        m[k] = __fmul_rn(m[k], mi);
        const float x = __fmul_rn(r[k], ri);
        r[k] = x > 0.0f ? fmaxf(x, least) : x;
    }
    store_codes(mc, i, n, vec, m);
    store_codes(vc, i, n, vec, r);
    if ((lane & 3) == 0 && some) {
        e.m_scale[i >> 6] = ms;
        e.v_scale[i >> 6] = rs;
    }
}

__global__ void __launch_bounds__(kOptThreads) adamw_kernel(const hilore_param *params, int n_params, int64_t n_tiles, AdamArgs a)
{
    const int lane = threadIdx.x & 31;
    const int64_t tile = (int64_t)blockIdx.x * kOptWarps + (threadIdx.x >> 5);
    if (tile >= n_tiles)
        return;
    const float gscale = a.grad_scale ? *a.grad_scale : 1.0f;
    if (!(fabsf(gscale) < INFINITY)) // the gradients are not finite: parameters and moments stay as they are
        return;
    AdamStep h;
    h.lr = a.lr_dev ? *a.lr_dev : a.lr;
    float inv_bc1 = a.inv_bc1;
    h.rsqrt_bc2 = a.rsqrt_bc2;
    if (a.step_dev) {
        const double t = (double)*a.step_dev;
        inv_bc1 = (float)(1.0 / -expm1(t * log(a.beta1)));
        h.rsqrt_bc2 = (float)rsqrt(-expm1(t * log(a.beta2)));
    }
    h.step = h.lr * inv_bc1;
    const hilore_param e = params[owner_of(params, n_params, tile)];
    const int64_t base = (tile - e.first) * kTile;
    const uintptr_t wide = reinterpret_cast<uintptr_t>(e.p) | reinterpret_cast<uintptr_t>(e.g) | reinterpret_cast<uintptr_t>(e.master);
    const uintptr_t st = reinterpret_cast<uintptr_t>(e.m) | reinterpret_cast<uintptr_t>(e.v);
    if (e.state == HILORE_STATE_F32) {
        const bool vec = ((wide | st) & 31) == 0;
#pragma unroll 1
        for (int k = 0; k < kTile / 256; ++k) {
            const int64_t i = base + k * 256 + lane * 8;
            const int n = (int)max((int64_t)0, min((int64_t)8, e.n - i));
            if (n > 0) adam_f32(e, a, h, gscale, i, n, vec);
        }
    } else {
        const bool vec = (wide & 31) == 0 && (st & 15) == 0;
#pragma unroll 1
        for (int k = 0; k < kTile / 512; ++k) { // all lanes together: blocks are reduced by shuffles
            const int64_t i = base + k * 512 + lane * 16;
            const int n = (int)max((int64_t)0, min((int64_t)16, e.n - i));
            adam_e4m3(e, a, h, gscale, i, n, vec);
        }
    }
}

// Checks a table and counts its tiles; `for_step`: everything, not the gradients alone.
static int check_params(const hilore_param *dev, const hilore_param *host, int32_t n, bool for_step, int64_t &tiles)
{
    tiles = 0;
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
    if (!(max_norm >= 0.0) || !workspace || (!norm && !scale))
        return HILORE_INVALID_ARG;
    const int bad = check_params(params_dev, params_host, n_params, false, tiles);
    if (bad)
        return bad;
    if (!aligned(norm, 4) || !aligned(scale, 4) || !aligned(workspace, 16))
        return HILORE_ALIGN;
    if (workspace_bytes < hilore_grad_norm_workspace_bytes())
        return HILORE_WORKSPACE;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int64_t grid = (int64_t)sm_count() * ctas_per_sm(grad_norm_kernel, kOptThreads, 0, 4);
    if (grid > kNormMaxGrid) grid = kNormMaxGrid;
    if (grid > (tiles + kOptWarps - 1) / kOptWarps) grid = (tiles + kOptWarps - 1) / kOptWarps;
    double *partial = static_cast<double *>(workspace);
    if (grid > 0) grad_norm_kernel<<<(unsigned)grid, kOptThreads, 0, st>>>(params_dev, n_params, tiles, partial);
    grad_norm_final_kernel<<<1, kOptThreads, 0, st>>>(partial, (int)grid, max_norm, norm, scale);
    return cudaGetLastError() == cudaSuccess ? HILORE_OK : HILORE_CUDA;
}

extern "C" int hilore_adamw_step(const hilore_param *params_dev, const hilore_param *params_host, int32_t n_params, double lr, const float *lr_dev,
                                 double beta1, double beta2, double eps, int64_t step, const int64_t *step_dev, const float *grad_scale,
                                 void *stream)
{
    int64_t tiles = 0;
    if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps >= 0.0) || !std::isfinite(lr))
        return HILORE_INVALID_ARG;
    if (!step_dev && step < 1)
        return HILORE_INVALID_ARG;
    const int bad = check_params(params_dev, params_host, n_params, true, tiles);
    if (bad)
        return bad;
    if (!aligned(lr_dev, 4) || !aligned(step_dev, 8) || !aligned(grad_scale, 4))
        return HILORE_ALIGN;
    if (tiles == 0)
        return HILORE_OK;
    const int64_t grid = (tiles + kOptWarps - 1) / kOptWarps;
    if (grid > 0x7FFFFFFF)
        return HILORE_SHAPE;
    AdamArgs a{};
    a.beta1 = beta1;
    a.beta2 = beta2;
    a.b1 = (float)beta1;
    a.omb1 = (float)(1.0 - beta1);
    a.b2 = (float)beta2;
    a.omb2 = (float)(1.0 - beta2);
    a.eps = (float)eps;
    a.lr = (float)lr;
    if (!step_dev) {
        a.inv_bc1 = (float)(1.0 / (1.0 - std::pow(beta1, (double)step)));
        a.rsqrt_bc2 = (float)(1.0 / std::sqrt(1.0 - std::pow(beta2, (double)step)));
    }
    a.lr_dev = lr_dev;
    a.grad_scale = grad_scale;
    a.step_dev = step_dev;
    adamw_kernel<<<(unsigned)grid, kOptThreads, 0, static_cast<cudaStream_t>(stream)>>>(params_dev, n_params, tiles, a);
    return cudaGetLastError() == cudaSuccess ? HILORE_OK : HILORE_CUDA;
}
