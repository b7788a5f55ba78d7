// Advantages and returns by a gated linear recurrence over the valid tokens of a sequence, and the backward pass of it.
#include <cmath>

#include "segments.cuh"

namespace hilore {

// From the last valid token of a sequence on, with x the advantage of the following valid token and q its discounted value:
//     A = (r - V) + q + w x,   w = gamma lambda c;      then x = A, q = gamma V
// and behind the last one x = 0, q = gamma bootstrap + outcome.  Over a run of tokens that is
//     x' = P x + Q q + B,   q' = c
// which composes.  All of it in fp64: sums over a hundred thousand tokens, powers of weights next to one.
struct AdvantageOp {
    struct Map {
        double P, Q, B, c;
        uint32_t flag, pad; // 0: no valid token, the state passes; 1: as above; 2: holds a sequence's end, x' = B, q' = c
    };
    struct State {
        double x, q;
    };
    static __device__ __forceinline__ Map identity() { return Map{1.0, 0.0, 0.0, 0.0, 0u, 0u}; }
    static __device__ __forceinline__ State start() { return State{0.0, 0.0}; }
    static __device__ __forceinline__ Map then(const Map &a, const Map &b)
    {
        if (b.flag == 2 || a.flag == 0) return b;
        if (b.flag == 0) return a;
        return Map{b.P * a.P, b.P * a.Q, fma(b.P, a.B, fma(b.Q, a.c, b.B)), b.c, a.flag, 0u};
    }
    static __device__ __forceinline__ State apply(const Map &m, const State &s)
    {
        if (m.flag == 0) return s;
        if (m.flag == 2) return State{m.B, m.c};
        return State{fma(m.P, s.x, fma(m.Q, s.q, m.B)), m.c};
    }
};

// From the first valid token of a sequence on, with y = w G of the valid token before and G its gradient:
//     G' = g + y,  y' = w G'
// over a run of tokens  G' = P y + B,  y' = wl G'.  `pos` is the run's last valid token, -1 for none since the sequence began.
struct AdvantageGradOp {
    struct Map {
        double P, B, wl;
        int32_t pos;
        uint32_t flag; // as above; 2: holds a sequence's start
    };
    struct State {
        double y, G;
        int32_t pos, pad;
    };
    static __device__ __forceinline__ Map identity() { return Map{1.0, 0.0, 0.0, -1, 0u}; }
    static __device__ __forceinline__ State start() { return State{0.0, 0.0, -1, 0}; }
    static __device__ __forceinline__ Map then(const Map &a, const Map &b)
    {
        if (b.flag == 2 || a.flag == 0) return b;
        if (b.flag == 0) return a;
        const double k = b.P * a.wl;
        return Map{k * a.P, fma(k, a.B, b.B), b.wl, b.pos, a.flag};
    }
    static __device__ __forceinline__ State apply(const Map &m, const State &s)
    {
        if (m.flag == 0) return s;
        const double G = m.flag == 2 ? m.B : fma(m.P, s.y, m.B);
        return State{m.wl * G, G, m.pos, 0};
    }
};

struct AdvantageArgs {
    Sequences q;
    const float *rewards, *outcome, *bootstrap, *trace;
    const void *values;
    int values_bf16;
    const uint8_t *mask;
    double gamma, weight; // gamma lambda
    float *adv, *returns;
    const float *grad_adv, *grad_returns, *adv_in;
    float *grad_rewards, *grad_outcome, *grad_values, *grad_bootstrap, *grad_trace;
    void *maps;       // [tiles] maps of whole tiles
    double *partials; // [tiles][3] count, mean, sum of squared deviations
    int tiles, vec, moments;
};

// The state that comes into tile `tile`: back over the tiles before it (`dir` away) to the one that holds the end of a sequence,
// then forward again, one map after the other, so that the bits do not depend on where the walk began.  By one warp; every
// lane returns it.
template <typename Op> __device__ typename Op::State state_into(const typename Op::Map *maps, int tile, int tiles, int dir, int lane)
{
    using Map = typename Op::Map;
    typename Op::State s = Op::start();
    int far = tile;
    for (;;) {
        const int t = far + dir * (lane + 1);
        const bool in = t >= 0 && t < tiles;
        const uint32_t stop = __ballot_sync(0xFFFFFFFFu, !in || maps[in ? t : 0].flag == 2);
        if (stop) {
            far += dir * __ffs(stop);
            break;
        }
        far += dir * 32;
    }
    // far: a tile with a sequence's end, or one step past the last tile
    const int n = (far - tile) * dir; // tiles tile + dir .. far
    for (int done = 0; done < n; done += 32) {
        const int k = n - done < 32 ? n - done : 32;
        const int t = far - dir * (done + lane);
        Map m = Op::identity();
        if (lane < k && t >= 0 && t < tiles) m = maps[t];
        for (int j = 0; j < k; ++j) s = Op::apply(shfl_words(m, j), s);
    }
    return s;
}

struct Moments { // count, mean and sum of squared deviations of a set of values
    double n, mean, m2;
    __device__ __forceinline__ void join(const Moments &o)
    {
        const double all = n + o.n;
        if (o.n == 0.0) return;
        if (n == 0.0) {
            *this = o;
            return;
        }
        const double d = o.mean - mean, f = o.n / all;
        mean = fma(d, f, mean);
        m2 += o.m2 + d * d * n * f;
        n = all;
    }
};

__device__ __forceinline__ Moments warp_join(Moments m)
{
#pragma unroll
    for (int by = 1; by < 32; by *= 2) {
        Moments o;
        o.n = __shfl_down_sync(0xFFFFFFFFu, m.n, by);
        o.mean = __shfl_down_sync(0xFFFFFFFFu, m.mean, by);
        o.m2 = __shfl_down_sync(0xFFFFFFFFu, m.m2, by);
        m.join(o); // lane 0 has all of them in the end; what others have is not used
    }
    return m;
}

// One tile of 2048 tokens per CTA, the last tokens in the first threads.  MAPS: write the tile's map alone.  Otherwise the outputs,
// with the maps of the other tiles complete.
template <bool MAPS> __global__ void __launch_bounds__(kSegThreads) advantage_kernel(const __grid_constant__ AdvantageArgs a)
{
    using Op = AdvantageOp;
    __shared__ TileShared sh;
    __shared__ Op::Map totals[kSegWarps];
    __shared__ Op::State incoming;
    __shared__ Moments moments[kSegWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, tile = blockIdx.x;
    grid_dependency_wait();
    grid_dependency_release();
    const int lo = tile * kSegTile, live = a.q.live(), hi = live - lo < kSegTile ? live : lo + kSegTile;
    if (hi <= lo) { // behind the last sequence
        if (tid == 0) {
            if (MAPS) static_cast<Op::Map *>(a.maps)[tile] = Op::identity();
            else if (a.moments)
                for (int i = 0; i < 3; ++i) a.partials[3 * tile + i] = 0.0;
        }
        return;
    }
    const int block = kSegThreads - 1 - tid, k = lo + block * kSegEach;
    float r[8], v[8], c[8];
    const uint32_t valid = load_mask8(a.mask, k, hi, a.vec);
    if (a.rewards) load8(a.rewards, k, hi, a.vec, r);
    if (a.values) {
        if (a.values_bf16) load8(static_cast<const uint16_t *>(a.values), k, hi, a.vec, v);
        else load8(static_cast<const float *>(a.values), k, hi, a.vec, v);
    }
    if (a.trace) load8(a.trace, k, hi, a.vec, c);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (!a.rewards) r[e] = 0.0f;
        if (!a.values) v[e] = 0.0f;
        if (!a.trace) c[e] = 1.0f;
    }
    tile_sequences(a.q, lo, hi, sh);
    const uint32_t ends = block_ends(sh, block);
    auto terminal = [&](int p) -> double {
        if (!a.outcome && !a.bootstrap) return 0.0;
        const int s = a.q.owner(p, sh.s0, sh.s1);
        return (a.outcome ? (double)a.outcome[s] : 0.0) + a.gamma * (a.bootstrap ? (double)a.bootstrap[s] : 0.0);
    };
    Op::Map mine = Op::identity();
#pragma unroll
    for (int e = 7; e >= 0; --e) {
        if (ends >> e & 1) mine = Op::Map{0.0, 0.0, 0.0, terminal(k + e), 2u, 0u};
        if (valid >> e & 1) {
            const double w = a.weight * (double)c[e], d = (double)r[e] - (double)v[e], q = a.gamma * (double)v[e];
            if (mine.flag == 0) mine = Op::Map{w, 1.0, d, q, 1u, 0u};
            else mine = Op::Map{w * mine.P, w * mine.Q, fma(w, mine.B, d + mine.c), q, mine.flag, 0u};
        }
    }
    Op::Map all;
    const Op::Map before = warp_scan<Op>(mine, lane, all);
    if (lane == 31) totals[warp] = all;
    if (MAPS) {
        __syncthreads();
        if (tid == 0) {
            Op::Map m = totals[0];
            for (int w = 1; w < kSegWarps; ++w) m = Op::then(m, totals[w]);
            static_cast<Op::Map *>(a.maps)[tile] = m;
        }
        return;
    }
    if (warp == 0) {
        const Op::State s = state_into<Op>(static_cast<const Op::Map *>(a.maps), tile, a.tiles, 1, lane);
        if (lane == 0) incoming = s;
    }
    __syncthreads();
    Op::State s = incoming;
    for (int w = 0; w < warp; ++w) s = Op::apply(totals[w], s);
    s = Op::apply(before, s);
    float adv[8], ret[8];
    double n = 0.0, shift = 0.0, sum = 0.0, squares = 0.0; // moments about the thread's first value
#pragma unroll
    for (int e = 7; e >= 0; --e) {
        adv[e] = ret[e] = 0.0f;
        if (ends >> e & 1) s = Op::State{0.0, terminal(k + e)};
        if (valid >> e & 1) {
            const double w = a.weight * (double)c[e], V = v[e];
            s.x = fma(w, s.x, ((double)r[e] - V) + s.q);
            s.q = a.gamma * V;
            adv[e] = (float)s.x;
            ret[e] = (float)(s.x + V);
            if (a.moments) {
                if (n == 0.0) shift = s.x;
                const double d = s.x - shift;
                n += 1.0;
                sum += d;
                squares = fma(d, d, squares);
            }
        }
    }
    if (a.adv) store8(a.adv, k, hi, a.vec, adv);
    if (a.returns) store8(a.returns, k, hi, a.vec, ret);
    if (a.moments) {
        Moments m{n, n > 0.0 ? shift + sum / n : 0.0, n > 0.0 ? squares - sum * sum / n : 0.0};
        m = warp_join(m);
        if (lane == 0) moments[warp] = m;
        __syncthreads();
        if (tid == 0) {
            for (int w = 1; w < kSegWarps; ++w) m.join(moments[w]);
            a.partials[3 * tile] = m.n;
            a.partials[3 * tile + 1] = m.mean;
            a.partials[3 * tile + 2] = m.m2;
        }
    }
}

__global__ void __launch_bounds__(kSegThreads) advantage_moments_kernel(const double *partials, int tiles, float *moments)
{
    __shared__ Moments sh[kSegWarps];
    grid_dependency_wait();
    grid_dependency_release();
    Moments m{0.0, 0.0, 0.0};
    for (int t = threadIdx.x; t < tiles; t += kSegThreads) m.join(Moments{partials[3 * t], partials[3 * t + 1], partials[3 * t + 2]});
    m = warp_join(m);
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = m;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kSegWarps; ++w) m.join(sh[w]);
        moments[0] = (float)m.mean;
        moments[1] = m.n > 0.0 ? (float)sqrt(fmax(m.m2 / m.n, 0.0) + (m.m2 - m.m2)) : 0.0f; // NaN stays
    }
}

template <bool MAPS> __global__ void __launch_bounds__(kSegThreads) advantage_grad_kernel(const __grid_constant__ AdvantageArgs a)
{
    using Op = AdvantageGradOp;
    __shared__ TileShared sh;
    __shared__ Op::Map totals[kSegWarps];
    __shared__ Op::State incoming;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, tile = blockIdx.x;
    grid_dependency_wait();
    grid_dependency_release();
    const int lo = tile * kSegTile, live = a.q.live(), hi = live - lo < kSegTile ? live : lo + kSegTile;
    const bool per_sequence = a.grad_outcome || a.grad_bootstrap;
    if (hi <= lo) { // behind the last sequence; sequences without a token have no gradient
        if (MAPS && tid == 0) static_cast<Op::Map *>(a.maps)[tile] = Op::identity();
        if (!MAPS && per_sequence && tile == 0)
            for (int64_t s = tid; s < a.q.n_seq; s += kSegThreads) {
                if (a.grad_outcome) a.grad_outcome[s] = 0.0f;
                if (a.grad_bootstrap) a.grad_bootstrap[s] = 0.0f;
            }
        return;
    }
    const int k = lo + tid * kSegEach;
    float ga[8], gr[8], c[8], A[8];
    const uint32_t valid = load_mask8(a.mask, k, hi, a.vec);
    if (a.grad_adv) load8(a.grad_adv, k, hi, a.vec, ga);
    if (a.grad_returns) load8(a.grad_returns, k, hi, a.vec, gr);
    if (a.trace) load8(a.trace, k, hi, a.vec, c);
    if (!MAPS && a.grad_trace) load8(a.adv_in, k, hi, a.vec, A);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (!a.grad_adv) ga[e] = 0.0f;
        if (!a.grad_returns) gr[e] = 0.0f;
        if (!a.trace) c[e] = 1.0f;
    }
    tile_sequences(a.q, lo, hi, sh);
    const uint32_t ends = block_ends(sh, tid);
    Op::Map mine = Op::identity();
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (valid >> e & 1) {
            const double w = a.weight * (double)c[e], g = (double)ga[e] + (double)gr[e];
            if (mine.flag == 0) mine = Op::Map{1.0, g, w, k + e, 1u};
            else mine = Op::Map{mine.wl * mine.P, fma(mine.wl, mine.B, g), w, k + e, mine.flag};
        }
        if (ends >> e & 1) mine = Op::Map{0.0, 0.0, 0.0, -1, 2u};
    }
    Op::Map all;
    const Op::Map before = warp_scan<Op>(mine, lane, all);
    if (lane == 31) totals[warp] = all;
    if (MAPS) {
        __syncthreads();
        if (tid == 0) {
            Op::Map m = totals[0];
            for (int w = 1; w < kSegWarps; ++w) m = Op::then(m, totals[w]);
            static_cast<Op::Map *>(a.maps)[tile] = m;
        }
        return;
    }
    if (warp == 0) {
        Op::State s = state_into<Op>(static_cast<const Op::Map *>(a.maps), tile, a.tiles, -1, lane);
        if (lane == 0) incoming = s;
    }
    __syncthreads();
    Op::State s = incoming;
    for (int w = 0; w < warp; ++w) s = Op::apply(totals[w], s);
    s = Op::apply(before, s);
    float dr[8], dv[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        dr[e] = dv[e] = 0.0f;
        if (valid >> e & 1) {
            const double w = a.weight * (double)c[e], G = ((double)ga[e] + (double)gr[e]) + s.y;
            if (a.grad_trace && s.pos >= 0) a.grad_trace[s.pos] = (float)(a.weight * (double)A[e] * s.G);
            dr[e] = (float)G;
            dv[e] = (float)(fma(a.gamma, s.G, (double)gr[e]) - G);
            s = Op::State{w * G, G, k + e, 0};
        } else if (a.grad_trace && k + e < hi) {
            a.grad_trace[k + e] = 0.0f;
        }
        if (ends >> e & 1) {
            if (a.grad_trace && s.pos >= 0) a.grad_trace[s.pos] = 0.0f; // nothing follows
            if (per_sequence) {
                const int o = a.q.owner(k + e, sh.s0, sh.s1);
                if (a.grad_outcome) a.grad_outcome[o] = (float)s.G;
                if (a.grad_bootstrap) a.grad_bootstrap[o] = (float)(a.gamma * s.G);
            }
            s = Op::start();
        }
    }
    if (a.grad_rewards) store8(a.grad_rewards, k, hi, a.vec, dr);
    if (a.grad_values) store8(a.grad_values, k, hi, a.vec, dv);
    if (per_sequence) { // sequences without a token, from this tile's first sequence to the next tile's (or from and to the ends)
        __shared__ int next;
        __syncthreads();
        if (warp == 0) {
            const int o = hi < live ? a.q.owner_warp(hi, lane) : (int)a.q.n_seq - 1;
            if (lane == 0) next = o;
        }
        __syncthreads();
        for (int64_t o = (tile == 0 ? 0 : sh.s0) + tid; o <= next; o += kSegThreads)
            if (a.q.bound((int)o + 1) <= a.q.bound((int)o)) {
                if (a.grad_outcome) a.grad_outcome[o] = 0.0f;
                if (a.grad_bootstrap) a.grad_bootstrap[o] = 0.0f;
            }
    }
}

static bool all_vectors(const AdvantageArgs &a)
{
    return vectors({a.rewards, a.trace, a.adv, a.returns, a.grad_adv, a.grad_returns, a.adv_in, a.grad_rewards, a.grad_values, a.grad_trace}, a.mask) &&
           aligned(a.values, a.values_bf16 ? 16 : 32);
}

} // namespace hilore

using namespace hilore;

extern "C" size_t hilore_advantages_workspace_bytes(int64_t n_tok)
{
    const size_t tiles = n_tok > 0 ? (size_t)((n_tok + kSegTile - 1) / kSegTile) : 0;
    return (tiles + 1) * (sizeof(AdvantageOp::Map) + 3 * sizeof(double));
}

extern "C" int hilore_advantages(const float *rewards, const float *outcome, const void *values, int32_t values_dtype, const float *bootstrap,
                                 const float *trace, const uint8_t *mask, const int32_t *cu_seqlens, int64_t n_seq, int64_t n_tok,
                                 double gamma, double lambda, float *adv, float *returns, float *moments, void *workspace,
                                 size_t workspace_bytes, void *stream)
{
    AdvantageArgs a{};
    if (!(gamma >= 0.0 && gamma <= 1.0) || !(lambda >= 0.0 && lambda <= 1.0) || (values_dtype != HILORE_BF16 && values_dtype != HILORE_F32))
        return HILORE_INVALID_ARG;
    const int bad = check_sequences(cu_seqlens, n_seq, n_tok, a.q, a.tiles);
    if (bad)
        return bad;
    if (!workspace || (n_tok > 0 && !adv && !returns && !moments))
        return HILORE_INVALID_ARG;
    a.rewards = rewards, a.outcome = outcome, a.values = values, a.values_bf16 = values_dtype == HILORE_BF16, a.bootstrap = bootstrap;
    a.trace = trace, a.mask = mask, a.gamma = gamma, a.weight = gamma * lambda, a.adv = adv, a.returns = returns, a.moments = moments != nullptr;
    if (!aligned(rewards, 4) || !aligned(outcome, 4) || !aligned(bootstrap, 4) || !aligned(trace, 4) || !aligned(adv, 4) || !aligned(returns, 4) ||
        !aligned(moments, 4) || !aligned(values, a.values_bf16 ? 2 : 4) || !aligned(workspace, 16))
        return HILORE_ALIGN;
    if (workspace_bytes < hilore_advantages_workspace_bytes(n_tok))
        return HILORE_WORKSPACE;
    a.maps = workspace;
    a.partials = reinterpret_cast<double *>(static_cast<AdvantageOp::Map *>(workspace) + a.tiles + 1);
    a.vec = all_vectors(a);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (a.tiles > 1 && launch_dependent(advantage_kernel<true>, dim3((unsigned)a.tiles), dim3(kSegThreads), 0, st, a) != cudaSuccess)
        return HILORE_CUDA;
    if (a.tiles > 0 && launch_dependent(advantage_kernel<false>, dim3((unsigned)a.tiles), dim3(kSegThreads), 0, st, a) != cudaSuccess)
        return HILORE_CUDA;
    if (moments && launch_dependent(advantage_moments_kernel, dim3(1), dim3(kSegThreads), 0, st, (const double *)a.partials, a.tiles, moments) != cudaSuccess)
        return HILORE_CUDA;
    return cudaGetLastError() == cudaSuccess ? HILORE_OK : HILORE_CUDA;
}

extern "C" int hilore_advantages_backward(const float *grad_adv, const float *grad_returns, const float *adv, const float *trace,
                                          const uint8_t *mask, const int32_t *cu_seqlens, int64_t n_seq, int64_t n_tok, double gamma,
                                          double lambda, float *grad_rewards, float *grad_outcome, float *grad_values, float *grad_bootstrap,
                                          float *grad_trace, void *workspace, size_t workspace_bytes, void *stream)
{
    AdvantageArgs a{};
    if (!(gamma >= 0.0 && gamma <= 1.0) || !(lambda >= 0.0 && lambda <= 1.0))
        return HILORE_INVALID_ARG;
    const int bad = check_sequences(cu_seqlens, n_seq, n_tok, a.q, a.tiles);
    if (bad)
        return bad;
    if (!workspace || (grad_trace && !adv && n_tok > 0))
        return HILORE_INVALID_ARG;
    a.grad_adv = grad_adv, a.grad_returns = grad_returns, a.adv_in = grad_trace ? adv : nullptr, a.trace = trace, a.mask = mask;
    a.gamma = gamma, a.weight = gamma * lambda, a.grad_rewards = grad_rewards, a.grad_outcome = grad_outcome, a.grad_values = grad_values;
    a.grad_bootstrap = grad_bootstrap, a.grad_trace = grad_trace;
    for (const float *p : {grad_adv, grad_returns, adv, trace, (const float *)grad_rewards, (const float *)grad_outcome, (const float *)grad_values,
                           (const float *)grad_bootstrap, (const float *)grad_trace})
        if (!aligned(p, 4)) return HILORE_ALIGN;
    if (!aligned(workspace, 16))
        return HILORE_ALIGN;
    if (workspace_bytes < hilore_advantages_workspace_bytes(n_tok))
        return HILORE_WORKSPACE;
    a.maps = workspace;
    a.vec = all_vectors(a);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (n_seq == 0)
        return HILORE_OK;
    const unsigned grid = (unsigned)(a.tiles > 0 ? a.tiles : 1);
    if (a.tiles > 1 && launch_dependent(advantage_grad_kernel<true>, dim3(grid), dim3(kSegThreads), 0, st, a) != cudaSuccess)
        return HILORE_CUDA;
    if (launch_dependent(advantage_grad_kernel<false>, dim3(grid), dim3(kSegThreads), 0, st, a) != cudaSuccess)
        return HILORE_CUDA;
    return cudaGetLastError() == cudaSuccess ? HILORE_OK : HILORE_CUDA;
}
