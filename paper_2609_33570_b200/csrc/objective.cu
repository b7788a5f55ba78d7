// Losses on token log-probabilities with their gradients: the clipped policy loss and the preference loss.
#include <cmath>

#include "segments.cuh"

namespace hilore {

constexpr int kStats = 5;          // sums that a CTA hands to the final kernel
constexpr int kObjectiveGrid = 2048; // most CTAs that do so

// Sums over the valid tokens of a sequence or of the part of it that lies in one tile.
struct Piece {
    double a, b, n;
};

// Tokens of a tile add to the sequence that they are in; a sequence's end starts anew.
struct SumOp {
    struct Map {
        double a, b;
        int32_t n;
        uint32_t flag; // 1: holds a sequence's end, the sums are those behind it
    };
    typedef Map State;
    static __device__ __forceinline__ Map identity() { return Map{0.0, 0.0, 0, 0u}; }
    static __device__ __forceinline__ Map then(const Map &x, const Map &y)
    {
        if (y.flag) return y;
        return Map{x.a + y.a, x.b + y.b, x.n + y.n, x.flag};
    }
    static __device__ __forceinline__ State apply(const Map &m, const State &s) { return then(s, m); }
};

// Where the sums of a call's sequences lie: of a sequence inside one tile in whole[s]; of one that goes over tiles t .. u in
// tail[t], head[t + 1] .. head[u].
struct Pieces {
    Piece *head, *tail, *whole;

    __device__ __forceinline__ Piece total(const Sequences &q, int s) const
    {
        const int lo = q.bound(s), hi = q.bound(s + 1);
        if (hi <= lo) return Piece{0.0, 0.0, 0.0};
        const int t = lo / kSegTile, u = (hi - 1) / kSegTile;
        if (t == u) return whole[s];
        Piece p = tail[t];
        for (int i = t + 1; i <= u; ++i) {
            p.a += head[i].a;
            p.b += head[i].b;
            p.n += head[i].n;
        }
        return p;
    }
};

struct SumArgs {
    Sequences q;
    const uint8_t *mask;
    const float *x, *minus; // a: sum of x - minus (or of x)
    const float *y, *less;  // b: sum of y - less (or of y)
    Pieces out;
    int vec;
};

// Sums of every sequence over its valid tokens, one tile per CTA.
__global__ void __launch_bounds__(kSegThreads) sequence_sums_kernel(const __grid_constant__ SumArgs a)
{
    using Op = SumOp;
    __shared__ TileShared sh;
    __shared__ Op::Map totals[kSegWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, tile = blockIdx.x;
    grid_dependency_wait();
    grid_dependency_release();
    const int lo = tile * kSegTile, live = a.q.live(), hi = live - lo < kSegTile ? live : lo + kSegTile;
    if (hi <= lo)
        return;
    const int k = lo + tid * kSegEach;
    float x[8], m[8], y[8], l[8];
    const uint32_t valid = load_mask8(a.mask, k, hi, a.vec);
    if (a.x) load8(a.x, k, hi, a.vec, x);
    if (a.minus) load8(a.minus, k, hi, a.vec, m);
    if (a.y && a.y != a.x) load8(a.y, k, hi, a.vec, y);
    if (a.less) load8(a.less, k, hi, a.vec, l);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (!a.x) x[e] = 0.0f;
        if (!a.minus) m[e] = 0.0f;
        if (!a.y) y[e] = 0.0f;
        else if (a.y == a.x) y[e] = x[e];
        if (!a.less) l[e] = 0.0f;
    }
    tile_sequences(a.q, lo, hi, sh);
    const uint32_t ends = block_ends(sh, tid);
    auto add = [&](Op::Map &s, int e) {
        if (!(valid >> e & 1)) return;
        s.a += (double)x[e] - (double)m[e];
        s.b += (double)y[e] - (double)l[e];
        s.n += 1;
    };
    Op::Map mine = Op::identity();
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        add(mine, e);
        if (ends >> e & 1) mine = Op::Map{0.0, 0.0, 0, 1u};
    }
    Op::Map all;
    const Op::Map before = warp_scan<Op>(mine, lane, all);
    if (lane == 31) totals[warp] = all;
    __syncthreads();
    Op::Map s = Op::identity();
    for (int w = 0; w < warp; ++w) s = Op::apply(totals[w], s);
    s = Op::apply(before, s);
    if (ends != 0 || tid == kSegThreads - 1) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            add(s, e);
            if (ends >> e & 1) {
                const int o = a.q.owner(k + e, sh.s0, sh.s1);
                const Piece p{s.a, s.b, (double)s.n};
                if (a.q.bound(o) >= lo) a.out.whole[o] = p;
                else a.out.head[tile] = p;
                s = Op::identity();
            }
        }
        if (tid == kSegThreads - 1 && hi == lo + kSegTile && !(ends >> 7 & 1)) { // goes on in the next tile
            const Piece p{s.a, s.b, (double)s.n};
            if (a.q.bound(sh.s1) >= lo) a.out.tail[tile] = p;
            else a.out.head[tile] = p;
        }
    }
}

// Sums of a CTA's five numbers into its slots, in a fixed order.
__device__ __forceinline__ void put_stats(const double (&v)[kStats], double *slots)
{
    __shared__ double sh[kStats][kSegWarps];
#pragma unroll
    for (int i = 0; i < kStats; ++i) {
        const double t = warp_sum(v[i]);
        if ((threadIdx.x & 31) == 0) sh[i][threadIdx.x >> 5] = t;
    }
    __syncthreads();
    if (threadIdx.x < kStats) {
        double t = 0.0;
        for (int w = 0; w < kSegWarps; ++w) t += sh[threadIdx.x][w];
        slots[threadIdx.x] = t;
    }
}

// The sum over the CTAs' slots, number `i` of it in every lane of warp i.
__device__ __forceinline__ double sum_slots(const double *partials, int ctas, int i)
{
    double t = 0.0;
    for (int c = threadIdx.x & 31; c < ctas; c += 32) t += partials[(size_t)c * kStats + i];
    return warp_sum(t);
}

// ------------------------------------------------------------------ policy loss

// exp(e) - e - 1 without the cancellation at small e: there the Taylor series of it, sum over j of e^(j+2) / (j+2)!, whose
// first term left out at |e| <= 1 is 2 / 13! of the first.
__device__ __forceinline__ float exp_minus_line(float e)
{
    if (fabsf(e) > 1.0f) return expf(e) - e - 1.0f;
    float s = 1.0f / 479001600.0f;
    s = fmaf(s, e, 1.0f / 39916800.0f);
    s = fmaf(s, e, 1.0f / 3628800.0f);
    s = fmaf(s, e, 1.0f / 362880.0f);
    s = fmaf(s, e, 1.0f / 40320.0f);
    s = fmaf(s, e, 1.0f / 5040.0f);
    s = fmaf(s, e, 1.0f / 720.0f);
    s = fmaf(s, e, 1.0f / 120.0f);
    s = fmaf(s, e, 1.0f / 24.0f);
    s = fmaf(s, e, 1.0f / 6.0f);
    s = fmaf(s, e, 0.5f);
    return e * e * s;
}

// What the token kernel needs of a sequence.
struct SequenceCoef {
    float weight; // w of its tokens
    float slope;  // sequence ratios: the policy term's gradient of every token
};

struct PolicyArgs {
    Sequences q;
    const float *logp, *old, *ref, *rollout, *adv, *moments, *grad_loss;
    const uint8_t *mask;
    const int64_t *N_dev;
    double N, clip_low, clip_high, log_low, log_high, log_dual, dual, cap, beta, adv_eps;
    int per_token, sequence_ratio, sequence_mean, kl, vec, tiles;
    Pieces pieces;
    SequenceCoef *coef;
    double *partials;
    int slots_before; // CTAs of the sequence kernel, whose slots come first
    float *omega;
};

__device__ __forceinline__ double inverse_norm(const PolicyArgs &a)
{
    const double N = a.N_dev ? (double)*a.N_dev : a.N;
    return N > 0.0 ? 1.0 / N : 0.0;
}

__device__ __forceinline__ float whitened(const PolicyArgs &a, float A)
{
    return a.moments ? (float)(((double)A - (double)a.moments[0]) / ((double)a.moments[1] + a.adv_eps)) : A;
}

// Weights of the tokens of each sequence, and with ratios of whole sequences the policy term and its gradient, a thread per
// sequence.
__global__ void __launch_bounds__(kSegThreads) policy_sequence_kernel(const __grid_constant__ PolicyArgs a)
{
    grid_dependency_wait();
    grid_dependency_release();
    const double inv = inverse_norm(a), g = a.grad_loss ? (double)*a.grad_loss : 1.0;
    double v[kStats] = {};
    for (int64_t s = (int64_t)blockIdx.x * kSegThreads + threadIdx.x; s < a.q.n_seq; s += (int64_t)gridDim.x * kSegThreads) {
        const Piece p = a.pieces.total(a.q, (int)s);
        SequenceCoef c{0.0f, 0.0f};
        if (p.n > 0.0 && inv > 0.0) {
            const double w = a.sequence_mean ? inv / p.n : inv;
            c.weight = (float)w;
            if (a.sequence_ratio) {
                const double d = p.a / p.n, A = (double)whitened(a, a.adv[s]);
                const double gap = a.rollout ? exp(p.b / p.n) : 1.0, i = gap > a.cap && a.rollout ? a.cap : gap; // NaN stays
                const bool flat = A >= 0.0 ? d > a.log_high : (d < a.log_low || d > a.log_dual);
                double u = exp(d);
                if (flat) u = A >= 0.0 ? 1.0 + a.clip_high : (d < a.log_low ? 1.0 - a.clip_low : a.dual);
                else c.slope = (float)(-w * i * A * u * g);
                v[1] -= p.n * w * i * A * u;
                if (flat && A != 0.0) v[3] += p.n * w;
                v[4] -= w * p.a;
            }
        }
        a.coef[s] = c;
    }
    put_stats(v, a.partials + (size_t)blockIdx.x * kStats);
}

__global__ void __launch_bounds__(kSegThreads) policy_token_kernel(const __grid_constant__ PolicyArgs a)
{
    __shared__ TileShared sh;
    const int tid = threadIdx.x;
    grid_dependency_wait();
    grid_dependency_release();
    const int live = a.q.live();
    const double inv = inverse_norm(a);
    const float g = a.grad_loss ? *a.grad_loss : 1.0f, beta = (float)a.beta;
    const bool by_sequence = a.sequence_ratio || a.sequence_mean;
    const float up = (float)(1.0 + a.clip_high), down = (float)(1.0 - a.clip_low), dual = (float)a.dual, cap = (float)a.cap;
    double v[kStats] = {};
    for (int tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
        const int lo = tile * kSegTile, hi = live - lo < kSegTile ? live : lo + kSegTile;
        if (hi <= lo)
            break;
        const int k = lo + tid * kSegEach;
        uint32_t valid = load_mask8(a.mask, k, hi, a.vec);
        if (!(inv > 0.0)) valid = 0;
        float s[8], o[8], r[8], b[8], A[8];
        load8(a.logp, k, hi, a.vec, s);
        if (!a.sequence_ratio) load8(a.old, k, hi, a.vec, o);
        if (a.ref) load8(a.ref, k, hi, a.vec, r);
        if (a.rollout && !a.sequence_ratio) load8(a.rollout, k, hi, a.vec, b);
        if (a.per_token) load8(a.adv, k, hi, a.vec, A);
        tile_sequences(a.q, lo, hi, sh);
        const uint32_t ends = block_ends(sh, tid);
        float w = (float)inv, slope = 0.0f, As = 0.0f, out[8];
        int next = 0; // the token at which the next sequence's numbers are needed
        if (!by_sequence && a.per_token) next = 8;
        float part[kStats] = {};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            out[e] = 0.0f;
            if (valid >> e & 1) {
                if (next <= e) {
                    const int q = a.q.owner(k + e, sh.s0, sh.s1);
                    if (by_sequence) w = a.coef[q].weight, slope = a.coef[q].slope;
                    if (!a.per_token && !a.sequence_ratio) As = a.adv[q];
                    const uint32_t rest = ends >> e; // this sequence's numbers hold up to its end
                    next = rest ? e + __ffs(rest) : 8;
                }
                float grad = slope;
                if (!a.sequence_ratio) {
                    const double d = (double)s[e] - (double)o[e]; // exact next to a border
                    const float rho = expf((float)d), Ae = whitened(a, a.per_token ? A[e] : As);
                    const bool flat = Ae >= 0.0f ? d > a.log_high : (d < a.log_low || d > a.log_dual);
                    const float gap = a.rollout ? expf(o[e] - b[e]) : 1.0f, wi = a.rollout ? w * (gap > cap ? cap : gap) : w; // NaN stays
                    const float u = !flat ? rho : (Ae >= 0.0f ? up : (d < a.log_low ? down : dual));
                    grad = flat ? 0.0f : -wi * Ae * rho * g;
                    part[1] -= wi * Ae * u;
                    if (flat && Ae != 0.0f) part[3] += w;
                    part[4] += w * (o[e] - s[e]);
                }
                if (a.ref) {
                    const float x = r[e] - s[e];
                    const float line = exp_minus_line(x);
                    const float kl = a.kl == HILORE_KL_K3 ? line : (a.kl == HILORE_KL_K2 ? 0.5f * x * x : -x);
                    const float d = a.kl == HILORE_KL_K3 ? -(fabsf(x) > 1.0f ? expf(x) - 1.0f : line + x) : (a.kl == HILORE_KL_K2 ? -x : 1.0f);
                    if (beta != 0.0f) grad = fmaf(beta * w * g, d, grad);
                    part[2] += w * kl;
                }
                out[e] = grad;
            }
        }
#pragma unroll
        for (int i = 1; i < kStats; ++i) v[i] += (double)part[i];
        store8(a.omega, k, lo, hi, a.vec, out);
        __syncthreads();
    }
    put_stats(v, a.partials + (size_t)(a.slots_before + blockIdx.x) * kStats);
}

// stats: loss, policy term, KL term, share on flat branches, mean of old - new
__global__ void __launch_bounds__(kSegThreads) policy_final_kernel(const double *partials, int ctas, double beta, float *stats)
{
    __shared__ double sums[kStats];
    grid_dependency_wait();
    grid_dependency_release();
    const int warp = threadIdx.x >> 5;
    if (warp < kStats) {
        const double t = sum_slots(partials, ctas, warp);
        if ((threadIdx.x & 31) == 0) sums[warp] = t;
    }
    __syncthreads();
    if (threadIdx.x < kStats) stats[threadIdx.x] = (float)(threadIdx.x == 0 ? (beta != 0.0 ? fma(beta, sums[2], sums[1]) : sums[1]) : sums[threadIdx.x]);
}

// ------------------------------------------------------------------ preference loss

struct PreferenceArgs {
    Sequences q;
    const float *rewards, *grad_loss;
    const uint8_t *mask;
    const int64_t *N_dev;
    double N, beta, margin, margin_reward, smoothing, nll;
    int G, loss, length_mean, vec, tiles, groups, per_cta;
    Pieces pieces;
    double *coef; // [n_seq] gradient of every valid token, before the division by N
    double *partials;
    double *scale; // 1 / N, times the gradient of the loss
    float *scores;
    float *omega;
};

// -ln sigmoid(z) and its derivative
__device__ __forceinline__ void softplus_minus(double z, double &value, double &slope)
{
    const double t = exp(-fabs(z));
    value = log1p(t) + fmax(-z, 0.0);
    slope = z >= 0.0 ? -t / (1.0 + t) : -1.0 / (1.0 + t);
}

// A CTA takes `per_cta` whole groups at a time: scores of their sequences into shared memory, then each sequence against the
// others of its group.
__global__ void __launch_bounds__(kSegThreads) preference_pairs_kernel(const __grid_constant__ PreferenceArgs a)
{
    extern __shared__ double smem[];
    const int room = a.per_cta * a.G;
    double *h = smem, *like = smem + room;             // score, mean log-probability
    double *per = smem + 2 * room;                     // 1 / |T| (0: no valid token)
    float *R = reinterpret_cast<float *>(smem + 3 * room);
    grid_dependency_wait();
    grid_dependency_release();
    double v[kStats] = {}; // loss, right order, gap, nll, pairs
    for (int64_t first = (int64_t)blockIdx.x * a.per_cta; first < a.groups; first += (int64_t)gridDim.x * a.per_cta) {
        const int n = (int)(a.groups - first < a.per_cta ? a.groups - first : a.per_cta) * a.G;
        const int64_t base = first * a.G;
        for (int i = threadIdx.x; i < n; i += kSegThreads) {
            const Piece p = a.pieces.total(a.q, (int)(base + i));
            const double inv = p.n > 0.0 ? 1.0 / p.n : 0.0;
            h[i] = p.n > 0.0 ? a.beta * (a.length_mean ? p.a / p.n : p.a) : 0.0;
            like[i] = p.n > 0.0 ? p.b / p.n : 0.0;
            per[i] = inv;
            R[i] = a.rewards[base + i];
            if (a.scores) a.scores[base + i] = (float)h[i];
        }
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += kSegThreads) {
            const int begin = i / a.G * a.G;
            const double hi = h[i];
            const float Ri = R[i];
            double c = 0.0;
            int wins = 0;
            if (per[i] > 0.0)
                for (int j = begin; j < begin + a.G; ++j) {
                    const float Rj = R[j];
                    if (!(per[j] > 0.0) || !(Ri > Rj || Rj > Ri)) continue;
                    const bool won = Ri > Rj;
                    const double gap = won ? hi - h[j] : h[j] - hi;
                    const double more = a.margin_reward != 0.0 ? a.margin_reward * (won ? (double)Ri - (double)Rj : (double)Rj - (double)Ri) : 0.0;
                    const double z = gap - a.margin - more;
                    double value, slope;
                    if (a.loss == HILORE_PREF_SIGMOID) {
                        softplus_minus(z, value, slope);
                        if (a.smoothing != 0.0) value += a.smoothing * z; // -ln sigmoid(-z) = z - ln sigmoid(z)
                        slope += a.smoothing;
                    } else if (a.loss == HILORE_PREF_HINGE) {
                        value = z >= 1.0 ? 0.0 : 1.0 - z;
                        slope = z >= 1.0 ? 0.0 : (z < 1.0 ? -1.0 : z);
                    } else {
                        const double t = (z - 0.5) / a.beta;
                        value = t * t;
                        slope = 2.0 * t / a.beta;
                    }
                    c += won ? slope : -slope;
                    if (won) {
                        ++wins;
                        v[0] += value;
                        if (gap > 0.0) v[1] += 1.0;
                        v[2] += gap;
                    }
                }
            v[3] -= wins * like[i];
            v[4] += wins;
            c *= a.length_mean ? a.beta * per[i] : a.beta;
            a.coef[base + i] = wins ? c - a.nll * wins * per[i] : c;
        }
        __syncthreads();
    }
    put_stats(v, a.partials + (size_t)blockIdx.x * kStats);
}

// stats: loss, share of pairs in the right order, mean gap of the scores, mean -log-probability per token of the winners
__global__ void __launch_bounds__(kSegThreads) preference_final_kernel(const __grid_constant__ PreferenceArgs a, int ctas, int64_t *pairs, float *stats)
{
    __shared__ double sums[kStats];
    grid_dependency_wait();
    grid_dependency_release();
    const int warp = threadIdx.x >> 5;
    if (warp < kStats) {
        const double t = sum_slots(a.partials, ctas, warp);
        if ((threadIdx.x & 31) == 0) sums[warp] = t;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        const double N = a.N_dev ? (double)*a.N_dev : (a.N > 0.0 ? a.N : sums[4]);
        const double inv = N > 0.0 ? 1.0 / N : 0.0;
        *a.scale = inv * (a.grad_loss ? (double)*a.grad_loss : 1.0);
        if (pairs) *pairs = (int64_t)sums[4];
        if (stats) {
            const bool none = !(inv > 0.0) || sums[4] == 0.0;
            stats[0] = none ? 0.0f : (float)((sums[0] + (a.nll != 0.0 ? a.nll * sums[3] : 0.0)) * inv);
            for (int i = 1; i < 4; ++i) stats[i] = none ? 0.0f : (float)(sums[i] * inv);
        }
    }
}

// The gradient of a sequence to each of its valid tokens.
__global__ void __launch_bounds__(kSegThreads) preference_token_kernel(const __grid_constant__ PreferenceArgs a)
{
    __shared__ TileShared sh;
    const int tid = threadIdx.x;
    grid_dependency_wait();
    grid_dependency_release();
    const int tile = blockIdx.x, lo = tile * kSegTile, live = a.q.live(), hi = live - lo < kSegTile ? live : lo + kSegTile;
    if (hi <= lo)
        return;
    const int k = lo + tid * kSegEach;
    const uint32_t valid = load_mask8(a.mask, k, hi, a.vec);
    const double scale = *a.scale;
    tile_sequences(a.q, lo, hi, sh);
    const uint32_t ends = block_ends(sh, tid);
    float out[8], c = 0.0f;
    int next = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        out[e] = 0.0f;
        if (valid >> e & 1) {
            if (next <= e) {
                c = scale != 0.0 ? (float)(a.coef[a.q.owner(k + e, sh.s0, sh.s1)] * scale) : 0.0f;
                const uint32_t rest = ends >> e;
                next = rest ? e + __ffs(rest) : 8;
            }
            out[e] = c;
        }
    }
    store8(a.omega, k, lo, hi, a.vec, out);
}

constexpr int kMaxGroup = 1024;

// Layout of a workspace: the CTAs' slots, the pieces of tiles and sequences, a number per sequence, one number.
struct Workspace {
    size_t partials, head, tail, whole, coef, scale, bytes;
};
static Workspace layout(int64_t n_seq, int64_t n_tok)
{
    Workspace w;
    const size_t tiles = n_tok > 0 ? (size_t)((n_tok + kSegTile - 1) / kSegTile) : 0, S = n_seq > 0 ? (size_t)n_seq : 0;
    w.partials = 0;
    w.head = w.partials + sizeof(double) * kStats * 2 * kObjectiveGrid;
    w.tail = w.head + sizeof(Piece) * tiles;
    w.whole = w.tail + sizeof(Piece) * tiles;
    w.coef = w.whole + sizeof(Piece) * S;
    w.scale = w.coef + sizeof(double) * S;
    w.bytes = w.scale + 16;
    return w;
}

static Pieces pieces_of(void *workspace, const Workspace &w)
{
    unsigned char *p = static_cast<unsigned char *>(workspace);
    return Pieces{reinterpret_cast<Piece *>(p + w.head), reinterpret_cast<Piece *>(p + w.tail), reinterpret_cast<Piece *>(p + w.whole)};
}

static int grid_of(int64_t work, int64_t most) { return (int)(work < 1 ? 1 : (work < most ? work : most)); }

} // namespace hilore

using namespace hilore;

extern "C" size_t hilore_policy_loss_workspace_bytes(int64_t n_seq, int64_t n_tok) { return layout(n_seq, n_tok).bytes; }
extern "C" size_t hilore_preference_loss_workspace_bytes(int64_t n_seq, int64_t n_tok) { return layout(n_seq, n_tok).bytes; }

extern "C" int hilore_policy_loss(const float *logp, const float *logp_old, const float *logp_ref, const float *logp_rollout,
                                  const uint8_t *mask, const float *adv, const float *adv_moments, const int32_t *cu_seqlens,
                                  int64_t n_seq, int64_t n_tok, const hilore_policy_terms *terms, int64_t N_norm,
                                  const int64_t *N_norm_dev, const float *grad_loss, float *stats, float *omega, void *workspace,
                                  size_t workspace_bytes, void *stream)
{
    PolicyArgs a{};
    if (!terms || !workspace || !stats)
        return HILORE_INVALID_ARG;
    const hilore_policy_terms &t = *terms;
    if (!(t.clip_low >= 0.0 && t.clip_low <= 1.0) || !(t.clip_high >= 0.0) || !(t.dual_clip == 0.0 || t.dual_clip >= 1.0) ||
        !std::isfinite(t.beta) || !(t.rollout_cap > 0.0) || !(t.adv_eps >= 0.0) || !std::isfinite(t.adv_eps))
        return HILORE_INVALID_ARG;
    if ((t.ratio != HILORE_RATIO_TOKEN && t.ratio != HILORE_RATIO_SEQUENCE) || (t.mean != HILORE_MEAN_TOKENS && t.mean != HILORE_MEAN_SEQUENCES) ||
        t.kl < HILORE_KL_K1 || t.kl > HILORE_KL_K3 || (t.adv_per_token != 0 && t.adv_per_token != 1) ||
        (t.adv_per_token && t.ratio == HILORE_RATIO_SEQUENCE))
        return HILORE_INVALID_ARG;
    const int bad = check_sequences(cu_seqlens, n_seq, n_tok, a.q);
    if (bad)
        return bad;
    a.tiles = (int)((n_tok + kSegTile - 1) / kSegTile);
    if (n_tok > 0 && (!logp || !logp_old || !adv || !omega || (t.beta != 0.0 && !logp_ref)))
        return HILORE_INVALID_ARG;
    if (!N_norm_dev && N_norm <= 0)
        return HILORE_ZERO_NORM;
    for (const float *p : {logp, logp_old, logp_ref, logp_rollout, adv, adv_moments, grad_loss, (const float *)stats, (const float *)omega})
        if (!aligned(p, 4)) return HILORE_ALIGN;
    if (!aligned(N_norm_dev, 8) || !aligned(workspace, 16))
        return HILORE_ALIGN;
    const Workspace w = layout(n_seq, n_tok);
    if (workspace_bytes < w.bytes)
        return HILORE_WORKSPACE;
    a.logp = logp, a.old = logp_old, a.ref = logp_ref, a.rollout = logp_rollout, a.adv = adv, a.moments = adv_moments, a.grad_loss = grad_loss;
    a.mask = mask, a.N_dev = N_norm_dev, a.N = (double)N_norm, a.clip_low = t.clip_low, a.clip_high = t.clip_high;
    a.log_low = std::log1p(-t.clip_low), a.log_high = std::log1p(t.clip_high);
    a.dual = t.dual_clip != 0.0 ? t.dual_clip : INFINITY, a.log_dual = std::log(a.dual), a.cap = t.rollout_cap, a.beta = t.beta, a.adv_eps = t.adv_eps;
    a.per_token = t.adv_per_token, a.sequence_ratio = t.ratio == HILORE_RATIO_SEQUENCE, a.sequence_mean = t.mean == HILORE_MEAN_SEQUENCES, a.kl = t.kl;
    a.vec = vectors({logp, logp_old, logp_ref, logp_rollout, a.per_token ? adv : nullptr, omega}, mask);
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    a.pieces = pieces_of(workspace, w);
    a.coef = reinterpret_cast<SequenceCoef *>(ws + w.coef);
    a.partials = reinterpret_cast<double *>(ws + w.partials);
    a.omega = omega;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int ctas = 0;
    if (a.tiles > 0 && (a.sequence_ratio || a.sequence_mean)) {
        SumArgs s{};
        s.q = a.q, s.mask = mask, s.out = a.pieces, s.vec = a.vec;
        if (a.sequence_ratio) s.x = logp, s.minus = logp_old;
        if (a.sequence_ratio && logp_rollout) s.y = logp_old, s.less = logp_rollout;
        if (launch_dependent(sequence_sums_kernel, dim3((unsigned)a.tiles), dim3(kSegThreads), 0, st, s) != cudaSuccess)
            return HILORE_CUDA;
        ctas = grid_of((n_seq + kSegThreads - 1) / kSegThreads, kObjectiveGrid);
        if (launch_dependent(policy_sequence_kernel, dim3((unsigned)ctas), dim3(kSegThreads), 0, st, a) != cudaSuccess)
            return HILORE_CUDA;
    }
    if (a.tiles > 0) {
        a.slots_before = ctas;
        int64_t most = (int64_t)sm_count() * ctas_per_sm(policy_token_kernel, kSegThreads, 0, 4);
        if (most > kObjectiveGrid) most = kObjectiveGrid;
        const int grid = grid_of(a.tiles, most);
        if (launch_dependent(policy_token_kernel, dim3((unsigned)grid), dim3(kSegThreads), 0, st, a) != cudaSuccess)
            return HILORE_CUDA;
        ctas += grid;
    }
    if (launch_dependent(policy_final_kernel, dim3(1), dim3(kSegThreads), 0, st, (const double *)a.partials, ctas, a.beta, stats) != cudaSuccess)
        return HILORE_CUDA;
    return cudaGetLastError() == cudaSuccess ? HILORE_OK : HILORE_CUDA;
}

extern "C" int hilore_preference_loss(const float *logp, const float *logp_ref, const uint8_t *mask, const float *rewards, int32_t G,
                                      const int32_t *cu_seqlens, int64_t n_seq, int64_t n_tok, const hilore_preference_terms *terms,
                                      int64_t N_norm, const int64_t *N_norm_dev, const float *grad_loss, float *scores, int64_t *pairs,
                                      float *stats, float *omega, void *workspace, size_t workspace_bytes, void *stream)
{
    PreferenceArgs a{};
    if (!terms || !workspace || !stats || G < 1)
        return HILORE_INVALID_ARG;
    const hilore_preference_terms &t = *terms;
    if (!(t.beta > 0.0) || !std::isfinite(t.beta) || !std::isfinite(t.margin) || !std::isfinite(t.margin_reward) || !std::isfinite(t.nll) ||
        !(t.smoothing >= 0.0 && t.smoothing <= 1.0) || t.loss < HILORE_PREF_SIGMOID || t.loss > HILORE_PREF_SQUARE ||
        (t.length_mean != 0 && t.length_mean != 1) || (t.smoothing != 0.0 && t.loss != HILORE_PREF_SIGMOID))
        return HILORE_INVALID_ARG;
    const int bad = check_sequences(cu_seqlens, n_seq, n_tok, a.q);
    if (bad)
        return bad;
    a.tiles = (int)((n_tok + kSegTile - 1) / kSegTile);
    if (n_seq % G != 0 || G > kMaxGroup)
        return HILORE_SHAPE;
    if ((n_tok > 0 && (!logp || !omega)) || (n_seq > 0 && !rewards))
        return HILORE_INVALID_ARG;
    if (!N_norm_dev && N_norm < 0)
        return HILORE_ZERO_NORM;
    for (const float *p : {logp, logp_ref, rewards, grad_loss, (const float *)scores, (const float *)stats, (const float *)omega})
        if (!aligned(p, 4)) return HILORE_ALIGN;
    if (!aligned(N_norm_dev, 8) || !aligned(pairs, 8) || !aligned(workspace, 16))
        return HILORE_ALIGN;
    const Workspace w = layout(n_seq, n_tok);
    if (workspace_bytes < w.bytes)
        return HILORE_WORKSPACE;
    a.rewards = rewards, a.grad_loss = grad_loss, a.mask = mask, a.N_dev = N_norm_dev, a.N = (double)N_norm, a.beta = t.beta, a.margin = t.margin;
    a.margin_reward = t.margin_reward, a.smoothing = t.smoothing, a.nll = t.nll, a.G = G, a.loss = t.loss, a.length_mean = t.length_mean;
    a.vec = vectors({logp, logp_ref, omega}, mask);
    a.groups = (int)(n_seq / G);
    a.per_cta = G >= kSegThreads ? 1 : kSegThreads / G;
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    a.pieces = pieces_of(workspace, w);
    a.coef = reinterpret_cast<double *>(ws + w.coef);
    a.partials = reinterpret_cast<double *>(ws + w.partials);
    a.scale = reinterpret_cast<double *>(ws + w.scale);
    a.scores = scores;
    a.omega = omega;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int ctas = 0;
    if (a.tiles > 0) {
        SumArgs s{};
        s.q = a.q, s.mask = mask, s.out = a.pieces, s.vec = a.vec, s.x = logp, s.minus = logp_ref, s.y = logp;
        if (launch_dependent(sequence_sums_kernel, dim3((unsigned)a.tiles), dim3(kSegThreads), 0, st, s) != cudaSuccess)
            return HILORE_CUDA;
    }
    if (a.groups > 0) {
        ctas = grid_of((a.groups + a.per_cta - 1) / a.per_cta, kObjectiveGrid);
        const size_t smem = (size_t)a.per_cta * G * (3 * sizeof(double) + sizeof(float));
        if (launch_dependent(preference_pairs_kernel, dim3((unsigned)ctas), dim3(kSegThreads), smem, st, a) != cudaSuccess)
            return HILORE_CUDA;
    }
    if (launch_dependent(preference_final_kernel, dim3(1), dim3(kSegThreads), 0, st, a, ctas, pairs, stats) != cudaSuccess)
        return HILORE_CUDA;
    if (a.tiles > 0 && launch_dependent(preference_token_kernel, dim3((unsigned)a.tiles), dim3(kSegThreads), 0, st, a) != cudaSuccess)
        return HILORE_CUDA;
    return cudaGetLastError() == cudaSuccess ? HILORE_OK : HILORE_CUDA;
}
