// Losses on token log-probabilities with their gradients: the clipped policy loss and the preference loss.
#include <cooperative_groups.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdlib>

#include "segments.cuh"

namespace cg = cooperative_groups;

namespace hilore {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kPerSm = 2;            // CTAs of the policy kernels on an SM,
constexpr int kSumsPerSm = 4;        // of the sums',
constexpr int kSumsPerSmOfFour = 2;  // and of those of four tensors, which need the registers
constexpr int kStats = 5;            // sums that a CTA hands on
constexpr int kMostCtas = 1024;      // that do so
constexpr uint32_t kAll = 0xFFFFFFFFu;

// Every warp has a share of neighbouring blocks of 256 tokens, eight to a lane; all of them run at once.
struct Share {
    int blocks, per_warp; // blocks of the call, of a warp
};

// Sums over the valid tokens of a sequence or of the part of it that lies in one share.
struct Piece {
    double a, b, n;
};

// Where the sums of a call's sequences lie: of a sequence inside one share in whole[s]; of one that goes over shares t .. u in
// tail[t], head[t + 1] .. head[u].
struct Pieces {
    Piece *head, *tail, *whole;
    int share; // tokens

    // By one thread, unless the sequence goes over more than `most` shares: then n is -1.
    __device__ __forceinline__ Piece total(const Sequences &q, int s, int most = 0x7FFFFFFF) const
    {
        const int lo = q.bound(s), hi = q.bound(s + 1);
        if (hi <= lo) return Piece{0.0, 0.0, 0.0};
        const int t = lo / share, u = (hi - 1) / share;
        if (t == u) return whole[s];
        if (u - t >= most) return Piece{0.0, 0.0, -1.0};
        Piece p = tail[t];
#pragma unroll 4
        for (int i = t + 1; i <= u; ++i) {
            p.a += head[i].a;
            p.b += head[i].b;
            p.n += head[i].n;
        }
        return p;
    }
    // By a warp; every lane returns it.
    __device__ __forceinline__ Piece total_warp(const Sequences &q, int s, int lane) const
    {
        const int lo = q.bound(s), hi = q.bound(s + 1);
        if (hi <= lo) return Piece{0.0, 0.0, 0.0};
        const int t = lo / share, u = (hi - 1) / share;
        if (t == u) return whole[s];
        Piece p{0.0, 0.0, 0.0};
#pragma unroll 4
        for (int i = t + lane; i <= u; i += 32) {
            const Piece x = i == t ? tail[i] : head[i];
            p.a += x.a;
            p.b += x.b;
            p.n += x.n;
        }
        return Piece{warp_sum(p.a), warp_sum(p.b), warp_sum(p.n)};
    }
};

// A warp's way through the sequences of its tokens: the current one, which holds the first token not yet passed, and its end.  Lane i knows
// where sequence first + i ends, so that the next one is most often found without a load.
struct Cursor {
    int s, end, first, ends;
    // The window of 32 sequences from s on.
    __device__ __forceinline__ void fill(const Sequences &q, int lane)
    {
        first = s;
        ends = (int64_t)s + lane < q.n_seq ? q.bound(s + lane + 1) : 0x7FFFFFFF;
    }
    __device__ __forceinline__ void at(const Sequences &q, int token, int lane)
    {
        s = q.owner_warp(token, lane);
        fill(q, lane);
        end = __shfl_sync(kAll, ends, 0);
    }
    // On to the sequence of `token`, which is not in this one but behind it.  Whether the window is another one.
    __device__ __forceinline__ bool on(const Sequences &q, int token, int lane)
    {
        const uint32_t hit = __ballot_sync(kAll, ends > token);
        if (hit) {
            const int j = __ffs(hit) - 1;
            s = (int)((int64_t)first + j < q.n_seq ? first + j : q.n_seq - 1);
            end = __shfl_sync(kAll, ends, j);
        } else {
            at(q, token, lane);
        }
        if (end <= token) end = 0x7FFFFFFF; // boundaries out of order
        return hit == 0;
    }
    // How many sequences of the window end before token hi, from this one on; 32: perhaps more.
    __device__ __forceinline__ int inside(int hi, int lane) const
    {
        const uint32_t in = __ballot_sync(kAll, ends < hi && lane >= s - first);
        return in >> 31 ? 32 : __popc(in);
    }
    // Where so many end that every lane walks those of its own eight tokens: the sequence of token hi - 1, or one before it.
    __device__ __forceinline__ int ahead(const Sequences &q, int hi, int lane) const
    {
        const uint32_t out = __ballot_sync(kAll, ends >= hi && lane >= s - first);
        return out ? first + __ffs(out) - 1 : q.owner_warp(hi - 1, lane);
    }
    // On to the sequence of token k, no further than `last`.
    __device__ __forceinline__ bool spread(const Sequences &q, int k, int last)
    {
        if (k < end) return false;
        s = q.owner(k, s, last);
        end = q.bound(s + 1);
        if (end <= k) end = 0x7FFFFFFF;
        return true;
    }
    __device__ __forceinline__ void next(const Sequences &q, int last) // to the one that begins where this one ends
    {
        const int token = end;
        if (s < last) ++s;
        end = q.bound(s + 1);
        if (end <= token) s = q.owner(token, s, last), end = q.bound(s + 1);
        if (end <= token) end = 0x7FFFFFFF;
    }
    __device__ __forceinline__ void join(const Sequences &q, int from, int lane) // the cursor of lane `from` is everyone's
    {
        s = __shfl_sync(kAll, s, from);
        end = __shfl_sync(kAll, end, from);
        fill(q, lane);
    }
};
// Sequences that end in a block are taken one after the other up to this many, from the window (sums: with a reduction each).  Where more do,
// all lanes walk those of their own tokens at the same time, and one lane adds up the shares of a long sequence behind them (500 K tokens behind twenty
// sequences of three, means of sequences: 134 us for 17 without the twenty).  Policy loss of 40000 sequences of 25 and 100 tokens with 4, 8, 16: 30, 30, 27 and 54,
// 47, 47 us; their preference loss with 1, 3, 8 in the sums: 25, 25, 30 and 46, 46, 47 us.
constexpr int kFew = 16, kFewSums = 3;

// Sums since the last end of a sequence, if there is one.
struct SumOp {
    struct Map {
        double a, b, n;
        uint32_t flag, pad;
    };
    static __device__ __forceinline__ Map identity() { return Map{0.0, 0.0, 0.0, 0u, 0u}; }
    static __device__ __forceinline__ Map then(const Map &a, const Map &b)
    {
        return b.flag ? b : Map{a.a + b.a, a.b + b.b, a.n + b.n, a.flag, 0u};
    }
};

struct SumArgs {
    Sequences q;
    Share w;
    const uint8_t *mask;
    const float *x, *minus; // a: sum of x - minus (or of x)
    const float *y, *less;  // b: sum of y - less (or of y); y may be x
    Pieces out;
    unsigned *done; // opt: a counter that the next kernel wants at zero
    int vec;
};

// Sums of every sequence over its valid tokens, in fp64.  X: whether there is a first sum, Y: 0 none, 1 of y - less, 2 of x.  A lane adds its tokens
// of the current sequence; at the sequence's end, or the share's, the warp adds the lanes up, so that no sum depends on scheduling.  Bound by memory
// where it has two tensors and a mask to read: 50 M tokens 82 us (4.8 TB/s of what is not masked).
template <bool X, int Y>
__global__ void __launch_bounds__(kThreads, Y == 1 ? kSumsPerSmOfFour : kSumsPerSm) sequence_sums_kernel(const __grid_constant__ SumArgs a)
{
    grid_dependency_wait();
    grid_dependency_release();
    if (a.done && blockIdx.x == 0 && threadIdx.x == 0) *a.done = 0;
    const int lane = threadIdx.x & 31, share = blockIdx.x * kWarps + (threadIdx.x >> 5);
    const int live = a.q.live(), tokens = a.w.per_warp * kBlock;
    if ((int64_t)share * tokens >= live)
        return;
    const int begin = share * tokens, stop = min(live - begin, tokens) + begin;
    Cursor c{0, 0x7FFFFFFF, 0, 0};
    Piece sum{0.0, 0.0, 0.0};
    int n = 0;
    bool opened = true; // whether the current sequence begins in the share
    auto finish = [&](bool ends) {
        const Piece p{X ? warp_sum(sum.a) : 0.0, Y ? warp_sum(sum.b) : 0.0, (double)__reduce_add_sync(kAll, (unsigned)n)};
        if (lane == 0) {
            if (!opened) a.out.head[share] = p;
            else if (ends) a.out.whole[c.s] = p;
            else a.out.tail[share] = p;
        }
        opened = true;
        sum = Piece{0.0, 0.0, 0.0};
        n = 0;
    };
    // a block's tensors are asked for while the block before is added up, its mask one block earlier
    constexpr int kX = X ? 8 : 1, kY = Y == 1 ? 8 : 1;
    struct {
        uint32_t valid;
        float x[kX], m[kX], y[kY], l[kY];
    } now{}, then{};
    Mask8 mask;
    auto ask = [&](auto &to, int base) { // with the block's mask read
        const int k = base + lane * 8, hi = min(base + kBlock, stop);
        to.valid = base < stop ? mask.bits(k, hi) : 0u;
        mask.read(a.mask, k + kBlock, stop, a.vec);
        if (to.valid == 0) return;
        if constexpr (X) {
            load8(a.x, k, hi, a.vec, to.x);
            if (a.minus) load8(a.minus, k, hi, a.vec, to.m);
        }
        if constexpr (Y == 1) {
            load8(a.y, k, hi, a.vec, to.y);
            if (a.less) load8(a.less, k, hi, a.vec, to.l);
        }
    };
    mask.read(a.mask, begin + lane * 8, stop, a.vec);
    ask(now, begin);
    c.at(a.q, begin, lane); // while the first block is on its way
    opened = a.q.bound(c.s) >= begin;
#pragma unroll 1
    for (int base = begin; base < stop; base += kBlock) {
        const int k = base + lane * 8, hi = min(base + kBlock, stop);
        const uint32_t valid = now.valid;
        ask(then, base + kBlock);
        if (c.end < hi && c.inside(hi, lane) > kFewSums) {
            const int last = c.ahead(a.q, hi, lane);
            const Piece before{X ? warp_sum(sum.a) : 0.0, Y ? warp_sum(sum.b) : 0.0, (double)__reduce_add_sync(kAll, (unsigned)n)};
            SumOp::Map mine = SumOp::identity(), first = mine, all; // since the last end in the lane's tokens; before the first
            int s_first = 0;
            if (k < hi) c.spread(a.q, k, last);
#pragma unroll 1
            for (int e = 0; k + e < hi && e < 8; ++e) { // read once more, as registers for it would cost all blocks
                if (valid >> e & 1) {
                    const double x = X ? (double)a.x[k + e] : 0.0;
                    if (X) mine.a += a.minus ? x - (double)a.minus[k + e] : x;
                    if (Y == 1) mine.b += (double)a.y[k + e] - (a.less ? (double)a.less[k + e] : 0.0);
                    if (Y == 2) mine.b += x;
                    mine.n += 1.0;
                }
                if (k + e + 1 < c.end) continue;
                if (mine.flag) a.out.whole[c.s] = Piece{mine.a, mine.b, mine.n};
                else first = mine, s_first = c.s;
                mine = SumOp::Map{0.0, 0.0, 0.0, 1u, 0u};
                if (e < 7 && k + e + 1 < hi) c.next(a.q, last);
            }
            __syncwarp();
            SumOp::Map in = warp_scan<SumOp>(mine, lane, all);
            if (!in.flag) in.a += before.a, in.b += before.b, in.n += before.n;
            if (mine.flag) {
                const Piece p{in.a + first.a, in.b + first.b, in.n + first.n};
                if (a.q.bound(s_first) < begin) a.out.head[share] = p;
                else a.out.whole[s_first] = p;
            }
            all = shfl_words(all, 31); // an end is in it
            sum = lane == 0 ? Piece{all.a, all.b, 0.0} : Piece{0.0, 0.0, 0.0};
            n = lane == 0 ? (int)all.n : 0;
            c.join(a.q, (hi - 1 - base) >> 3, lane);
            if (c.end <= hi) {
                if (c.end >= stop) return;
                c.on(a.q, hi, lane);
            }
            opened = true;
        } else {
#pragma unroll 1
            for (int lo = base;;) { // the block's part of each sequence
                const uint32_t run = c.end >= hi && lo == base ? valid : valid & range_bits(k, lo, c.end);
                if (__all_sync(kAll, run == 0xFFu)) {
#pragma unroll
                    for (int e = 0; e < 8; e += 2) {
                        if constexpr (X) sum.a += ((double)now.x[e] - (double)now.m[e]) + ((double)now.x[e + 1] - (double)now.m[e + 1]);
                        if constexpr (Y == 1) sum.b += ((double)now.y[e] - (double)now.l[e]) + ((double)now.y[e + 1] - (double)now.l[e + 1]);
                        if constexpr (Y == 2) sum.b += (double)now.x[e] + (double)now.x[e + 1];
                    }
                    n += 8;
                } else if (__any_sync(kAll, run != 0)) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const bool in = run >> e & 1;
                        if constexpr (X) sum.a += pick(in, (double)now.x[e] - (double)now.m[e], 0.0);
                        if constexpr (Y == 1) sum.b += pick(in, (double)now.y[e] - (double)now.l[e], 0.0);
                        if constexpr (Y == 2) sum.b += pick(in, (double)now.x[e], 0.0);
                    }
                    n += __popc(run);
                }
                if (c.end > hi) break;
                finish(true);
                if (c.end >= stop) return; // the share ends with it
                lo = c.end;
                c.on(a.q, lo, lane);
                if (lo >= hi) break;
            }
        }
        now = then;
    }
    finish(false);
}

// A CTA's numbers added up over its threads, in a fixed order: number i in every thread's copy of `sums`, which is in shared memory.
template <int FIRST> __device__ __forceinline__ void sum_threads(const double (&v)[kStats], double (&sums)[kStats])
{
    __shared__ double sh[kStats][kWarps];
#pragma unroll
    for (int i = FIRST; i < kStats; ++i) {
        const double t = warp_sum(v[i]);
        if ((threadIdx.x & 31) == 0) sh[i][threadIdx.x >> 5] = t;
    }
    __syncthreads();
    if ((int)threadIdx.x >= FIRST && threadIdx.x < kStats) {
        double t = 0.0;
        for (int w = 0; w < kWarps; ++w) t += sh[threadIdx.x][w];
        sums[threadIdx.x] = t;
    }
    __syncthreads();
}

// Into the CTA's slots.
__device__ __forceinline__ void put_stats(const double (&v)[kStats], double *slots)
{
    __shared__ double sums[kStats];
    sum_threads<0>(v, sums);
    if (threadIdx.x < kStats) slots[threadIdx.x] = sums[threadIdx.x];
}

// The sums over the CTAs' slots, of the numbers from FIRST on.
template <int FIRST> __device__ __forceinline__ void sum_slots(const double *partials, int ctas, double (&sums)[kStats])
{
    double v[kStats] = {};
    for (int c = threadIdx.x; c < ctas; c += kThreads)
#pragma unroll
        for (int i = FIRST; i < kStats; ++i) v[i] += __ldcg(partials + (size_t)c * kStats + i);
    sum_threads<FIRST>(v, sums);
}

// ------------------------------------------------------------------ policy loss

// exp(e) - e - 1 without the cancellation at small e: the Taylor series, sum over j of e^(j+2) / (j+2)!, of which the first term left
// out at |e| <= 2 is 2^14 2 / 16! = 1.6e-9 of the first.  Larger e need another form.  A number, or two at once.
constexpr float kLargest = 2.0f;
#define HILORE_TWICE(x) {1.0f / x, 1.0f / x}
static __constant__ float2 kInverseFactorials[14] = {
    HILORE_TWICE(2.0f), HILORE_TWICE(6.0f), HILORE_TWICE(24.0f), HILORE_TWICE(120.0f), HILORE_TWICE(720.0f),
    HILORE_TWICE(5040.0f), HILORE_TWICE(40320.0f), HILORE_TWICE(362880.0f), HILORE_TWICE(3628800.0f), HILORE_TWICE(39916800.0f),
    HILORE_TWICE(479001600.0f), HILORE_TWICE(6227020800.0f), HILORE_TWICE(87178291200.0f), HILORE_TWICE(1307674368000.0f)};
#undef HILORE_TWICE
__device__ __forceinline__ float exp_minus_line(float e)
{
    float s = kInverseFactorials[13].x;
#pragma unroll
    for (int j = 12; j >= 0; --j) s = fmaf(s, e, kInverseFactorials[j].x);
    return s * (e * e);
}
__device__ __forceinline__ void exp_minus_line(float e0, float e1, float &v0, float &v1)
{
    const uint64_t *factors = reinterpret_cast<const uint64_t *>(kInverseFactorials);
    const uint64_t e = f32x2_pack(e0, e1);
    uint64_t s = factors[13];
#pragma unroll
    for (int j = 12; j >= 0; --j) s = f32x2_fma(s, e, factors[j]);
    f32x2_unpack(f32x2_mul(s, f32x2_mul(e, e)), v0, v1);
}

constexpr float kNear = 80.0f;
// exp(d) = 2^(d log2 e) for |d| <= kNear, with log2 e in two parts: the power of the first part's product, as it is rounded, and to first
// order that of what the rounding and the second part leave.
__device__ __forceinline__ float exp_near(float d)
{
    constexpr float kLog2e = 1.44269502162933349609375f, kRest = 1.92596299112661747e-8f, kLn2 = 0.693147180559945309f;
    const float t = d * kLog2e, rest = fmaf(d, kRest, fmaf(d, kLog2e, -t));
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(t));
    return fmaf(y, rest * kLn2, y);
}

struct PolicyArgs {
    Sequences q;
    Share w;
    const float *logp, *old, *ref, *rollout, *adv, *moments, *grad_loss;
    const uint8_t *mask;
    const int64_t *N_dev;
    double N, clip_low, clip_high, log_low, log_high, log_dual, dual, cap, beta, adv_eps;
    float near; // distance of a logarithm of a ratio from its bounds within which it is compared in fp64
    int sequence_mean, k2, dual_clip, vec;
    Pieces pieces;
    double *partials;
    unsigned *done;
    float *stats, *omega;
    int cluster; // the call is one cluster
};

__device__ __forceinline__ double inverse_norm(const PolicyArgs &a)
{
    const double N = a.N_dev ? (double)*a.N_dev : a.N;
    return N > 0.0 ? 1.0 / N : 0.0;
}

enum { kNoKl = 0, kEasyKl = 1, kK3 = 2 }; // kEasyKl: K1 or K2

// The KL term and its derivative by s, at e = s_ref - s.
template <int KL> __device__ __forceinline__ void kl_term(float e, bool k2, float &value, float &slope)
{
    if (KL == kK3) {
        // both forms, and a choice: a branch would cost as much
        const float near = exp_minus_line(e), all = expf(e);
        const bool far = fabsf(e) > kLargest;
        value = far ? all - e - 1.0f : near;
        slope = far ? 1.0f - all : -(near + e);
    } else {
        value = k2 ? 0.5f * e * e : -e;
        slope = k2 ? -e : 1.0f;
    }
}

// stats: loss, policy term, KL term, share on flat branches, mean of old - new; by a whole CTA
__device__ __forceinline__ void policy_stats(const double *partials, int ctas, double beta, float *stats)
{
    __shared__ double sums[kStats];
    sum_slots<0>(partials, ctas, sums);
    if (threadIdx.x < kStats) stats[threadIdx.x] = (float)(threadIdx.x == 0 ? (beta != 0.0 ? fma(beta, sums[2], sums[1]) : sums[1]) : sums[threadIdx.x]);
}
__global__ void __launch_bounds__(kThreads) policy_final_kernel(const double *partials, int ctas, double beta, float *stats)
{
    grid_dependency_wait();
    grid_dependency_release();
    policy_stats(partials, ctas, beta, stats);
}

// A CTA's numbers, and by the last CTA to come, or the first one of a cluster, the statistics (otherwise the kernel behind makes them).
__device__ __forceinline__ void policy_hand_on(const PolicyArgs &a, const double (&v)[kStats])
{
    __shared__ bool last;
    put_stats(v, a.partials + (size_t)blockIdx.x * kStats);
    if (a.cluster) {
        cg::this_cluster().sync();
        if (blockIdx.x == 0) policy_stats(a.partials, gridDim.x, a.beta, a.stats);
    } else if (a.done) {
        __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) last = atomicAdd(a.done, 1u) == gridDim.x - 1;
        __syncthreads();
        if (last) {
            __threadfence();
            policy_stats(a.partials, gridDim.x, a.beta, a.stats);
        }
    }
}

// Ratios of tokens.  SEQ: there is something to a sequence, its weight or its advantage, which a lane looks up for one sequence of a window of 32.
// Which side of a bound a ratio is on is decided in fp32 but for the few next to it, which are compared in fp64, as the formula does.  What a sum has
// in common (1 / N, signs) is multiplied in at its end.  A lane's eight tokens of a block are added up in fp32, as these are: seven roundings beside
// theirs, and eight conversions less; then in fp64.  A kernel for each kind of terms, as a term that is not asked for costs registers and
// instructions all the same.
// Memory and issue slots bound it alike: 60 M tokens with advantages per token and K3 to a reference 214 us, 5.9 TB/s, 508 instructions of a warp for 256
// tokens.  Blocks with a ratio next to a bound, or with what is far out (K3: |s_ref - s| > 2), go token by token through both forms of each term: with one
// such token in 2560 211 us, in 256 250, in 10 279, for 206 without one.  It was 530 in tiles of 2048 tokens with one kernel for all terms, 237 with shares of warps and a kernel for each kind, and the rest is
// masks read a block ahead and products in place of branches.
// 13 M tokens in 40000 sequences of 327, weights per sequence, 75 us; 133 with each sequence looked up when it came.
template <bool SEQ, int KL, bool ROLLOUT, bool PER_TOKEN> __global__ void __launch_bounds__(kThreads, kPerSm) policy_token_kernel(const __grid_constant__ PolicyArgs a)
{
    const int lane = threadIdx.x & 31, share = blockIdx.x * kWarps + (threadIdx.x >> 5);
    // behind the sums' launch, which waited for all before it, nothing but the sums has to be waited for
    if (!a.done) grid_dependency_wait();
    grid_dependency_release();
    const int live = a.q.live(), tokens = a.w.per_warp * kBlock;
    const double inv = inverse_norm(a);
    double v[kStats] = {};
    if ((int64_t)share * tokens < live) {
        const int begin = share * tokens, stop = min(live - begin, tokens) + begin;
        const float g = a.grad_loss ? *a.grad_loss : 1.0f;
        const float mean = a.moments ? a.moments[0] : 0.0f, scale = a.moments ? (float)(1.0 / ((double)a.moments[1] + a.adv_eps)) : 1.0f;
        const bool strange = !(fabsf(mean) <= FLT_MAX) || !(fabsf(scale) <= FLT_MAX); // then masked tokens must not go as zeros
        const float high = (float)a.log_high, low = (float)a.log_low, dual_log = (float)a.log_dual;
        const float most_up = (float)(1.0 + a.clip_high), most_down = (float)(1.0 - a.clip_low), dual = (float)a.dual, cap = (float)a.cap;
        const float beta = a.beta != 0.0 ? (float)(a.beta * inv * g) : 0.0f, slope_of = (float)(-inv * g);
        Cursor c{0, 0x7FFFFFFF, 0, 0};
        float w = 1.0f, A_of = 0.0f; // of the sequence: weight / inv, advantage
        float w_of = 1.0f, A_lane = 0.0f; // of the window's sequences,
        bool far = false;                 // or not, as its sums lie over many shares
        auto weight = [&](double n) { return n > 0.0 ? (float)(1.0 / n) : 0.0f; };
        auto look = [&]() { // the window's: of sequences that begin in the share, and of the first one
            const int before = __shfl_up_sync(kAll, c.ends, 1);
            const int o = c.first + lane;
            far = false;
            if (o >= a.q.n_seq || (lane > 0 && before >= stop)) return;
            if (a.sequence_mean) {
                const double n = a.pieces.total(a.q, o, 4).n;
                far = n < 0.0;
                w_of = weight(n);
            }
            if (!PER_TOKEN) A_lane = (__ldg(a.adv + o) - mean) * scale;
        };
        auto enter = [&](bool other) {
            if (other) look();
            const int i = c.s - c.first;
            w = __shfl_sync(kAll, w_of, i);
            A_of = __shfl_sync(kAll, A_lane, i);
            if (__ballot_sync(kAll, far) >> i & 1) w = weight(a.pieces.total_warp(a.q, c.s, lane).n);
        };
        auto enter_lane = [&]() {
            if (a.sequence_mean) w = weight(a.pieces.total(a.q, c.s).n);
            if (!PER_TOKEN) A_of = (__ldg(a.adv + c.s) - mean) * scale;
        };
        Mask8 mask;
        mask.read(a.mask, begin + lane * 8, stop, a.vec);
#pragma unroll 1
        for (int base = begin; base < stop; base += kBlock) {
            const int k = base + lane * 8, hi = min(base + kBlock, stop);
            const uint32_t valid = inv > 0.0 ? mask.bits(k, hi) : 0u;
            float s[8] = {}, o[8] = {}, r[8] = {}, b[8] = {}, A[8] = {}, out[8];
            if (valid) {
                load8(a.logp, k, hi, a.vec, s);
                load8(a.old, k, hi, a.vec, o);
                if (KL) load8(a.ref, k, hi, a.vec, r);
                if (ROLLOUT) load8(a.rollout, k, hi, a.vec, b);
                if (PER_TOKEN) load8(a.adv, k, hi, a.vec, A);
            }
            mask.read(a.mask, k + kBlock, stop, a.vec);
            if (SEQ && base == begin) { // while the first block is on its way
                c.at(a.q, begin, lane);
                if (a.done) grid_dependency_wait();
                enter(true);
            }
            zero8(out);
            float wt[8]; // weights / inv; and advantages, if they are of sequences
            const bool whole = !SEQ || c.end >= hi;
            if (SEQ) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    wt[e] = w;
                    if (!PER_TOKEN) A[e] = A_of;
                }
            }
            if (!whole) {
                if (c.inside(hi, lane) > kFew) {
                    const int last = c.ahead(a.q, hi, lane), rim = min(k + 8, hi);
                    bool going = false;
                    if (k < hi) {
                        const bool moved = c.spread(a.q, k, last);
                        if (moved) enter_lane();
                        going = moved || c.end < rim;
                    }
                    int lo = k;
#pragma unroll 1
                    while (__any_sync(kAll, going)) {
                        if (going) {
                            const uint32_t run = range_bits(k, lo, c.end);
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                if (run >> e & 1) {
                                    wt[e] = w;
                                    if (!PER_TOKEN) A[e] = A_of;
                                }
                            going = c.end < rim;
                            if (going) lo = c.end, c.next(a.q, last), enter_lane();
                        }
                    }
                    const int from = (hi - 1 - base) >> 3;
                    w = __shfl_sync(kAll, w, from);
                    A_of = __shfl_sync(kAll, A_of, from);
                    c.join(a.q, from, lane);
                    look();
                } else {
#pragma unroll 1
                    while (c.end < hi) {
                        const int lo = c.end;
                        enter(c.on(a.q, lo, lane));
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (k + e >= lo) {
                                wt[e] = w;
                                if (!PER_TOKEN) A[e] = A_of;
                            }
                    }
                }
            }
            // Nearly always a block has no ratio within rounding of a bound and nothing far out: then masked tokens go as zeros, which add
            // nothing to any sum, and a ratio that a bound moves is on a flat branch.
            if (valid != 0xFFu) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (!(valid >> e & 1)) {
                        s[e] = o[e] = 0.0f;
                        if (KL) r[e] = 0.0f;
                        if (ROLLOUT) b[e] = 0.0f;
                        A[e] = PER_TOKEN ? mean : 0.0f;
                    }
            }
            bool odd = strange;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float d = s[e] - o[e];
                odd |= !(fabsf(d) <= kNear);
                odd |= fminf(fabsf(d - high), fabsf(d - low)) <= a.near;
                if (a.dual_clip) odd |= fabsf(d - dual_log) <= a.near;
                if (KL) odd |= !(fabsf(r[e] - s[e]) <= (KL == kK3 ? kLargest : kNear));
                if (ROLLOUT) odd |= !(fabsf(o[e] - b[e]) <= kNear);
            }
            float term = 0.0f, kls = 0.0f, drift = 0.0f, flats = 0.0f;
            if (!__any_sync(kAll, odd)) {
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    float value[2], slope[2];
                    if (KL == kK3) {
                        const float e0 = r[e] - s[e], e1 = r[e + 1] - s[e + 1];
                        exp_minus_line(e0, e1, value[0], value[1]);
                        slope[0] = -(value[0] + e0);
                        slope[1] = -(value[1] + e1);
                    } else if (KL) {
#pragma unroll
                        for (int i = 0; i < 2; ++i) kl_term<KL>(r[e + i] - s[e + i], a.k2, value[i], slope[i]);
                    }
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float d = s[e + i] - o[e + i], rho = exp_near(d);
                        float x = PER_TOKEN ? (A[e + i] - mean) * scale : A[e + i];
                        // the ratio's bounds; none where x is NaN, which stays, nor where it is 0
                        const float least = x < 0.0f ? most_down : 0.0f;
                        float most = x > 0.0f ? most_up : INFINITY;
                        if (a.dual_clip) most = x < 0.0f ? dual : most;
                        if (SEQ) x *= wt[e + i];
                        if (ROLLOUT) x *= fminf(exp_near(o[e + i] - b[e + i]), cap);
                        const float u = fminf(fmaxf(rho, least), most), held = x * u;
                        const bool flat = u != rho; // by the ratio: products of an infinite or a tiny x would be equal
                        float grad = flat ? 0.0f : slope_of * held;
                        flats += flat ? (SEQ ? wt[e + i] : 1.0f) : 0.0f;
                        term += held;
                        drift = SEQ ? fmaf(wt[e + i], d, drift) : drift + d;
                        if (KL) {
                            kls = SEQ ? fmaf(wt[e + i], value[i], kls) : kls + value[i];
                            grad = fmaf(SEQ ? beta * wt[e + i] : beta, slope[i], grad);
                        }
                        out[e + i] = grad;
                    }
                }
                if (valid != 0xFFu) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) out[e] = valid >> e & 1 ? out[e] : 0.0f;
                }
            } else {
                // which tokens are on a flat branch, and which of these on the dual clip's
                uint32_t flat = 0, over = 0;
                bool close = false;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float Ae = PER_TOKEN ? (A[e] - mean) * scale : A[e], d = s[e] - o[e];
                    // A >= 0: beyond the bound where d > high; A < 0: where -d > -low; NaN: never
                    const bool up = Ae >= 0.0f;
                    const float past = __uint_as_float(__float_as_uint(d) ^ (up ? 0u : 0x80000000u)) - (up ? high : -low);
                    flat |= past > 0.0f && Ae == Ae ? 1u << e : 0u;
                    close |= fabsf(past) <= a.near;
                    if (a.dual_clip) {
                        over |= Ae < 0.0f && d > dual_log ? 1u << e : 0u;
                        close |= fabsf(d - dual_log) <= a.near;
                    }
                }
                if (close) { // next to a bound: compared as the formula does
                    flat = over = 0;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float Ae = PER_TOKEN ? (A[e] - mean) * scale : A[e];
                        const double D = (double)s[e] - (double)o[e];
                        if (Ae >= 0.0f ? D > a.log_high : Ae < 0.0f && D < a.log_low) flat |= 1u << e;
                        if (Ae < 0.0f && D > a.log_dual) over |= 1u << e;
                    }
                }
                flat |= over;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const bool in = valid >> e & 1, on_flat = flat >> e & 1;
                    const float Ae = PER_TOKEN ? (A[e] - mean) * scale : A[e], d = s[e] - o[e];
                    const float rho = fabsf(d) <= kNear ? exp_near(d) : expf(d); // the same bits as above where that is enough
                    float bound = Ae >= 0.0f ? most_up : most_down;
                    if (a.dual_clip) bound = over >> e & 1 ? dual : bound;
                    const float we = SEQ ? wt[e] : 1.0f;
                    float x = SEQ ? Ae * we : Ae;
                    bool none = Ae == 0.0f && fabsf(d) <= FLT_MAX; // nothing, though ratio or weight may be beyond fp32
                    if (ROLLOUT) {
                        const float gap = o[e] - b[e], i = fabsf(gap) <= kNear ? exp_near(gap) : expf(gap);
                        x *= i > cap ? cap : i; // NaN stays
                        none = none && fabsf(gap) <= FLT_MAX;
                    }
                    const float gain = none ? 0.0f : x * (on_flat ? bound : rho);
                    float grad = on_flat ? 0.0f : slope_of * gain;
                    term += in ? gain : 0.0f;
                    drift = in ? fmaf(we, d, drift) : drift;
                    flats += in && on_flat && Ae != 0.0f ? we : 0.0f;
                    if (KL) {
                        float value, slope;
                        kl_term<KL>(r[e] - s[e], a.k2, value, slope);
                        kls = in ? fmaf(we, value, kls) : kls;
                        if (beta != 0.0f) grad = fmaf(SEQ ? beta * we : beta, slope, grad);
                    }
                    if (in) out[e] = grad;
                }
            }
            v[1] -= (double)term;
            if (KL) v[2] += (double)kls;
            v[3] += (double)flats;
            v[4] -= (double)drift;
            if (SEQ && c.end <= hi && c.end < stop) enter(c.on(a.q, hi, lane));
            if (a.vec && hi - base == kBlock) store8(a.omega + k, out);
            else store8(a.omega, k, base, hi, a.vec, out);
        }
    }
#pragma unroll
    for (int i = 1; i < kStats; ++i) v[i] *= inv;
    if (a.done) grid_dependency_wait(); // all threads, before anything is written
    policy_hand_on(a, v);
}

// Ratios of whole sequences: of a sequence the policy term's gradient is the same for every token.  The window's lanes work out ratio, bound and slope
// in fp64, each for its sequence; the share that holds a sequence's first token adds what the statistics have of it, once.  1 M tokens in 512 sequences
// 16 us for both launches, which is latency; 57 M without a KL term 154 us (5 TB/s), 37 M with K3 170.
template <int KL> __global__ void __launch_bounds__(kThreads, kPerSm) policy_sequence_kernel(const __grid_constant__ PolicyArgs a)
{
    const int lane = threadIdx.x & 31, share = blockIdx.x * kWarps + (threadIdx.x >> 5);
    if (!a.done) grid_dependency_wait(); // as above
    grid_dependency_release();
    const int live = a.q.live(), tokens = a.w.per_warp * kBlock;
    const double inv = inverse_norm(a), g = a.grad_loss ? (double)*a.grad_loss : 1.0;
    double v[kStats] = {};
    if ((int64_t)share * tokens < live) {
        const int begin = share * tokens, stop = min(live - begin, tokens) + begin;
        Cursor c{0, 0x7FFFFFFF, 0, 0};
        const float beta = (float)(a.beta * g);
        float w = 0.0f, slope_of = 0.0f;
        // Into w and slope_of; counts: into the statistics as well.
        auto entered = [&](int o, const Piece &p, bool counts) {
            w = slope_of = 0.0f;
            if (!(p.n > 0.0) || !(inv > 0.0)) return;
            const double per = 1.0 / p.n, weight = a.sequence_mean ? inv * per : inv, d = p.a * per;
            double A = (double)__ldg(a.adv + o);
            if (a.moments) A = (A - (double)a.moments[0]) / ((double)a.moments[1] + a.adv_eps);
            const bool none = A == 0.0 && fabs(d) <= DBL_MAX && (!a.rollout || fabs(p.b) <= DBL_MAX); // nothing, though u or i may be beyond fp64
            const double gap = a.rollout && !none ? exp(p.b * per) : 1.0, i = a.rollout && gap > a.cap ? a.cap : gap; // NaN stays
            const bool flat = A >= 0.0 ? d > a.log_high : A < 0.0 && (d < a.log_low || d > a.log_dual);
            double u = none ? 1.0 : exp(d);
            w = (float)weight;
            if (flat) u = A >= 0.0 ? 1.0 + a.clip_high : (d < a.log_low ? 1.0 - a.clip_low : a.dual);
            else slope_of = (float)(-weight * i * A * u * g);
            if (counts) {
                v[1] -= p.n * weight * i * A * u;
                if (flat && A != 0.0) v[3] += p.n * weight;
                v[4] -= weight * p.a;
            }
        };
        float w_of = 0.0f, slope_lane = 0.0f; // of the window's sequences,
        bool far = false;                     // or not, as its sums lie over many shares
        int counted = begin;                  // the tokens before it are those of sequences that the statistics have
        auto look = [&]() { // the window's: of sequences that begin in the share, and of the first one
            int before = __shfl_up_sync(kAll, c.ends, 1);
            const int o = c.first + lane;
            far = false;
            if (o < a.q.n_seq && (lane == 0 || before < stop)) {
                const Piece p = a.pieces.total(a.q, o, 4);
                far = p.n < 0.0;
                if (lane == 0) before = a.q.bound(o);
                entered(o, p, before >= counted);
                w_of = w, slope_lane = slope_of;
            }
            counted = __shfl_sync(kAll, c.ends, 31);
        };
        auto enter = [&](bool other) {
            if (other) look();
            const int i = c.s - c.first;
            w = __shfl_sync(kAll, w_of, i);
            slope_of = __shfl_sync(kAll, slope_lane, i);
            if (__ballot_sync(kAll, far) >> i & 1) entered(c.s, a.pieces.total_warp(a.q, c.s, lane), lane == 0 && a.q.bound(c.s) >= begin);
        };
        auto enter_lane = [&](int k) { // by the lane of token k: what no window has, and begins there, counts
            Piece p = a.pieces.total(a.q, c.s, 4);
            const int b = a.q.bound(c.s);
            const bool no = p.n < 0.0;
            if (no) p = a.pieces.total(a.q, c.s);
            entered(c.s, p, b >= k && (no || b >= counted));
        };
        Mask8 mask;
        mask.read(a.mask, begin + lane * 8, stop, a.vec);
#pragma unroll 1
        for (int base = begin; base < stop; base += kBlock) {
            const int k = base + lane * 8, hi = min(base + kBlock, stop);
            const uint32_t valid = inv > 0.0 ? mask.bits(k, hi) : 0u;
            mask.read(a.mask, k + kBlock, stop, a.vec);
            float s[8] = {}, r[8] = {}, out[8];
            if (KL && valid) {
                load8(a.logp, k, hi, a.vec, s);
                load8(a.ref, k, hi, a.vec, r);
            }
            if (base == begin) {
                c.at(a.q, begin, lane);
                if (a.done) grid_dependency_wait();
                enter(true);
            }
            float wt[8], slopes[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) wt[e] = w, slopes[e] = slope_of;
            if (c.end < hi) {
                if (c.inside(hi, lane) > kFew) {
                    const int last = c.ahead(a.q, hi, lane), rim = min(k + 8, hi);
                    bool going = false;
                    if (k < hi) {
                        const bool moved = c.spread(a.q, k, last);
                        if (moved) enter_lane(k);
                        going = moved || c.end < rim;
                    }
                    int lo = k;
#pragma unroll 1
                    while (__any_sync(kAll, going)) {
                        if (going) {
                            const uint32_t run = range_bits(k, lo, c.end);
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                if (run >> e & 1) wt[e] = w, slopes[e] = slope_of;
                            going = c.end < rim;
                            if (going) lo = c.end, c.next(a.q, last), enter_lane(k);
                        }
                    }
                    const int from = (hi - 1 - base) >> 3;
                    const float w_last = __shfl_sync(kAll, w, from), slope_last = __shfl_sync(kAll, slope_of, from);
                    c.join(a.q, from, lane);
                    counted = max(counted, c.end);
                    look();
                    w = w_last, slope_of = slope_last;
                } else {
#pragma unroll 1
                    while (c.end < hi) {
                        const int lo = c.end;
                        enter(c.on(a.q, lo, lane));
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (k + e >= lo) wt[e] = w, slopes[e] = slope_of;
                    }
                }
            }
            float kls = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const bool in = valid >> e & 1;
                float grad = slopes[e];
                if (KL) {
                    float value, slope;
                    kl_term<KL>(r[e] - s[e], a.k2, value, slope);
                    kls = in ? fmaf(wt[e], value, kls) : kls;
                    if (beta != 0.0f) grad = fmaf(beta * wt[e], slope, grad);
                }
                out[e] = in ? grad : 0.0f;
            }
            if (KL) v[2] += (double)kls;
            if (c.end <= hi && c.end < stop) enter(c.on(a.q, hi, lane));
            if (a.vec && hi - base == kBlock) store8(a.omega + k, out);
            else store8(a.omega, k, base, hi, a.vec, out);
        }
    }
    if (a.done) grid_dependency_wait();
    policy_hand_on(a, v);
}

// ------------------------------------------------------------------ preference loss

struct PreferenceArgs {
    Sequences q;
    Share w;
    const float *rewards, *grad_loss;
    const uint8_t *mask;
    const int64_t *N_dev;
    double N, beta, margin, margin_reward, smoothing, nll;
    int G, loss, length_mean, vec, groups, per_cta, slices, team, ctas;
    Pieces pieces;
    double *coef; // [n_seq] gradient of every valid token, before the division by N
    double *partials;
    float *scores, *stats;
    int64_t *pairs;
    float *omega;
    int behind;  // other launches of the call came first
};

// A CTA takes `per_cta` whole groups at a time, or one of the `slices` of the responses of a larger one: scores of all sequences of these
// groups into shared memory, then each sequence against the others of its group, both ways, so that the gradient needs no atomics.  Bound by 64-bit
// exponentials and logarithms: 32768 responses in groups of 16 take 12 us, 512 responses to one prompt 25 (one CTA for them 600).
__global__ void __launch_bounds__(kThreads) preference_pairs_kernel(const __grid_constant__ PreferenceArgs a)
{
    grid_dependency_wait();
    grid_dependency_release();
    extern __shared__ double smem[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, room = a.per_cta * a.G;
    double *h = smem, *like = smem + room;             // score, mean log-probability
    double *per = smem + 2 * room;                     // 1 / |T| (0: no valid token)
    float *R = reinterpret_cast<float *>(smem + 3 * room);
    double v[kStats] = {}; // loss, right order, gap, nll, pairs
    const int64_t items = a.slices > 1 ? (int64_t)a.groups * a.slices : (a.groups + a.per_cta - 1) / a.per_cta;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t first = a.slices > 1 ? item / a.slices : item * a.per_cta;
        const int slice = a.slices > 1 ? (int)(item - first * a.slices) : 0;
        const int n = (int)(a.groups - first < a.per_cta ? a.groups - first : a.per_cta) * a.G;
        const int each = a.slices > 1 ? (n + a.slices - 1) / a.slices : n, from = slice * each, to = min(n, from + each);
        const int64_t base = first * a.G;
        auto put = [&](int i, const Piece &p) {
            const double inv = p.n > 0.0 ? 1.0 / p.n : 0.0;
            h[i] = p.n > 0.0 ? a.beta * (a.length_mean ? p.a * inv : p.a) : 0.0;
            like[i] = p.n > 0.0 ? p.b * inv : 0.0;
            per[i] = inv;
            R[i] = a.rewards[base + i];
            if (a.scores && i >= from && i < to) a.scores[base + i] = (float)h[i];
        };
        bool far = false;
        for (int i = threadIdx.x; i < n; i += kThreads) {
            const Piece p = a.pieces.total(a.q, (int)(base + i), 32);
            far |= p.n < 0.0;
            put(i, p);
        }
        if (__syncthreads_or(far)) {
            for (int i = warp; i < n; i += kWarps) {
                const Piece p = a.pieces.total_warp(a.q, (int)(base + i), lane);
                if (lane == 0) put(i, p);
            }
            __syncthreads();
        }
        // a.team neighbouring threads share the others of a response's group
        const int part = threadIdx.x & (a.team - 1);
        for (int i = from + threadIdx.x / a.team; i < to; i += kThreads / a.team) {
            const int begin = i / a.G * a.G;
            const double hi = h[i];
            const float Ri = R[i];
            double c = 0.0;
            int wins = 0;
            if (per[i] > 0.0)
                for (int j = begin + part; j < begin + a.G; j += a.team) {
                    const float Rj = R[j];
                    if (!(per[j] > 0.0) || !(Ri > Rj || Rj > Ri)) continue;
                    const bool won = Ri > Rj;
                    const double gap = won ? hi - h[j] : h[j] - hi;
                    const double more = a.margin_reward != 0.0 ? a.margin_reward * (won ? (double)Ri - (double)Rj : (double)Rj - (double)Ri) : 0.0;
                    const double z = gap - a.margin - more;
                    double value = 0.0, slope;
                    if (a.loss == HILORE_PREF_SIGMOID) {
                        const double t = exp(-fabs(z)); // -ln sigmoid(z) and its derivative
                        slope = a.smoothing - (z >= 0.0 ? t : 1.0) / (1.0 + t);
                        if (won) { // each logarithm with its weight: one of them may be infinite, or all but nothing beside the other
                            const double both = log1p(t);
                            if (a.smoothing < 1.0) value = (1.0 - a.smoothing) * (both + fmax(-z, 0.0));
                            if (a.smoothing > 0.0) value += a.smoothing * (both + fmax(z, 0.0));
                        }
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
            // teams are whole parts of a warp, and their threads take the same turns
            const uint32_t team = a.team == 32 ? kAll : ((1u << a.team) - 1) << (threadIdx.x & 31 & ~(a.team - 1));
            for (int by = a.team / 2; by > 0; by /= 2) {
                c += __shfl_xor_sync(team, c, by);
                wins += __shfl_xor_sync(team, wins, by);
            }
            if (part == 0) {
                if (wins) v[3] -= wins * like[i]; // not 0 * infinity of a response that wins nothing
                v[4] += wins;
                c *= a.length_mean ? a.beta * per[i] : a.beta;
                a.coef[base + i] = wins ? c - a.nll * wins * per[i] : c;
            }
        }
        __syncthreads();
    }
    put_stats(v, a.partials + (size_t)blockIdx.x * kStats);
}

// The gradient of a sequence to each of its valid tokens.  Every CTA adds up the pairs of the CTAs before for the division by N; the first
// one writes the statistics: loss, share of pairs in the right order, mean gap of the scores, mean -log-probability per token of the winners.
// Reads a mask and writes a number a token: 50 M tokens 50 us (5 TB/s).
__global__ void __launch_bounds__(kThreads, 4) preference_token_kernel(const __grid_constant__ PreferenceArgs a)
{
    __shared__ double sums[kStats];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, share = blockIdx.x * kWarps + warp;
    // behind the other launches, which waited for all before them, nothing but their results has to be waited for
    if (!a.behind) grid_dependency_wait();
    grid_dependency_release();
    const int live = a.q.live(), tokens = a.w.per_warp * kBlock;
    const bool some = (int64_t)share * tokens < live;
    const int begin = some ? share * tokens : 0, stop = some ? min(live - begin, tokens) + begin : 0;
    Cursor c{0, 0, 0, 0};
    constexpr int kAhead = 4; // blocks whose masks are on their way: there is little else to do
    Mask8 mask[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) mask[i].read(a.mask, begin + i * kBlock + lane * 8, stop, a.vec);
    if (some) c.at(a.q, begin, lane);
    if (a.behind) grid_dependency_wait();
    const bool count = !a.N_dev && !(a.N > 0.0);
    if (blockIdx.x == 0) sum_slots<0>(a.partials, a.ctas, sums);
    else if (count) sum_slots<kStats - 1>(a.partials, a.ctas, sums);
    const double N = a.N_dev ? (double)*a.N_dev : (count ? sums[kStats - 1] : a.N);
    const double inv = N > 0.0 ? 1.0 / N : 0.0;
    if (blockIdx.x == 0 && threadIdx.x < 4) {
        const int i = threadIdx.x;
        const bool none = !(inv > 0.0) || sums[4] == 0.0;
        if (i == 0 && a.pairs) *a.pairs = (int64_t)sums[4];
        a.stats[i] = none ? 0.0f : (float)((i == 0 ? sums[0] + (a.nll != 0.0 ? a.nll * sums[3] : 0.0) : sums[i]) * inv);
    }
    const double scale = inv * (a.grad_loss ? (double)*a.grad_loss : 1.0);
    if (!some)
        return;
    float coef, coef_of = 0.0f; // of the sequence, of the window's
    auto of = [&](int o) { return inv > 0.0 ? (float)(__ldcg(a.coef + o) * scale) : 0.0f; };
    auto enter = [&](bool other) {
        if (other && c.first + lane < a.q.n_seq) coef_of = of(c.first + lane);
        coef = __shfl_sync(kAll, coef_of, c.s - c.first);
    };
    enter(true);
#pragma unroll 1
    for (int first = begin; first < stop; first += kAhead * kBlock) {
        uint32_t valids = 0;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int k = first + i * kBlock + lane * 8;
            valids |= mask[i].bits(k, stop) << (8 * i);
            mask[i].read(a.mask, k + kAhead * kBlock, stop, a.vec);
        }
#pragma unroll 1
        for (int base = first; base < min(first + kAhead * kBlock, stop); base += kBlock, valids >>= 8) {
            const int k = base + lane * 8, hi = min(base + kBlock, stop);
            const uint32_t valid = valids & 0xFFu;
            float out[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) out[e] = valid >> e & 1 ? coef : 0.0f;
            if (c.end < hi) {
                if (c.inside(hi, lane) > kFew) {
                    const int last = c.ahead(a.q, hi, lane), rim = min(k + 8, hi);
                    bool going = false;
                    if (k < hi) {
                        const bool moved = c.spread(a.q, k, last);
                        if (moved) coef = of(c.s);
                        going = moved || c.end < rim;
                    }
                    int lo = k;
#pragma unroll 1
                    while (__any_sync(kAll, going)) {
                        if (going) {
                            const uint32_t run = valid & range_bits(k, lo, c.end);
#pragma unroll
                            for (int e = 0; e < 8; ++e) out[e] = run >> e & 1 ? coef : out[e];
                            going = c.end < rim;
                            if (going) lo = c.end, c.next(a.q, last), coef = of(c.s);
                        }
                    }
                    c.join(a.q, (hi - 1 - base) >> 3, lane);
                    enter(true);
                } else {
#pragma unroll 1
                    while (c.end < hi) {
                        const int lo = c.end;
                        enter(c.on(a.q, lo, lane));
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (k + e >= lo) out[e] = valid >> e & 1 ? coef : 0.0f;
                    }
                }
            }
            if (c.end <= hi && c.end < stop) enter(c.on(a.q, hi, lane));
            if (a.vec && hi - base == kBlock) store8(a.omega + k, out);
            else store8(a.omega, k, base, hi, a.vec, out);
        }
    }
}

constexpr int kMaxGroup = 1024;

// All warps of a call run at once, `per_sm` CTAs on an SM.
static Share share_of(int64_t n_tok, int per_sm)
{
    const int64_t blocks = (n_tok + kBlock - 1) / kBlock, warps = (int64_t)sm_count() * per_sm * kWarps;
    return Share{(int)blocks, (int)((blocks + warps - 1) / warps < 1 ? 1 : (blocks + warps - 1) / warps)};
}
static unsigned ctas_of(const Share &w)
{
    const int64_t warps = ((int64_t)w.blocks + w.per_warp - 1) / w.per_warp;
    return (unsigned)((warps + kWarps - 1) / kWarps);
}

// A call of up to kClusterBlocks blocks without sums of sequences is one launch: its CTAs are a thread-block cluster, whose barrier lies
// before the statistics (8192 tokens one call after the other: 5 us, 8 us as two launches).  With sums it gains nothing.
constexpr int kCluster = 8;                          // CTAs that any device grants
constexpr int64_t kClusterBlocks = kCluster * kWarps; // a block of a warp
static bool clusters_on()
{
    const char *off = std::getenv("HILORE_DISABLE_CLUSTER_LAUNCH");
    return off == nullptr || off[0] == '\0' || (off[0] == '0' && off[1] == '\0');
}
static bool one_cluster(int64_t n_tok) { return n_tok > 0 && (n_tok + kBlock - 1) / kBlock <= kClusterBlocks && clusters_on(); }
static unsigned cluster_of(const Share &w) // CTAs beyond the last share have nothing to do
{
    unsigned n = 1;
    while (n < ctas_of(w)) n *= 2;
    return n;
}
template <typename A> static cudaError_t launch_cluster(void (*kernel)(A), unsigned ctas, size_t smem, cudaStream_t st, const A &a)
{
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, a);
}

// Layout of a workspace: the CTAs' slots, the pieces of shares and sequences, a number per sequence.
constexpr int64_t kMostShares = 148 * 8 * kWarps; // on any device that this runs on, with up to eight CTAs of it on an SM
struct Workspace {
    size_t partials, done, head, tail, whole, coef, bytes;
};
static Workspace layout(int64_t n_seq, int64_t n_tok)
{
    Workspace w;
    const int64_t blocks = n_tok > 0 ? (n_tok + kBlock - 1) / kBlock : 0;
    const size_t shares = (size_t)(blocks < kMostShares ? blocks : kMostShares), S = n_seq > 0 ? (size_t)n_seq : 0;
    w.partials = 0;
    w.done = w.partials + sizeof(double) * kStats * kMostCtas;
    w.head = w.done + 16;
    w.tail = w.head + sizeof(Piece) * shares;
    w.whole = w.tail + sizeof(Piece) * shares;
    w.coef = w.whole + sizeof(Piece) * S;
    w.bytes = w.coef + sizeof(double) * S + 16;
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
    const bool sequence_ratio = t.ratio == HILORE_RATIO_SEQUENCE, per_token = t.adv_per_token != 0;
    a.sequence_mean = t.mean == HILORE_MEAN_SEQUENCES, a.k2 = t.kl == HILORE_KL_K2, a.dual_clip = t.dual_clip != 0.0;
    double widest = 0.0;
    for (double b : {a.log_low, a.log_high, a.log_dual})
        if (std::isfinite(b) && std::fabs(b) > widest) widest = std::fabs(b);
    a.near = (float)(widest * 0x1p-21 + 0x1p-20); // sixteen roundings of a ratio, and the two of a difference as large as the bound
    a.vec = vectors({logp, logp_old, logp_ref, logp_rollout, per_token ? adv : nullptr, omega}, mask);
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    a.pieces = pieces_of(workspace, w);
    a.partials = reinterpret_cast<double *>(ws + w.partials);
    a.omega = omega;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    a.stats = stats;
    if (n_tok == 0)
        return launch_dependent(policy_final_kernel, dim3(1), dim3(kThreads), 0, st, (const double *)a.partials, 0, a.beta, stats) == cudaSuccess &&
                       cudaGetLastError() == cudaSuccess
                   ? HILORE_OK
                   : HILORE_CUDA;
    const int kl = !logp_ref ? kNoKl : (t.kl == HILORE_KL_K3 ? kK3 : kEasyKl);
    void (*kernel)(PolicyArgs) = nullptr;
    if (sequence_ratio) {
        kernel = kl == kNoKl ? policy_sequence_kernel<kNoKl> : (kl == kK3 ? policy_sequence_kernel<kK3> : policy_sequence_kernel<kEasyKl>);
    } else {
#define HILORE_KLS(SEQ, ROLL, PER) {policy_token_kernel<SEQ, kNoKl, ROLL, PER>, policy_token_kernel<SEQ, kEasyKl, ROLL, PER>, policy_token_kernel<SEQ, kK3, ROLL, PER>}
        static void (*const kernels[3][2][3])(PolicyArgs) = {{HILORE_KLS(false, false, true), HILORE_KLS(false, true, true)},
                                                             {HILORE_KLS(true, false, true), HILORE_KLS(true, true, true)},
                                                             {HILORE_KLS(true, false, false), HILORE_KLS(true, true, false)}};
#undef HILORE_KLS
        kernel = kernels[!per_token ? 2 : (a.sequence_mean ? 1 : 0)][logp_rollout != nullptr][kl];
    }
    SumArgs s{};
    s.q = a.q, s.mask = mask, s.vec = a.vec, s.out = a.pieces;
    if (sequence_ratio) s.x = logp, s.minus = logp_old;
    if (sequence_ratio && logp_rollout) s.y = logp_old, s.less = logp_rollout;
    const bool sums = sequence_ratio || a.sequence_mean;
    if (!sums && one_cluster(n_tok)) {
        a.w = share_of(n_tok, 1);
        a.cluster = 1;
        if (launch_cluster(kernel, cluster_of(a.w), 0, st, a) == cudaSuccess)
            return HILORE_OK;
        (void)cudaGetLastError(); // refused: the launches below
        a.cluster = 0;
    }
    s.w = share_of(n_tok, s.y ? kSumsPerSmOfFour : kSumsPerSm);
    s.out.share = a.pieces.share = s.w.per_warp * kBlock;
    if (sums) {
        a.done = s.done = reinterpret_cast<unsigned *>(ws + w.done);
        void (*const sum)(SumArgs) = !sequence_ratio ? sequence_sums_kernel<false, 0> : (logp_rollout ? sequence_sums_kernel<true, 1> : sequence_sums_kernel<true, 0>);
        if (launch_dependent(sum, dim3(ctas_of(s.w)), dim3(kThreads), 0, st, s) != cudaSuccess)
            return HILORE_CUDA;
    }
    a.w = share_of(n_tok, kPerSm);
    const unsigned ctas = ctas_of(a.w);
    if (launch_dependent(kernel, dim3(ctas), dim3(kThreads), 0, st, a) != cudaSuccess)
        return HILORE_CUDA;
    if (!a.done && launch_dependent(policy_final_kernel, dim3(1), dim3(kThreads), 0, st, (const double *)a.partials, (int)ctas, a.beta, stats) != cudaSuccess)
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
    // Sixteen pairs in a row, of 64-bit exponentials and logarithms, take 15 us: threads share them as long as all of them run at once.
    a.team = 1;
    while (a.team < 32 && 2 * a.team <= G && 2 * a.team * n_seq <= (int64_t)sm_count() * 4 * kThreads) a.team *= 2;
    // Few responses go over all SMs, as 64-bit arithmetic is what takes long: 64 pairs on one SM 14 us, on 32 of them 12.
    a.per_cta = (int)std::max<int64_t>(1, std::min<int64_t>(kThreads / (G * a.team), (a.groups + sm_count() - 1) / sm_count()));
    a.slices = (G * a.team + kThreads - 1) / kThreads;
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    a.pieces = pieces_of(workspace, w);
    a.coef = reinterpret_cast<double *>(ws + w.coef);
    a.partials = reinterpret_cast<double *>(ws + w.partials);
    a.scores = scores, a.stats = stats, a.pairs = pairs, a.omega = omega;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const size_t smem = (size_t)a.per_cta * G * (3 * sizeof(double) + sizeof(float));
    SumArgs s{};
    s.q = a.q, s.mask = mask, s.vec = a.vec, s.x = logp, s.minus = logp_ref, s.out = a.pieces;
    s.w = share_of(n_tok, kSumsPerSm);
    s.out.share = a.pieces.share = s.w.per_warp * kBlock;
    if (n_tok > 0 && launch_dependent(sequence_sums_kernel<true, 2>, dim3(ctas_of(s.w)), dim3(kThreads), 0, st, s) != cudaSuccess)
        return HILORE_CUDA;
    if (a.groups > 0) {
        a.ctas = grid_of(a.slices > 1 ? (int64_t)a.groups * a.slices : (a.groups + a.per_cta - 1) / a.per_cta, kMostCtas);
        if (launch_dependent(preference_pairs_kernel, dim3((unsigned)a.ctas), dim3(kThreads), smem, st, a) != cudaSuccess)
            return HILORE_CUDA;
    }
    a.behind = n_tok > 0 && a.groups > 0;
    a.w = share_of(n_tok, 4);
    if (launch_dependent(preference_token_kernel, dim3(n_tok > 0 ? ctas_of(a.w) : 1u), dim3(kThreads), 0, st, a) != cudaSuccess)
        return HILORE_CUDA;
    return cudaGetLastError() == cudaSuccess ? HILORE_OK : HILORE_CUDA;
}
