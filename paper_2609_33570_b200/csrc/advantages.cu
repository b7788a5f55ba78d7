// Advantages and returns by a gated linear recurrence over the valid tokens of a sequence, and the backward pass of it.
#include <algorithm>
#include <climits>
#include <cmath>
#include <type_traits>

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
    static __device__ __forceinline__ double last_weight(const Map &, double w) { return w; }
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
        double G;
        int32_t pos, pad;
    };
    static __device__ __forceinline__ Map identity() { return Map{1.0, 0.0, 0.0, -1, 0u}; }
    static __device__ __forceinline__ State start() { return State{0.0, -1, 0}; }
    static __device__ __forceinline__ Map then(const Map &a, const Map &b)
    {
        if (b.flag == 2 || a.flag == 0) return b;
        if (b.flag == 0) return a;
        const double k = b.P * a.wl;
        return Map{k * a.P, fma(k, a.B, b.B), b.wl, b.pos, a.flag};
    }
    // Maps are joined from the beginning of a sequence on, where nothing comes in.
    static __device__ __forceinline__ State apply(const Map &m, const State &s) { return m.flag ? State{m.B, m.pos, 0} : s; }
    static __device__ __forceinline__ double last_weight(const Map &m, double w) { return m.flag ? m.wl : w; }
};

constexpr int kAdvThreads = 128; // four warps that know nothing of one another but at the end
constexpr int kAdvWarps = kAdvThreads / 32;
constexpr int kStages = 3;       // blocks of 256 tokens whose tensors a warp has in flight or at work
constexpr int kMaskStages = 8;   // and their masks, which say what to read of the tensors: more than 2 kStages, a power of two
constexpr uint32_t kAll = 0xFFFFFFFFu;

// How the work is dealt out.  A warp has one chunk of `chunk` tokens.  A sequence that goes on in the next chunk needs what comes out of
// that, or goes into it: maps of parts of chunks, made by a launch of their own before.  Two ways:
//   Even: a warp owns the tokens of its chunk.  A chunk's map covers its first sequence (backward pass: its last one) where that one
//   goes on in the chunk before (behind).  Every warp has as much to do as the others.
//   By pieces: a warp owns the pieces that begin in its chunk.  A piece is a whole sequence, or 2^piece tokens (the last one fewer) of
//   a longer one, so that nothing but long sequences needs more than one pass.  piece >= chunk, so no chunk holds the beginnings of
//   two pieces that are not the first of their sequence (or not the last), and a map's place is its chunk.
struct AdvantageArgs {
    Sequences q;
    const float *rewards, *outcome, *bootstrap, *trace;
    const void *values;
    int values_bf16;
    const uint8_t *mask;
    double gamma, weight; // gamma lambda
    double small[9];      // weight^0 .. weight^8
    double powers[5];     // weight^8, ^16, .. ^128
    float *adv, *returns;
    const float *grad_adv, *grad_returns, *adv_in;
    float *grad_rewards, *grad_outcome, *grad_values, *grad_bootstrap, *grad_trace;
    void *maps;       // [chunks]
    double *partials; // [CTAs][3] count, mean, sum of squared deviations
    int chunks, chunk, piece, vec;
    int even;
    int second; // second: a launch of this call came first, and what it did not write is there without waiting for it
};

// Where a chunk's part begins that would begin at token t of sequence s; the end of the last sequence if there is none.
__device__ __forceinline__ int part_from(const AdvantageArgs &a, int t, int s, int live)
{
    if (t >= live) return live;
    if (a.even) return t;
    const int b = a.q.bound(s), e = a.q.bound(s + 1);
    const uint32_t off = t > b ? (uint32_t)(t - b) : 0u, up = ((off + (1u << a.piece) - 1) >> a.piece) << a.piece;
    const int64_t p = (int64_t)b + up, at = p < e ? p : e;
    return (int)(at < t ? t : (at > live ? live : at)); // boundaries out of order stay inside
}

// The state behind the maps of `n` pieces, first to last; maps(i) gives the map of piece i.  A lane takes neighbouring ones: one scan of
// the warp, where a scan for each 32 of them took 14 us for a sequence of 640.
template <typename Op, typename F> __device__ __forceinline__ typename Op::State behind_pieces(typename Op::State s, int n, int lane, F maps, double &wl)
{
    if (n <= 0) return s;
    const int each = (n + 31) / 32, end = min(n, (lane + 1) * each);
    typename Op::Map m = Op::identity(), all;
#pragma unroll 2
    for (int i = lane * each; i < end; ++i) m = Op::then(m, maps(i));
    warp_scan<Op>(m, lane, all);
    all = shfl_words(all, 31);
    wl = Op::last_weight(all, wl);
    return Op::apply(all, s);
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
#pragma unroll 1
    for (int by = 1; by < 32; by *= 2) {
        Moments o;
        o.n = __shfl_down_sync(kAll, m.n, by);
        o.mean = __shfl_down_sync(kAll, m.mean, by);
        o.m2 = __shfl_down_sync(kAll, m.m2, by);
        m.join(o); // lane 0 has all of them in the end; what others have is not used
    }
    return m;
}

// x' = P x + B over the lanes: this lane's from those before it (all the lanes' in the last one).
struct Line {
    double P, B;
};
__device__ __forceinline__ Line scan_lines(Line &m, int lane)
{
#pragma unroll
    for (int by = 1; by < 32; by *= 2) {
        const double P = __shfl_up_sync(kAll, m.P, by), B = __shfl_up_sync(kAll, m.B, by);
        if (lane >= by) {
            m.B = fma(m.P, B, m.B);
            m.P *= P;
        }
    }
    Line before;
    before.P = __shfl_up_sync(kAll, m.P, 1);
    before.B = __shfl_up_sync(kAll, m.B, 1);
    return lane == 0 ? Line{1.0, 0.0} : before;
}

// The same where a lane's tokens may begin anew, so that nothing comes through them, not even what is not finite.
__device__ __forceinline__ Line scan_cuts(Line &m, bool &cut, int lane)
{
#pragma unroll
    for (int by = 1; by < 32; by *= 2) {
        const double P = __shfl_up_sync(kAll, m.P, by), B = __shfl_up_sync(kAll, m.B, by);
        const bool c = __shfl_up_sync(kAll, (int)cut, by);
        if (lane >= by && !cut) {
            m.B = fma(m.P, B, m.B);
            m.P *= P;
            cut = c;
        }
    }
    Line before;
    before.P = __shfl_up_sync(kAll, m.P, 1);
    before.B = __shfl_up_sync(kAll, m.B, 1);
    cut = __shfl_up_sync(kAll, (int)cut, 1);
    if (lane == 0) cut = false;
    return lane == 0 ? Line{1.0, 0.0} : before;
}

// The same where every lane's P is powers[0], with x before the first lane.
__device__ __forceinline__ double scan_even(double B, const double (&powers)[5], int lane, double x)
{
    if (lane == 0) B = fma(powers[0], x, B);
#pragma unroll
    for (int i = 0; i < 5; ++i) {
        const double before = __shfl_up_sync(kAll, B, 1 << i);
        if (lane >= (1 << i)) B = fma(powers[i], before, B);
    }
    const double before = __shfl_up_sync(kAll, B, 1);
    return lane == 0 ? x : before;
}

// A warp's way through the blocks of 256 tokens of [begin, end), from the last to the first (BACK: lane 0 has the last eight) or from
// the first to the last.  Masks run ahead of the tensors, and blocks of which no bit asks for anything are not read.
template <int TENSORS> struct FeedMemory { // of a warp
    Stage stage[kStages][TENSORS];
    uint2 mask[kMaskStages][32];
};
template <bool BACK, int TENSORS> struct Feed {
    FeedMemory<TENSORS> *mem;
    const uint8_t *mask;
    int begin, end, n_tok, off; // off: this lane's first token in a block
    int left;                   // blocks from this one on
    int base, i;                // this block's first token, its number
    uint32_t pipe;              // eight bits of each of the blocks that have been asked for
    bool vec;

    __device__ __forceinline__ static int ahead(int by) { return BACK ? -by * kBlock : by * kBlock; }
    // Whether the block from token b on can be read eight tokens at a time.
    __device__ __forceinline__ bool whole(int b) const { return vec && b + kBlock <= n_tok; }
    __device__ __forceinline__ void ask_mask(int by) const
    {
        if (mask == nullptr || by >= left) return;
        const int b = base + ahead(by);
        uint2 *to = &mem->mask[(i + by) & (kMaskStages - 1)][threadIdx.x & 31];
        if (whole(b)) copy_async(to, mask + b + off, 8);
        else *to = mask_bytes(mask, b + off, n_tok);
    }
    template <typename F> __device__ __forceinline__ void ask(int by, int slot, F fetch)
    {
        uint32_t v = 0;
        if (by < left) {
            const int b = base + ahead(by);
            v = b >= begin && b + kBlock <= end ? 0xFFu : range_bits(b + off, begin, end);
            if (mask != nullptr) v &= mask_bits(mem->mask[(i + by) & (kMaskStages - 1)][threadIdx.x & 31]);
            if (__any_sync(kAll, v != 0)) fetch(mem->stage[slot], b, whole(b));
        }
        pipe |= v << (8 * by);
    }
    template <typename F> __device__ __forceinline__ void start(F fetch)
    {
        const int last = (end - 1) & ~(kBlock - 1), first = begin & ~(kBlock - 1);
        base = BACK ? last : first;
        left = (last - first) / kBlock + 1;
        i = 0;
        pipe = 0;
#pragma unroll 1
        for (int by = 0; by < kMaskStages; ++by) ask_mask(by);
        copy_commit();
        copy_wait<0>();
#pragma unroll 1
        for (int by = 0; by < kStages; ++by) {
            ask(by, by, fetch);
            copy_commit();
        }
    }
    // Waits for this block: its bits; its tensors are in stage[slot], and the masks of the next blocks are there.
    __device__ __forceinline__ uint32_t arrive() const
    {
        copy_wait<kStages - 1>();
        __syncwarp();
        return pipe & 0xFFu;
    }
    // Once the block's tensors are in registers: asks for a later one in their place.
    template <typename F> __device__ __forceinline__ void release(int slot, F fetch)
    {
        __syncwarp();
        ask(kStages, slot, fetch);
        ask_mask(kMaskStages);
        copy_commit();
    }
    __device__ __forceinline__ void next()
    {
        pipe >>= 8;
        base += ahead(1);
        ++i;
        --left;
    }
};

// How many bits the lanes before this one have.
__device__ __forceinline__ int bits_before(uint32_t bits, int lane)
{
    const int own = __popc(bits);
    int n = own;
#pragma unroll
    for (int by = 1; by < 32; by *= 2) {
        const int more = __shfl_up_sync(kAll, n, by);
        if (lane >= by) n += more;
    }
    return n - own;
}

// MAPS: the map of the part of the chunk that goes on in the chunk before (even chunks), or of the piece that begins in it and is not its
// sequence's first.  Otherwise the outputs, from the chunk's last block of 256 tokens to its first, eight tokens to a lane.
//   A block inside one sequence: a lane's rightmost valid token takes the discounted value that follows it from the nearest lane to the right,
//   so that each lane's tokens are x' = P x + B; a scan of these over the warp gives every lane what comes in, a second walk the advantages.
//   Where all are valid P is the same power for all lanes, and the scan has one product a step.
//   A block with ends inside: the same, cut.  Sequences are numbered from the right by the bits of their ends; a valid token whose number is not
//   that of the valid token before it takes what is behind its sequence instead, and lets nothing through, not even what is not finite.
// The first form needs nothing but its own sequence's state, so a block's 17 bytes a token are on their way long before (copies into shared memory,
// three blocks ahead, masks eight ahead as they say what to copy).  What bounds it: memory for many tokens in sequences without masked parts (67 M
// tokens of padded rows 168 us, 6.8 TB/s counted over all of them, though masked parts are not read); latency of the steps of a block otherwise
// (4.3 M tokens in 2048 sequences with masked parts 43 us, 15 of maps, 25 of outputs and 5 of moments, partly behind one another).
// 24 warps an SM with all of its registers, 20 with a trace; with moments 8 bytes of a thread are spilled, 38 with a trace as well.  A form without
// a trace that spilled 36 took 184 us where this one takes 168.
template <bool TRACE, bool MOMENTS, bool MAPS> __global__ void __launch_bounds__(kAdvThreads, TRACE ? 5 : 6) advantage_kernel(const __grid_constant__ AdvantageArgs a)
{
    using Op = AdvantageOp;
    constexpr int kTensors = TRACE ? 3 : 2;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ Moments joined[kAdvWarps];
    __shared__ uint32_t ends_of[kAdvWarps][kBlock / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, chunk = blockIdx.x * kAdvWarps + warp;
    if (MAPS || !a.second) grid_dependency_wait();
    grid_dependency_release();
    const int live = a.q.live();
    double shift = 0.0, sum = 0.0, squares = 0.0; // moments about a value of the warp's own,
    bool known = false;                           // once there is one
    int taken = 0;                                // of so many
    if (chunk < a.chunks && (int64_t)chunk * a.chunk < live) {
        const int t0 = chunk * a.chunk, t1 = min(live - t0, a.chunk) + t0;
        int s, s1, begin = 0, end = 0, cur = 0; // cur: where the current sequence begins
        a.q.owner_warp2(t0, !a.even && t1 < live ? t1 : t1 - 1, lane, s, s1);
        Op::State st = Op::start();
        bool closed = false; // MAPS: the part holds its sequence's end
        int behind = 0;      // maps of the last sequence behind this chunk's part
        auto terminal = [&](int o) -> double {
            return (a.outcome ? (double)__ldg(a.outcome + o) : 0.0) + a.gamma * (a.bootstrap ? (double)__ldg(a.bootstrap + o) : 0.0);
        };
        if (MAPS) {
            const int b = a.q.bound(s), e = a.q.bound(s + 1);
            if (a.even) {
                if (b < t0) begin = t0, end = min(e, t1);
            } else {
                const uint32_t off = t0 > b ? (uint32_t)(t0 - b) : 0u, up = (off + (1u << a.piece) - 1) >> a.piece;
                const int64_t p = b + ((int64_t)max(up, 1u) << a.piece);
                if (p >= t0 && p < t1 && p < e) begin = (int)p, end = e - begin < (1 << a.piece) ? e : begin + (1 << a.piece);
            }
            closed = end == e;
            if (end > begin && closed) st.q = terminal(s);
        } else {
            begin = part_from(a, t0, s, live);
            end = part_from(a, t1, s1, live);
            if (end > begin) {
                s = s1;
                cur = a.q.bound(s);
                if (cur >= end) s = a.q.owner_warp(end - 1, lane), cur = a.q.bound(s);
                st.q = terminal(s);
                const int e = a.q.bound(s + 1);
                if (e > end) behind = a.even ? (int)((uint32_t)(e - 1) / (uint32_t)a.chunk) - chunk : (int)(((uint32_t)(e - end) + (1u << a.piece) - 1) >> a.piece);
            }
        }
        if (end > begin) {
            Feed<true, kTensors> feed;
            feed.mem = reinterpret_cast<FeedMemory<kTensors> *>(smem) + warp;
            feed.mask = a.mask, feed.begin = begin, feed.end = end, feed.n_tok = (int)a.q.n_tok, feed.off = (31 - lane) * 8, feed.vec = a.vec;
            auto fetch = [&](Stage (&to)[kTensors], int first, bool whole) {
                const int all = (int)a.q.n_tok;
                if (a.rewards) fetch_block(to[0], lane, a.rewards, first, all, whole);
                if (a.values) {
                    if (a.values_bf16) fetch_block(to[1], lane, static_cast<const uint16_t *>(a.values), first, all, whole);
                    else fetch_block(to[1], lane, static_cast<const float *>(a.values), first, all, whole);
                }
                if (TRACE) fetch_block(to[kTensors - 1], lane, a.trace, first, all, whole);
            };
            feed.start(fetch);
            if (!MAPS && a.second) {
                grid_dependency_wait();
                double none = 0.0;
                st = behind_pieces<Op>(st, behind, lane, [&](int i) {
                    const int far = behind - 1 - i;
                    return static_cast<const Op::Map *>(a.maps)[a.even ? chunk + 1 + far : (end + ((int64_t)far << a.piece)) / a.chunk]; }, none);
            }
            double P_all = 1.0, w_right = a.weight; // MAPS: product of the weights but the rightmost one's, and that
            int count = 0;
            int slot = 0;
#pragma unroll 1
            for (; feed.left > 0; feed.next(), slot = slot + 1 == kStages ? 0 : slot + 1) {
                const uint32_t valid = feed.arrive();
                const int base = feed.base, k = base + feed.off, lo = max(base, begin), hi = min(base + kBlock, end);
                const uint32_t some = __ballot_sync(kAll, valid != 0);
                float adv[8], ret[8];
                if (!MAPS && cur >= hi) { // on to the sequence before, whose end is where this block ends
                    s = a.q.owner_warp(hi - 1, lane);
                    cur = a.q.bound(s);
                    st = Op::State{0.0, terminal(s)};
                }
                Stage *x = feed.mem->stage[slot];
                float r[8], v[8], c[8];
                double D[8];
                auto read = [&]() {
                    if (a.rewards) read8(x[0], 31 - lane, r);
                    else zero8(r);
                    if (!a.values) zero8(v);
                    else if (a.values_bf16) read8_bf16(x[1], 31 - lane, v);
                    else read8(x[1], 31 - lane, v);
                    if (TRACE) read8(x[kTensors - 1], 31 - lane, c);
                };
                // Tokens of which some are masked.  CUTS: sequence number j, from the right, is that of the lane's last token but for the ends of
                // sequences among its tokens; behind number n there is later[n].
                auto uneven = [&](auto has_cuts, uint32_t ends, int j, const double *later) {
                    constexpr bool CUTS = decltype(has_cuts)::value;
                    // masked tokens hold the value that follows them, and leave B and z as they are
                    float leftmost = v[0];
#pragma unroll
                    for (int e = 7; e >= 0; --e)
                        if (valid >> e & 1) leftmost = v[e];
                    const uint32_t right = some & ((1u << lane) - 1);
                    const int near = right ? 31 - __clz(right) : 0;
                    const float from = __shfl_sync(kAll, leftmost, near);
                    const int j_left = CUTS && valid ? j + __popc(ends >> (__ffs(valid) - 1)) : 0;
                    int j_before = CUTS ? __shfl_sync(kAll, j_left, near) : 0; // of the valid token before
                    if (CUTS && !right) j_before = 0;
                    uint32_t cuts = 0; // valid tokens that are the last of their sequence
                    double q = right ? a.gamma * (double)from : st.q;
                    Line m{1.0, 0.0};
                    bool apart = MAPS && TRACE && count == 0 && right == 0; // this lane's first weight may be the piece's rightmost
#pragma unroll
                    for (int e = 7; e >= 0; --e) {
                        const bool in = valid >> e & 1;
                        const double V = (double)v[e];
                        const double w = TRACE ? a.weight * (double)c[e] : a.weight;
                        if (CUTS) {
                            j += ends >> e & 1;
                            if (in && j != j_before) {
                                q = later[j];
                                m.B = 0.0;
                                cuts |= 1u << e;
                            }
                            if (in) j_before = j;
                        }
                        D[e] = ((double)r[e] - V) + q;
                        if (in) m.B = fma(w, m.B, D[e]);
                        if (in) q = a.gamma * V;
                        if (TRACE) {
                            if (in && !apart) m.P *= w;
                            if (MAPS && in && apart) w_right = w, apart = false;
                        }
                    }
                    if (!TRACE) m.P = a.small[__popc(valid)];
                    if (MAPS && TRACE && count == 0) w_right = __shfl_sync(kAll, w_right, __ffs(some) - 1);
                    bool cut = cuts != 0;
                    const Line before = CUTS ? scan_cuts(m, cut, lane) : scan_lines(m, lane);
                    double z = CUTS && cut ? before.B : fma(before.P, st.x, before.B);
#pragma unroll
                    for (int e = 7; e >= 0; --e) {
                        adv[e] = ret[e] = 0.0f;
                        if (CUTS && (cuts >> e & 1)) z = 0.0;
                        if (valid >> e & 1) z = fma(TRACE ? a.weight * (double)c[e] : a.weight, z, D[e]);
                        D[e] = z;
                        if (valid >> e & 1) adv[e] = (float)z;
                        if (valid >> e & 1) ret[e] = (float)(z + (double)v[e]);
                    }
                    if (MAPS && TRACE) P_all *= __shfl_sync(kAll, m.P, 31);
                    st.x = __shfl_sync(kAll, z, 31);
                    st.q = a.gamma * (double)__shfl_sync(kAll, leftmost, 31 - __clz(some));
                    if (MAPS) count += TRACE ? 1 : (int)__reduce_add_sync(kAll, (unsigned)__popc(valid));
                    if (MOMENTS) {
                        // an advantage of the warp's first block: where the lane with the first bit ended
                        if (!known) shift = __shfl_sync(kAll, z, __ffs(some) - 1), known = true;
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const double d = D[e] - shift;
                            if (valid >> e & 1) sum += d;
                            if (valid >> e & 1) squares = fma(d, d, squares);
                        }
                        taken += __popc(valid);
                    }
                    return CUTS ? __shfl_sync(kAll, j_left, 31 - __clz(some)) : 0; // number of the sequence of the block's first valid token
                };
                if (MAPS || cur <= lo) {
                    if (some == 0) {
                        feed.release(slot, fetch);
                        zero8(adv);
                        zero8(ret);
                    } else {
                        read();
                        feed.release(slot, fetch);
                        if (!TRACE && __all_sync(kAll, valid == 0xFFu)) { // every lane's P is weight^8
                            const float from = __shfl_up_sync(kAll, v[0], 1);
                            double q = lane == 0 ? st.q : a.gamma * (double)from, B = 0.0;
#pragma unroll
                            for (int e = 7; e >= 0; --e) {
                                const double V = (double)v[e];
                                D[e] = ((double)r[e] - V) + q;
                                q = a.gamma * V;
                                B = fma(a.weight, B, D[e]);
                            }
                            double z = scan_even(B, a.powers, lane, st.x);
#pragma unroll
                            for (int e = 7; e >= 0; --e) {
                                D[e] = z = fma(a.weight, z, D[e]);
                                adv[e] = (float)z;
                                ret[e] = (float)(z + (double)v[e]);
                            }
                            st.x = __shfl_sync(kAll, z, 31);
                            st.q = a.gamma * (double)__shfl_sync(kAll, v[0], 31);
                            if (MAPS) count += kBlock;
                            if (MOMENTS) {
                                if (!known) shift = __shfl_sync(kAll, z, 0), known = true;
                                double s1[2] = {0.0, 0.0}, s2[2] = {0.0, 0.0};
#pragma unroll
                                for (int e = 0; e < 8; ++e) {
                                    const double d = D[e] - shift;
                                    s1[e & 1] += d;
                                    s2[e & 1] = fma(d, d, s2[e & 1]);
                                }
                                sum += s1[0] + s1[1];
                                squares += s2[0] + s2[1];
                                taken += 8;
                            }
                        } else {
                            uneven(std::false_type(), 0u, 0, nullptr);
                        }
                    }
                    if (!MAPS) {
                        if (a.vec && hi - lo == kBlock) {
                            if (a.adv) store8(a.adv + k, adv);
                            if (a.returns) store8(a.returns + k, ret);
                        } else {
                            if (a.adv) store8(a.adv, k, lo, hi, a.vec, adv);
                            if (a.returns) store8(a.returns, k, lo, hi, a.vec, ret);
                        }
                    }
                    continue;
                }
                if (MAPS) continue; // parts of one sequence
                // Sequences end inside, number 0 (from the right) is s.  The state behind each goes into memory that the tensors have left.
                read();
                uint32_t *bits = ends_of[warp];
                if (lane < kBlock / 32) bits[lane] = 0;
                __syncwarp();
                double *later = reinterpret_cast<double *>(x[0].x);
                int numbers = 0, right = 0x7FFFFFFF, others;
                for (;; s -= 32) {
                    const int o = s - lane, begins = o >= 0 ? a.q.bound(o) : 0;
                    int next = __shfl_up_sync(kAll, begins, 1);
                    if (lane == 0) next = right;
                    const uint32_t out = __ballot_sync(kAll, begins <= lo);
                    others = out ? __ffs(out) - 1 : 32;
                    const bool there = lane <= others && begins < next; // not empty
                    const uint32_t there_all = __ballot_sync(kAll, there);
                    if (there) later[min(numbers + __popc(there_all & ((1u << lane) - 1)), kBlock - 1)] = terminal(max(o, 0));
                    if (there && lane < others && begins <= hi) atomicOr(&bits[(begins - 1 - base) >> 5], 1u << ((begins - 1 - base) & 31));
                    numbers += __popc(there_all);
                    right = __shfl_sync(kAll, begins, 31);
                    if (out) {
                        cur = __shfl_sync(kAll, begins, others);
                        break;
                    }
                }
                s = max(s - others, 0);
                __syncwarp();
                const uint32_t ends = bits[feed.off >> 5] >> (feed.off & 31) & 0xFFu;
                const int j = bits_before(ends, lane); // ends behind the lane's tokens
                int j_first = 0;
                if (some != 0) {
                    j_first = uneven(std::true_type(), ends, j, later);
                } else {
                    zero8(adv);
                    zero8(ret);
                }
                numbers = min(numbers, kBlock) - 1;
                if (j_first != numbers) st = Op::State{0.0, later[numbers]};
                feed.release(slot, fetch);
                if (a.adv) store8(a.adv, k, lo, hi, a.vec, adv);
                if (a.returns) store8(a.returns, k, lo, hi, a.vec, ret);
            }
            if (MAPS && lane == 0) {
                // x' = Q (w x + q) + B,  q' = c
                const double Q = TRACE ? P_all : (count > 0 ? pow(a.weight, (double)(count - 1)) : 1.0);
                static_cast<Op::Map *>(a.maps)[chunk] = Op::Map{Q * w_right, Q, st.x, st.q, closed ? 2u : (count > 0 ? 1u : 0u), 0u};
            }
        }
    }
    if (!MAPS && a.second) grid_dependency_wait(); // no CTA ends before the maps' launch has
    if (MOMENTS) {
        const double n = (double)__reduce_add_sync(kAll, (unsigned)taken);
        sum = warp_sum(sum);
        squares = warp_sum(squares);
        if (lane == 0) joined[warp] = n > 0.0 ? Moments{n, shift + sum / n, squares - sum * sum / n} : Moments{0.0, 0.0, 0.0};
        __syncthreads();
        if (threadIdx.x == 0) {
            Moments m = joined[0];
            for (int w = 1; w < kAdvWarps; ++w) m.join(joined[w]);
            double *slot = a.partials + 3 * (size_t)blockIdx.x;
            slot[0] = m.n;
            slot[1] = m.mean;
            slot[2] = m.m2;
        }
    }
}

// Joins the CTAs' counts, means and sums of squared deviations in one launch: 845 of them for 4.3 M tokens, 5 us, 2731 for 67 M padded ones, one for every
// 16384 tokens (24576 in pieces) beyond some 20 M.
constexpr int kMomentThreads = 1024;

__global__ void __launch_bounds__(kMomentThreads) advantage_moments_kernel(const double *partials, int ctas, float *moments)
{
    __shared__ Moments sh[32];
    grid_dependency_wait();
    grid_dependency_release();
    Moments m{0.0, 0.0, 0.0};
#pragma unroll 4
    for (int t = threadIdx.x; t < ctas; t += kMomentThreads) m.join(Moments{partials[3 * (size_t)t], partials[3 * (size_t)t + 1], partials[3 * (size_t)t + 2]});
    m = warp_join(m);
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = m;
    __syncthreads();
    if (threadIdx.x < 32) {
        m = warp_join(sh[threadIdx.x]);
        if (threadIdx.x == 0) {
            moments[0] = (float)m.mean;
            moments[1] = m.n > 0.0 ? (float)sqrt(fmax(m.m2 / m.n, 0.0) + (m.m2 - m.m2)) : 0.0f; // NaN stays
        }
    }
}

constexpr int kGradThreads = 96; // three warps, as four of up to four tensors would not fit into 48 KB
constexpr int kGradWarps = kGradThreads / 32;

// The tokens of a chunk's part from the first to the last.  MAPS: the map of the part that goes on in the next chunk, or of the piece that begins in
// the chunk and is not its sequence's last.  Blocks as in the forward kernel; here a lane's first valid token takes the weight of the valid token
// before it from the nearest lane to the left, and every sequence that ends gives its last gradient.  d c of a token needs the advantage of its
// follower: where that is in a later block, the token stays open until then.
// 16 M tokens in 8000 sequences 75 us (3.6 TB/s): eight CTAs on an SM, 24 warps; with seven 86, with six 97, though with eight the outputs' form without a
// trace spills (52 bytes of a thread stored, 64 read).  By the trace as well (29 bytes a token, 150 registers) 13 M tokens with masked parts take 147 us
// with four CTAs, 169 with five, which spill.
template <bool TRACE, bool BY_TRACE, bool MAPS>
__global__ void __launch_bounds__(kGradThreads, BY_TRACE ? 4 : (TRACE ? 5 : 8)) advantage_grad_kernel(const __grid_constant__ AdvantageArgs a)
{
    using Op = AdvantageGradOp;
    constexpr int kTensors = 2 + TRACE + BY_TRACE;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ uint32_t ends_of[kGradWarps][kBlock / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, chunk = blockIdx.x * kGradWarps + warp;
    if (MAPS || !a.second) grid_dependency_wait();
    grid_dependency_release();
    const int live = a.q.live();
    const bool per_sequence = a.grad_outcome || a.grad_bootstrap;
    auto put = [&](int o, double G) {
        if (a.grad_outcome) a.grad_outcome[o] = (float)G;
        if (a.grad_bootstrap) a.grad_bootstrap[o] = (float)(a.gamma * G);
    };
    if (!MAPS && live <= 0) { // no tokens: no gradients
        if (a.second) grid_dependency_wait();
        if (per_sequence)
            for (int64_t o = (int64_t)blockIdx.x * kGradThreads + threadIdx.x; o < a.q.n_seq; o += (int64_t)gridDim.x * kGradThreads) put((int)o, 0.0);
        return;
    }
    int s = 0, s1, b = 0, begin = 0, end = 0, e_cur = live; // e_cur: where the current sequence ends
    bool opened = false; // MAPS: the part holds its sequence's beginning
    if (chunk < a.chunks && (int64_t)chunk * a.chunk < live) {
        const int t0 = chunk * a.chunk, t1 = min(live - t0, a.chunk) + t0;
        a.q.owner_warp2(t0, MAPS || a.even || t1 >= live ? t1 - 1 : t1, lane, s, s1);
        if (MAPS && a.even) {
            const int from = a.q.bound(s1);
            if (a.q.bound(s1 + 1) > t1) begin = max(t0, from), end = t1;
            opened = from >= t0;
        } else if (MAPS) {
#pragma unroll 1
            for (int which = 0; which < 2; ++which) { // of the chunk's first sequence, or of its last
                const int o = which == 0 ? s : s1, from = a.q.bound(o), e = a.q.bound(o + 1);
                const uint32_t off = t0 > from ? (uint32_t)(t0 - from) : 0u, up = ((off + (1u << a.piece) - 1) >> a.piece) << a.piece;
                const int64_t p = (int64_t)from + up;
                if (p >= t0 && p < t1 && p + (1 << a.piece) < e) begin = (int)p, end = begin + (1 << a.piece), opened = p == from;
            }
        } else {
            begin = part_from(a, t0, s, live);
            end = part_from(a, t1, s1, live);
        }
    }
    const int s_first = s;
    if (!MAPS && end > begin) {
        b = a.q.bound(s);
        e_cur = a.q.bound(s + 1);
        if (begin >= e_cur) s = a.q.owner_warp(begin, lane), b = a.q.bound(s), e_cur = a.q.bound(s + 1);
    }
    Feed<false, kTensors> feed;
    feed.mem = reinterpret_cast<FeedMemory<kTensors> *>(smem) + warp;
    feed.mask = a.mask, feed.begin = begin, feed.end = end, feed.n_tok = (int)a.q.n_tok, feed.off = lane * 8, feed.vec = a.vec;
    auto fetch = [&](Stage (&to)[kTensors], int first, bool whole) {
        const int all = (int)a.q.n_tok;
        if (a.grad_adv) fetch_block(to[0], lane, a.grad_adv, first, all, whole);
        if (a.grad_returns) fetch_block(to[1], lane, a.grad_returns, first, all, whole);
        if (TRACE) fetch_block(to[2], lane, a.trace, first, all, whole);
        if (BY_TRACE) fetch_block(to[kTensors - 1], lane, a.adv_in, first, all, whole);
    };
    if (end > begin) feed.start(fetch);
    if (!MAPS && a.second) grid_dependency_wait(); // for the maps; and no CTA ends before their launch has
    if (!MAPS && per_sequence && chunk == 0)       // sequences without a token ahead of the first one
        for (int o = lane; o < s_first; o += 32) put(o, 0.0);
    if (end <= begin)
        return;
    Op::State st = Op::start();
    double w_before = 0.0; // TRACE: weight of the valid token before
    if (!MAPS && a.second)
        st = behind_pieces<Op>(st, begin <= b ? 0 : (a.even ? chunk - b / a.chunk : (begin - b) >> a.piece), lane,
                               [&](int i) { return static_cast<const Op::Map *>(a.maps)[a.even ? b / a.chunk + i : (b + ((int64_t)i << a.piece)) / a.chunk]; }, w_before);
    if (BY_TRACE && (uint32_t)st.pos >= (uint32_t)live) st.pos = -1; // boundaries out of order: a map that nobody made
    // The current sequence's last gradient, then on to the one that holds token `to`; those between without a token get zeros.
    auto next_sequence = [&](int to) {
        if (lane == 0) {
            if (BY_TRACE && st.pos >= 0) a.grad_trace[st.pos] = 0.0f; // nothing follows
            put(s, st.G);
        }
        for (int64_t base = (int64_t)s + 1;; base += 32) {
            const int64_t o = base + lane;
            const uint32_t hit = __ballot_sync(kAll, o >= a.q.n_seq || a.q.bound((int)o + 1) > to);
            if (per_sequence && o < a.q.n_seq && lane < (hit ? __ffs(hit) - 1 : 32)) put((int)o, 0.0);
            if (hit) {
                const int64_t at = base + __ffs(hit) - 1;
                s = (int)(at < a.q.n_seq ? at : a.q.n_seq - 1);
                break;
            }
        }
        e_cur = a.q.bound(s + 1);
        if (e_cur <= to) e_cur = live; // behind the last one, or boundaries out of order
        st = Op::start();
        w_before = 0.0;
    };
    double P_all = 1.0; // MAPS: product of the weights but the last one's
    int count = 0;
    int slot = 0;
#pragma unroll 1
    for (; feed.left > 0; feed.next(), slot = slot + 1 == kStages ? 0 : slot + 1) {
        const uint32_t valid = feed.arrive();
        const int base = feed.base, k = base + feed.off, lo = max(base, begin), hi = min(base + kBlock, end);
        if (!MAPS && e_cur <= lo) next_sequence(lo);
        const uint32_t some = __ballot_sync(kAll, valid != 0);
        Stage *x = feed.mem->stage[slot];
        float dr[8], dv[8], dc[8];
        int open = -1; // this lane's token that waits for its follower
        float ga[8], gr[8], c[8], A[8];
        double g[8];
        auto read = [&]() {
            if (a.grad_adv) read8(x[0], lane, ga);
            else zero8(ga);
            if (a.grad_returns) read8(x[1], lane, gr);
            else zero8(gr);
            if (TRACE) read8(x[2], lane, c);
            if (BY_TRACE) read8(x[kTensors - 1], lane, A);
        };
        auto store = [&]() {
            if (a.vec && hi - lo == kBlock) {
                if (a.grad_rewards) store8(a.grad_rewards + k, dr);
                if (a.grad_values) store8(a.grad_values + k, dv);
            } else {
                if (a.grad_rewards) store8(a.grad_rewards, k, lo, hi, a.vec, dr);
                if (a.grad_values) store8(a.grad_values, k, lo, hi, a.vec, dv);
            }
            if (BY_TRACE) {
                if (open < 0) store8(a.grad_trace, k, lo, hi, a.vec, dc);
                else
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (k + e >= lo && k + e < hi && k + e != open) a.grad_trace[k + e] = dc[e];
            }
        };
        // The gradient by the trace of the block's tokens, whose own gradients are in g.  CUTS: as below, n the number of the last sequence.
        auto by_trace = [&](auto has_cuts, uint32_t ends, int j, int n) {
            constexpr bool CUTS = decltype(has_cuts)::value;
            const uint32_t left = some & ((1u << lane) - 1), right = lane == 31 ? 0u : some & (0xFFFFFFFEu << lane);
            float first_A = 0.0f;
#pragma unroll
            for (int e = 7; e >= 0; --e) first_A = valid >> e & 1 ? A[e] : first_A;
            const int j_first = CUTS && valid ? j + __popc(ends & ((1u << (__ffs(valid) - 1)) - 1)) : 0;
            if (!left && valid && st.pos >= 0) // the token left open by a block before
                a.grad_trace[st.pos] = CUTS && j_first != 0 ? 0.0f : (float)(a.weight * (double)first_A * st.G);
            const int near = right ? __ffs(right) - 1 : 0;
            float next_A = __shfl_sync(kAll, first_A, near);
            int j_next = CUTS ? __shfl_sync(kAll, j_first, near) : 0;
            bool known = right != 0;
#pragma unroll
            for (int e = 7; e >= 0; --e) {
                const bool in = valid >> e & 1;
                const int j_of = CUTS ? j + __popc(ends & ((1u << e) - 1)) : 0;
                dc[e] = in && (!CUTS || (known && j_next == j_of)) ? (float)(a.weight * (double)next_A * g[e]) : 0.0f;
                if (in && !known && (!CUTS || j_of == n)) open = k + e;
                if (in) next_A = A[e], j_next = j_of;
                known = known || in;
            }
        };
        // Tokens of which some are masked.  CUTS: `ends` are those of the lane's tokens that end their sequence, the first of them is of sequence
        // number j, counted from the left; the last gradient of number j, if it ends, goes to lasts[j].
        auto uneven = [&](auto has_cuts, uint32_t ends, int j, double *lasts) {
            constexpr bool CUTS = decltype(has_cuts)::value;
            const uint32_t left = some & ((1u << lane) - 1);
            const int from = left ? 31 - __clz(left) : 0, tail = 31 - __clz(some);
            double w_in = a.weight;
            if (TRACE) {
                float c_last = 0.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) c_last = valid >> e & 1 ? c[e] : c_last;
                const float before = __shfl_sync(kAll, c_last, from);
                w_in = left ? a.weight * (double)before : w_before;
                w_before = a.weight * (double)__shfl_sync(kAll, c_last, tail);
            }
            const int j_last = CUTS && valid ? j + __popc(ends & ((1u << (31 - __clz(valid))) - 1)) : 0;
            int j_before = CUTS ? __shfl_sync(kAll, j_last, from) : 0; // of the valid token before
            if (CUTS && !left) j_before = 0;
            const int j_in = j_before;
            int j_now = j;
            uint32_t cuts = 0; // valid tokens that are the first of their sequence
            Line m{1.0, 0.0};
            double w = MAPS && TRACE && count == 0 && !left ? 1.0 : w_in; // the weight of what comes into the piece is applied to it before
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const bool in = valid >> e & 1;
                if (CUTS && in && j_now != j_before) cuts |= 1u << e, m.B = w = 0.0;
                if (CUTS && in) j_before = j_now;
                if (CUTS) j_now += ends >> e & 1;
                const double sum = (double)ga[e] + (double)gr[e], B = fma(w, m.B, sum);
                if (!CUTS) g[e] = sum;
                m.B = in ? B : m.B;
                if (TRACE) {
                    const double P = w * m.P;
                    m.P = in ? P : m.P;
                    w = in ? a.weight * (double)c[e] : w;
                } else if (CUTS) {
                    w = a.weight;
                }
            }
            if (!TRACE) m.P = a.small[__popc(valid)];
            bool cut = cuts != 0;
            const Line before = CUTS ? scan_cuts(m, cut, lane) : scan_lines(m, lane);
            double G = CUTS && cut ? before.B : fma(before.P, st.G, before.B);
            if (MAPS && TRACE) P_all *= __shfl_sync(kAll, m.P, 31);
            w = w_in;
            j_before = j_in;
            if (CUTS) { // once more, as registers to hold it would cost all blocks
                __syncwarp();
                read();
                __syncwarp();
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const bool in = valid >> e & 1;
                if (CUTS && (cuts >> e & 1)) G = w = 0.0;
                const double now = fma(w, G, CUTS ? (double)ga[e] + (double)gr[e] : g[e]);
                dr[e] = in ? (float)now : 0.0f;
                dv[e] = in ? (float)(fma(a.gamma, G, (double)gr[e]) - now) : 0.0f;
                g[e] = now;
                G = in ? now : G;
                if (TRACE) w = in ? a.weight * (double)c[e] : w;
                else if (CUTS) w = a.weight;
                if (CUTS) {
                    if (in) j_before = j;
                    if (ends >> e & 1) lasts[min(j, kBlock - 1)] = j_before == j ? G : 0.0, ++j;
                }
            }
            st.G = __shfl_sync(kAll, G, tail);
            return CUTS ? __shfl_sync(kAll, j_last, tail) : 0; // number of the sequence of the block's last valid token
        };
        const int last_of = valid ? k + 31 - __clz(valid) : -1;
        if (MAPS || e_cur >= hi) {
            if (some == 0) {
                feed.release(slot, fetch);
                zero8(dr);
                zero8(dv);
                if (BY_TRACE) zero8(dc);
            } else {
                read();
                feed.release(slot, fetch);
                if (!TRACE && __all_sync(kAll, valid == 0xFFu)) { // every lane's P is weight^8
                    double B = 0.0;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        g[e] = (double)ga[e] + (double)gr[e];
                        B = fma(a.weight, B, g[e]);
                    }
                    double G = scan_even(B, a.powers, lane, st.G);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const double now = fma(a.weight, G, g[e]);
                        dr[e] = (float)now;
                        dv[e] = (float)(fma(a.gamma, G, (double)gr[e]) - now);
                        G = g[e] = now;
                    }
                    if (BY_TRACE && !MAPS) by_trace(std::false_type(), 0u, 0, 0);
                    st.G = __shfl_sync(kAll, G, 31);
                } else {
                    const double G_before = st.G;
                    uneven(std::false_type(), 0u, 0, nullptr);
                    if (BY_TRACE && !MAPS) {
                        const double G_now = st.G;
                        st.G = G_before;
                        by_trace(std::false_type(), 0u, 0, 0);
                        st.G = G_now;
                    }
                }
                st.pos = __shfl_sync(kAll, last_of, 31 - __clz(some));
                if (MAPS) count += TRACE ? 1 : (int)__reduce_add_sync(kAll, (unsigned)__popc(valid));
            }
            if (!MAPS) store();
            continue;
        }
        if (MAPS) continue; // parts of one sequence
        // Sequences end inside, number 0 (from the left) is s.
        uint32_t *bits = ends_of[warp];
        if (lane < kBlock / 32) bits[lane] = 0;
        __syncwarp();
        const int s_left = s;
        int numbers = 0, others;
        // all of them: f(sequence, its number, whether it ends inside, where) by a lane of each that is not empty, and empty(sequence)
        auto each = [&](auto f, auto empty) {
            numbers = 0;
            int left = INT_MIN;
            for (int from = s_left;; from += 32) {
                const int64_t o = (int64_t)from + lane;
                const int behind = o < a.q.n_seq ? a.q.bound((int)o + 1) : 0x7FFFFFFF;
                int before = __shfl_up_sync(kAll, behind, 1);
                if (lane == 0) before = left;
                const uint32_t out = __ballot_sync(kAll, behind >= hi);
                others = out ? __ffs(out) - 1 : 32;
                const bool there = lane <= others && behind > before;
                const uint32_t there_all = __ballot_sync(kAll, there);
                if (there) f((int)o, min(numbers + __popc(there_all & ((1u << lane) - 1)), kBlock - 1), lane < others, behind);
                else if (lane < others) empty((int)o);
                numbers += __popc(there_all);
                left = __shfl_sync(kAll, behind, 31);
                if (out) {
                    s = (int)min((int64_t)from + others, a.q.n_seq - 1);
                    e_cur = __shfl_sync(kAll, behind, others);
                    if (e_cur == 0x7FFFFFFF) e_cur = live;
                    break;
                }
            }
        };
        each([&](int, int, bool ends, int behind) {
            if (ends && behind > base) atomicOr(&bits[(behind - 1 - base) >> 5], 1u << ((behind - 1 - base) & 31)); }, [&](int) {});
        __syncwarp();
        const uint32_t ends = bits[feed.off >> 5] >> (feed.off & 31) & 0xFFu;
        const int j = bits_before(ends, lane); // ends before the lane's tokens
        numbers = min(numbers, kBlock) - 1;
        double *lasts = reinterpret_cast<double *>(x[0].x); // in the tensors' place once they have been read
        int j_last = 0;
        const int n = numbers;
        if (some != 0) {
            read();
            const double G_before = st.G;
            j_last = uneven(std::true_type(), ends, j, lasts);
            if (BY_TRACE) {
                const double G_now = st.G;
                st.G = G_before;
                by_trace(std::true_type(), ends, j, n);
                st.G = G_now;
            }
            st.pos = __shfl_sync(kAll, last_of, 31 - __clz(some));
        } else {
            zero8(dr);
            zero8(dv);
            if (BY_TRACE) zero8(dc);
            if (BY_TRACE && lane == 0 && st.pos >= 0) a.grad_trace[st.pos] = 0.0f; // nothing follows
            for (int i = lane; i < n; i += 32) lasts[i] = i == 0 ? st.G : 0.0;
        }
        store();
        __syncwarp();
        if (per_sequence)
            each([&](int o, int number, bool ends, int) {
                if (ends) put(o, lasts[number]); }, [&](int o) { put(o, 0.0); });
        if (j_last != n) st = Op::start(), w_before = 0.0;
        feed.release(slot, fetch);
    }
    if (MAPS) {
        const double P = TRACE ? P_all : (count > 0 ? pow(a.weight, (double)(count - 1)) : 1.0);
        if (lane == 0)
            static_cast<Op::Map *>(a.maps)[chunk] = Op::Map{P, st.G, TRACE ? w_before : a.weight, st.pos, opened ? 2u : (count > 0 ? 1u : 0u)};
    } else if (e_cur <= end) {
        next_sequence(end);
    }
}

static bool all_vectors(const AdvantageArgs &a)
{
    return vectors({a.rewards, a.trace, a.adv, a.returns, a.grad_adv, a.grad_returns, a.adv_in, a.grad_rewards, a.grad_values, a.grad_trace}, a.mask) &&
           aligned(a.values, a.values_bf16 ? 16 : 32);
}

// Even chunks read most of a long sequence twice, for its maps and for itself, pieces are uneven work.  Forward, us, even chunks and pieces:
// 8 M tokens in sequences of 2000: 59, 46; of 130 K: 49, 101.  40 M tokens in sequences of 2000: 189, 145; of 6700: 184, 157; of 13 K: 185, 232;
// of 400 K: 180, 247.  16 M tokens in 2000 sequences: 90, 92.  So pieces need sequences for most warps, of a length that few of them pass.
// A warp joins the maps of all chunks of its last sequence behind its own, so a sequence's maps are read half its chunks' square times: a call of one
// sequence of 16 M tokens takes 172 us, of 60 M 1370, of 240 M 27000, most of it this.
// Largest chunks: of 40 M tokens in even chunks of 16 blocks 180 us, in one wave of 43 212; in pieces from chunks of 16 blocks 154 us, of 24 145,
// of 32 157.
constexpr int64_t kWarps = 148 * 24; // warps that run at once without a trace; with one 148 * 20, in the gradient 148 * 15, or 12 by the trace
constexpr int kLargestEven = 16, kLargestPieces = 24; // blocks of a chunk where warps do not all run at once
static void deal(AdvantageArgs &a)
{
    const int64_t share = (a.q.n_tok + kWarps * kBlock - 1) / (kWarps * kBlock); // blocks of a warp if all run at once
    a.even = share <= 8 || a.q.n_seq < kWarps * 7 / 10 || a.q.n_tok / a.q.n_seq >= 8192;
    const int largest = a.even ? kLargestEven : kLargestPieces;
    a.chunk = kBlock * (int)(share < 1 ? 1 : (share > largest + largest / 2 ? largest : share));
    if (a.q.n_tok <= 4 * kBlock) a.chunk = 4 * kBlock; // one launch instead of two
    a.piece = 14;
    a.chunks = (int)((a.q.n_tok + a.chunk - 1) / a.chunk);
    for (int i = 0; i < 9; ++i) a.small[i] = std::pow(a.weight, i);
    a.powers[0] = a.small[8];
    for (int i = 1; i < 5; ++i) a.powers[i] = a.powers[i - 1] * a.powers[i - 1];
}

// Whether there can be maps to make, as far as the host knows.
static bool long_sequences(const AdvantageArgs &a)
{
    if (a.even) return a.chunks > 1;
    return (a.q.cu ? a.q.n_tok : a.q.T) > (int64_t)1 << a.piece;
}

} // namespace hilore

using namespace hilore;

extern "C" size_t hilore_advantages_workspace_bytes(int64_t n_tok)
{
    // chunks of any number of tokens up to n_tok: no more than run at once, or of the smaller of the largest sizes
    const int64_t blocks = n_tok > 0 ? (n_tok + kBlock - 1) / kBlock : 0;
    const size_t chunks = (size_t)std::max(std::min(blocks, kWarps), (blocks + kLargestEven - 1) / kLargestEven);
    return (chunks + 1) * sizeof(AdvantageOp::Map) + (chunks / kAdvWarps + 1) * 3 * sizeof(double);
}

extern "C" int hilore_advantages(const float *rewards, const float *outcome, const void *values, int32_t values_dtype, const float *bootstrap,
                                 const float *trace, const uint8_t *mask, const int32_t *cu_seqlens, int64_t n_seq, int64_t n_tok,
                                 double gamma, double lambda, float *adv, float *returns, float *moments, void *workspace,
                                 size_t workspace_bytes, void *stream)
{
    AdvantageArgs a{};
    if (!(gamma >= 0.0 && gamma <= 1.0) || !(lambda >= 0.0 && lambda <= 1.0) || (values_dtype != HILORE_BF16 && values_dtype != HILORE_F32))
        return HILORE_INVALID_ARG;
    const int bad = check_sequences(cu_seqlens, n_seq, n_tok, a.q);
    if (bad)
        return bad;
    if (!workspace || (n_tok > 0 && !adv && !returns && !moments))
        return HILORE_INVALID_ARG;
    a.rewards = rewards, a.outcome = outcome, a.values = values, a.values_bf16 = values_dtype == HILORE_BF16, a.bootstrap = bootstrap;
    a.trace = trace, a.mask = mask, a.gamma = gamma, a.weight = gamma * lambda, a.adv = adv, a.returns = returns;
    if (!aligned(rewards, 4) || !aligned(outcome, 4) || !aligned(bootstrap, 4) || !aligned(trace, 4) || !aligned(adv, 4) || !aligned(returns, 4) ||
        !aligned(moments, 4) || !aligned(values, a.values_bf16 ? 2 : 4) || !aligned(workspace, 16))
        return HILORE_ALIGN;
    if (workspace_bytes < hilore_advantages_workspace_bytes(n_tok))
        return HILORE_WORKSPACE;
    a.maps = workspace;
    a.vec = all_vectors(a);
    deal(a);
    a.partials = reinterpret_cast<double *>(static_cast<AdvantageOp::Map *>(workspace) + a.chunks + 1);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const unsigned grid = (unsigned)((a.chunks + kAdvWarps - 1) / kAdvWarps);
    const size_t smem = kAdvWarps * (trace ? sizeof(FeedMemory<3>) : sizeof(FeedMemory<2>));
    a.second = long_sequences(a);
    if (grid > 0 && a.second &&
        launch_dependent(trace ? advantage_kernel<true, false, true> : advantage_kernel<false, false, true>, dim3(grid), dim3(kAdvThreads), smem, st, a) != cudaSuccess)
        return HILORE_CUDA;
    void (*kernel)(AdvantageArgs) = moments ? (trace ? advantage_kernel<true, true, false> : advantage_kernel<false, true, false>)
                                            : (trace ? advantage_kernel<true, false, false> : advantage_kernel<false, false, false>);
    if (grid > 0 && launch_dependent(kernel, dim3(grid), dim3(kAdvThreads), smem, st, a) != cudaSuccess)
        return HILORE_CUDA;
    if (moments && launch_dependent(advantage_moments_kernel, dim3(1), dim3(kMomentThreads), 0, st, (const double *)a.partials, (int)grid, moments) != cudaSuccess)
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
    const int bad = check_sequences(cu_seqlens, n_seq, n_tok, a.q);
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
    deal(a);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (n_seq == 0)
        return HILORE_OK;
    const unsigned grid = a.chunks > 0 ? (unsigned)((a.chunks + kGradWarps - 1) / kGradWarps) : 1u;
    void (*const maps)(AdvantageArgs) = trace ? advantage_grad_kernel<true, false, true> : advantage_grad_kernel<false, false, true>;
    void (*const kernel)(AdvantageArgs) =
        grad_trace ? (trace ? advantage_grad_kernel<true, true, false> : advantage_grad_kernel<false, true, false>)
                   : (trace ? advantage_grad_kernel<true, false, false> : advantage_grad_kernel<false, false, false>);
    const size_t smem[3] = {kGradWarps * sizeof(FeedMemory<2>), kGradWarps * sizeof(FeedMemory<3>), kGradWarps * sizeof(FeedMemory<4>)};
    a.second = long_sequences(a);
    if (a.second && launch_dependent(maps, dim3(grid), dim3(kGradThreads), smem[trace != nullptr], st, a) != cudaSuccess)
        return HILORE_CUDA;
    if (launch_dependent(kernel, dim3(grid), dim3(kGradThreads), smem[(trace != nullptr) + (grad_trace != nullptr)], st, a) != cudaSuccess)
        return HILORE_CUDA;
    return cudaGetLastError() == cudaSuccess ? HILORE_OK : HILORE_CUDA;
}
