// The vocabulary end of an actor update: rules on logits (penalties for repeated tokens, biases, grammar masks,
// temperature), log-probabilities of the sampled tokens under them, and the gradient of the logits from the update
// coefficients omega_t = dL/dlogp_t that the coefficient pass writes.
//
// All of it streams rows of V logits once, so HBM is the bound; what a row's rules say about single tokens is kept
// off that stream.  A CTA owns a range of the vocabulary and walks a block of consecutive rows.  It keeps the tokens of the
// row's history in a table of counts in shared memory, with a list of those that occur.  The slots of a training sequence
// have growing prefixes of one sequence as their histories: going to the next row then adds a token or two to the table
// instead of clearing it and scanning the history again (gradient of 2048 x 128256 bf16 rows under prefixes of up
// to 1536 tokens: 248 us, 301 with a scan per row; the bytes alone 163).  The stream runs as if no token were listed; the listed
// ones are worked out on their own, one per thread, and written over the stream's results or, where a sum is wanted, left out of
// the stream by one bit per token.  Other ways: counts asked for inside the stream, where a warp takes its listed tokens one
// by one, took 930 us for that gradient; a hash table over a larger range, which probes and overflows, 320 us for 96 rows of 151936
// fp32 logits with histories of up to 16384 tokens, now 55 (the bytes 19).  Counts in global memory would cost 4 bytes per
// logit, twice the bf16 logits themselves.
#include "common.cuh"

#include <cooperative_groups.h>
#include <cstdlib>

namespace cg = cooperative_groups;

namespace hilore {

constexpr float kLog2eF = 1.4426950408889634f;
constexpr float kLowest = -3.402823466e38f; // the running maximum of a row starts here: a row of -inf keeps a finite one
constexpr float kNothing = -1e30f;          // an lse at or below this belongs to a row without a token to choose from
constexpr uint32_t kSeen = 0x80000000u;     // bit of a count: the token occurs in the history

__device__ __forceinline__ float ex2_ftz(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// 32 bytes of logits as fp32 values.
template <typename T> struct Lane;
template <> struct Lane<uint16_t> { // bf16
    static constexpr int N = 16;
    static __device__ __forceinline__ float one(const uint16_t *p) { return __uint_as_float((uint32_t)*p << 16); }
    static __device__ __forceinline__ void put(uint16_t *p, float v) { *p = (uint16_t)cvt_bf16x2(0.0f, v); }
    static __device__ __forceinline__ void unpack(const uint32_t (&w)[8], float (&z)[16])
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            z[2 * i] = bf16_lo(w[i]);
            z[2 * i + 1] = bf16_hi(w[i]);
        }
    }
    static __device__ __forceinline__ void pack(const float (&z)[16], uint32_t (&w)[8])
    {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            w[i] = cvt_bf16x2(z[2 * i + 1], z[2 * i]);
    }
};
template <> struct Lane<float> {
    static constexpr int N = 8;
    static __device__ __forceinline__ float one(const float *p) { return *p; }
    static __device__ __forceinline__ void put(float *p, float v) { *p = v; }
    static __device__ __forceinline__ void unpack(const uint32_t (&w)[8], float (&z)[8])
    {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            z[i] = __uint_as_float(w[i]);
    }
    static __device__ __forceinline__ void pack(const float (&z)[8], uint32_t (&w)[8])
    {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            w[i] = __float_as_uint(z[i]);
    }
};

// A row in the frame of its 32-byte vectors: position f = v + lead, so that position 0 is 32-byte aligned whatever the
// leading dimension is.  Vectors are moved where they lie wholly in the row; what is left at its two ends goes element by
// element, a thread each, out of the way of the vectors' code.
template <typename T> struct Row {
    T *origin; // address of position 0; never dereferenced outside [lead, end)
    int lead, end;
    __device__ __forceinline__ Row(const T *row, int V)
    {
        lead = (int)((reinterpret_cast<uintptr_t>(row) & 31) / sizeof(T));
        origin = const_cast<T *>(row) - lead;
        end = lead + V;
    }
    // Positions [a, b) as far as they are the row's: elements [lo, fa), vectors [fa, fb), elements [fb, hi).
    struct Parts {
        int lo, fa, fb, hi;
    };
    __device__ __forceinline__ Parts parts(int a, int b) const { return parts(a, b, lead, end); }
    __device__ __forceinline__ Parts parts(int a, int b, int first, int last) const // vectors within [first, last) alone
    {
        constexpr int N = Lane<T>::N;
        Parts p{max(a, lead), 0, 0, min(b, end)};
        p.fa = (max(p.lo, first) + N - 1) & ~(N - 1);
        p.fb = min(p.hi, last) & ~(N - 1);
        if (p.fa >= p.fb) p.fa = p.fb = p.hi;
        return p;
    }
    __device__ __forceinline__ void load(int f, uint32_t (&w)[8]) const { ld_global_256(origin + f, w); }
    __device__ __forceinline__ void store(int f, const float (&z)[Lane<T>::N]) const
    {
        uint32_t w[8];
        Lane<T>::pack(z, w);
        st_global_256(origin + f, w);
    }
};

// Calls f(position) for the elements of `p` that are in no vector.
template <int THREADS, typename P, typename F> __device__ __forceinline__ void each_edge(const P &p, const F &f)
{
    const int left = max(p.fa - p.lo, 0), n = left + max(p.hi - p.fb, 0);
#pragma unroll 1
    for (int i = threadIdx.x; i < n; i += THREADS)
        f(i < left ? p.lo + i : p.fb + (i - left));
}

// Reads of a row in the frame of another one (the row that is written).  Where the two addresses differ modulo 32 bytes, a
// vector is put together from two neighbouring aligned ones by a shift of whole words and, for bf16, of half a word; the
// second one hits L1.  (Element-wise stores instead took 8.6 times as long as the bytes.)
template <typename T> struct Source {
    const T *exact;   // exact + f is the element of position f
    const T *aligned; // aligned + f starts the aligned vector of the read row that holds it, `shift` elements earlier
    int shift;        // 0: the frames agree
    Row<T> own;       // the read row in its own frame
    __device__ __forceinline__ Source(const T *row, int V, const Row<T> &frame) : own(row, V)
    {
        exact = row - frame.lead;
        const int d = own.lead - frame.lead; // position f of the frame is position f + d of the read row's own frame
        shift = d < 0 ? d + Lane<T>::N : d;
        aligned = own.origin + (d - shift);  // d - shift is 0 or -N
    }
    // Parts of positions [a, b) of the frame whose vectors can be read.
    __device__ __forceinline__ typename Row<T>::Parts parts(const Row<T> &frame, int a, int b) const
    {
        if (shift == 0) return frame.parts(a, b);
        const int to_own = (int)(aligned - own.origin); // position f of the frame: the vectors at f + to_own and the next one
        return frame.parts(a, b, max(frame.lead, own.lead - to_own), min(frame.end, own.end - to_own - Lane<T>::N));
    }
    template <bool SHIFTED> __device__ __forceinline__ void load(int f, uint32_t (&w)[8]) const
    {
        if (!SHIFTED) {
            ld_global_256(exact + f, w);
            return;
        }
        constexpr int N = Lane<T>::N;
        uint32_t v[16];
        ld_cached(aligned + f, v);
        ld_cached(aligned + f + N, v + 8);
        constexpr int kPerWord = 4 / (int)sizeof(T);
        const int words = shift / kPerWord;
#pragma unroll
        for (int k = 4; k > 0; k >>= 1)
            if (words & k) {
#pragma unroll
                for (int i = 0; i + k < 16; ++i)
                    v[i] = v[i + k];
            }
        const bool half = kPerWord == 2 && (shift & 1);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            w[i] = half ? __funnelshift_r(v[i], v[i + 1], 16) : v[i];
    }
    static __device__ __forceinline__ void ld_cached(const T *p, uint32_t *v)
    {
        asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                     : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
                     : "l"(p));
    }
};

// ------------------------------------------------------------------------------------------------------ the rules of a row
struct RowRules {
    float inv_temp, rep, inv_rep, freq, pres;
    int64_t hist_lo, hist_mid, hist_hi; // history; empty where the penalties of the row are neutral
    int64_t bias_lo, bias_hi;
    const uint32_t *mask; // words of the grammar, or nullptr
    __device__ __forceinline__ bool history() const { return hist_lo < hist_hi; }
    __device__ __forceinline__ bool listed() const { return hist_lo < hist_hi || bias_lo < bias_hi; }
};

__device__ __forceinline__ float inverse_temperature(const float *temperature, int64_t row)
{
    const float t = temperature ? temperature[row] : 1.0f;
    return t > 0.0f ? __fdiv_rn(1.0f, t) : 1.0f; // 0 (greedy) and what is no temperature: not scaled
}

// The inverse temperature of a softmax: that of an infinite temperature is the smallest number instead of zero, whose product with
// the -inf of a denied token would be NaN.
__device__ __forceinline__ float softmax_factor(float inv_temp) { return fmaxf(inv_temp, __uint_as_float(1u)); }

__device__ __forceinline__ RowRules row_rules(const hilore_logit_rules &R, int64_t row)
{
    RowRules q;
    q.inv_temp = inverse_temperature(R.temperature, row);
    q.rep = R.repetition ? R.repetition[row] : 1.0f;
    q.inv_rep = __fdiv_rn(1.0f, q.rep);
    q.freq = R.frequency ? R.frequency[row] : 0.0f;
    q.pres = R.presence ? R.presence[row] : 0.0f;
    q.hist_lo = q.hist_hi = q.hist_mid = q.bias_lo = q.bias_hi = 0;
    if (R.tokens) {
        const int64_t lo = max((int64_t)0, R.hist_begin[row]), mid = R.resp_begin[row], hi = min(R.n_tokens, R.hist_end[row]);
        if (lo < hi && !(q.rep == 1.0f && q.freq == 0.0f && q.pres == 0.0f)) {
            q.hist_lo = lo;
            q.hist_mid = min(max(mid, lo), hi);
            q.hist_hi = hi;
        }
    }
    if (R.bias_tokens) {
        q.bias_lo = max((int64_t)0, R.bias_offsets[row]);
        q.bias_hi = max(q.bias_lo, min(R.n_bias, R.bias_offsets[row + 1]));
    }
    q.mask = nullptr;
    if (R.allow) {
        const int64_t a = R.allow_row ? (int64_t)R.allow_row[row] : row;
        if (a >= 0 && a < R.n_allow) q.mask = reinterpret_cast<const uint32_t *>(R.allow) + a * R.allow_ld;
    }
    return q;
}

// Bits of the N tokens from v on that the grammar denies (those outside the vocabulary are arbitrary).
template <int N> __device__ __forceinline__ uint32_t denied(const uint32_t *words, int n_words, int v)
{
    const int i = v >> 5, sh = v & 31;
    const uint32_t lo = (i >= 0 && i < n_words) ? __ldg(words + i) : 0u;
    const uint32_t hi = (sh > 32 - N && i + 1 < n_words) ? __ldg(words + i + 1) : 0u;
    return ~__funnelshift_r(lo, hi, sh) & ((1u << N) - 1u);
}

__device__ __forceinline__ bool is_denied(const uint32_t *words, int v) { return words != nullptr && !(__ldg(words + (v >> 5)) >> (v & 31) & 1u); }

// The tokens of a row's history that fall into a range of `width` tokens from v0 on: a bit per token, and a table of the
// occurrences in the generated part.  Three forms of the table:
//   kCount16  16 bits per token, for generated parts below 2^16 tokens;
//   kCount32  32 bits per token;
//   kBiased   two words per token, kSeen and the occurrences, and the number of the last entry of the bias list that names it, for
//             lists of more than kBiasCap entries.  Shorter ones are kept beside the table: bias_v[k] is the token of entry k if it is in
//             the range (else -1), and `biased` has its bit.
// A bit per token says that its place is not zero, and those places are listed as far as the list reaches.  A whole history goes in by
// atomics without a result (counts and bits; nothing waits for them), and the list is made from the bits; fresh
// tokens of a following row are appended.  (Lists made by atomics that return the count before cost a round trip to shared memory
// per token, and their order, which sums would depend on, is not the same in every call.)
enum { kCount16 = 0, kCount32 = 1, kBiased = 2 };
constexpr int kBiasCap = 512;
constexpr int kSlack = 16;    // a range of positions [a, e) covers tokens from a - 15 on, depending on the row's alignment
constexpr int kBlockRows = 8; // rows of a block at most

__host__ __device__ constexpr int table_words(int form, int width) { return form == kCount16 ? (width + 1) >> 1 : form == kCount32 ? width : 2 * width; }

// A row of a CTA's block: its rules, and how to get from the table of the row before to this one's.
struct RowPlan {
    RowRules q;
    int form, n_bias;         // n_bias: entries of a short list
    bool used;                // the row is worked on: one that ends before the CTA's range, which its alignment decides, is not
    bool follows;             // its history is that of the last row with a table and the `fresh` tokens from `from` on
    int fresh, fresh_prompt;  // ... of which the first fresh_prompt are prompt
    const int32_t *from;
    int first[4];             // the first four of them
};

// Plans of a block's rows, one thread each.  `used` is set.  Ends with the CTA synchronised.
__device__ __forceinline__ void plan_rows(RowPlan *plan, int rows, const hilore_logit_rules &R)
{
    const int i = threadIdx.x;
    if (i < rows) {
        RowPlan &p = plan[i];
        const int64_t list = p.q.bias_hi - p.q.bias_lo;
        p.n_bias = list <= kBiasCap ? (int)list : 0;
        p.form = list > kBiasCap ? kBiased : p.q.hist_hi - p.q.hist_mid < (1 << 16) ? kCount16 : kCount32;
    }
    __syncthreads();
    if (i < rows) {
        RowPlan &p = plan[i];
        p.follows = false;
        p.fresh = p.fresh_prompt = 0;
        p.from = R.tokens;
        int j = -1; // the last row before this one that leaves a table
        for (int k = 0; k < i; ++k)
            if (plan[k].used && (plan[k].q.history() || plan[k].form == kBiased)) j = k;
        if (j >= 0 && p.q.history() && p.form != kBiased && plan[j].form == p.form) {
            const RowRules &a = plan[j].q, &b = p.q;
            // the same tokens of the common part are prompt, and few enough come after it
            p.follows = a.hist_lo == b.hist_lo && a.hist_hi <= b.hist_hi && a.hist_mid == min(b.hist_mid, a.hist_hi) && b.hist_hi - a.hist_hi < (1 << 20);
            if (p.follows) {
                p.from = R.tokens + a.hist_hi;
                p.fresh = (int)(b.hist_hi - a.hist_hi);
                p.fresh_prompt = (int)max((int64_t)0, b.hist_mid - a.hist_hi);
                for (int k = 0; k < 4; ++k)
                    p.first[k] = k < p.fresh ? __ldg(p.from + k) : -1;
            }
        }
    }
    __syncthreads();
}

// Layout in shared memory: biased [BITS] (bit v - v0: a short bias list names the token), touch [BITS] (bit v - v0: the place is
// listed), bias_v and bias_x [kBiasCap] (token and value of the entries of a short bias list), then the table.
template <int BITS> struct Listed {
    static constexpr int kFixed = BITS * 8 + kBiasCap * 8; // bytes before the table
    static_assert(BITS % 4 == 0, "16-byte pieces");
    unsigned char *base;
    int *n;         // places listed; above the capacity of the list it is not complete
    uint32_t *doubles; // 1: a token is named twice by the short bias list
    uint32_t *sums; // one word per warp

    __device__ __forceinline__ uint32_t *biased() const { return reinterpret_cast<uint32_t *>(base); }
    __device__ __forceinline__ uint32_t *touch() const { return reinterpret_cast<uint32_t *>(base + BITS * 4); }
    __device__ __forceinline__ int *bias_v() const { return reinterpret_cast<int *>(base + BITS * 8); }
    __device__ __forceinline__ float *bias_x() const { return reinterpret_cast<float *>(base + BITS * 8 + kBiasCap * 4); }
    __device__ __forceinline__ uint32_t *word() const { return reinterpret_cast<uint32_t *>(base + kFixed); }
    // Occurrences in the generated part with kSeen if there are any at all: of a listed place, and of any place.
    __device__ __forceinline__ uint32_t count_at(int s, int form) const
    {
        if (form == kBiased) return word()[2 * s];
        return kSeen | (form == kCount32 ? word()[s] : word()[s >> 1] >> (16 * (s & 1)) & 0xFFFFu);
    }
    __device__ __forceinline__ uint32_t count_of(int s, int form) const { return touch()[s >> 5] >> (s & 31) & 1u ? count_at(s, form) : 0u; }
    __device__ __forceinline__ bool is_biased(int s) const { return biased()[s >> 5] >> (s & 31) & 1u; }
    __device__ __forceinline__ void count(int s, bool prompt, int form) const
    {
        const int odd = form == kCount16 ? s & 1 : 0;
        uint32_t *w = word() + (form == kCount16 ? s >> 1 : form == kBiased ? 2 * s : s);
        if (!prompt) atomicAdd(w, 1u << (16 * odd));
        if (form == kBiased) atomicOr(w, kSeen);
    }

    // Brings table and bias entries to the row's rules for tokens [v0, v0 + width).  `follow`: by adding the plan's fresh tokens to the
    // table of the row before; `sorted`: the list has to be as it would be made from the bits after that as well, so that sums over it
    // do not depend on where the row's block began.  Ends with the CTA synchronised.
    template <int THREADS>
    __device__ __forceinline__ void fill(const hilore_logit_rules &R, const RowPlan &p, int V, int v0, int width, int form, bool follow, bool sorted,
                                         uint16_t *list, int cap) const
    {
        const int tid = threadIdx.x, bits = ((width + 127) >> 7) * 4;
        const bool counts = p.q.history() || form == kBiased, clear = counts && !follow;
        const int low = max(v0, 0);
        const uint32_t span = (uint32_t)max(min(v0 + width, V) - low, 0); // tokens [low, low + span)
        int before = 0;
        if (clear || p.n_bias > 0) {
            __syncthreads(); // the row before is done with both
            if (clear) {
                const int quads = (table_words(form, width) + 3) >> 2;
                for (int i = tid; i < quads; i += THREADS)
                    reinterpret_cast<uint4 *>(word())[i] = make_uint4(0, 0, 0, 0);
                for (int i = tid; i < bits / 4; i += THREADS)
                    reinterpret_cast<uint4 *>(touch())[i] = make_uint4(0, 0, 0, 0);
            }
            if (p.n_bias > 0)
                for (int i = tid; i < bits / 4; i += THREADS)
                    reinterpret_cast<uint4 *>(biased())[i] = make_uint4(0, 0, 0, 0);
            if (tid == 0) *doubles = 0;
            __syncthreads();
            for (int64_t i = p.q.bias_lo + tid; i < p.q.bias_hi; i += THREADS) {
                const int v = __ldg(R.bias_tokens + i), k = (int)(i - p.q.bias_lo);
                const int s = v - v0;
                const bool in = (uint32_t)(v - low) < span;
                if (form != kBiased) {
                    bias_v()[k] = in ? v : -1;
                    bias_x()[k] = __ldg(R.bias_values + i);
                    if (in && (atomicOr(biased() + (s >> 5), 1u << (s & 31)) >> (s & 31) & 1u)) atomicOr(doubles, 1u);
                } else if (in) {
                    atomicMax(word() + 2 * s + 1, (uint32_t)k + 1u);
                    atomicOr(touch() + (s >> 5), 1u << (s & 31));
                }
            }
        }
        if (follow) {
            if (sorted) {
                before = *n;
                __syncthreads();
            }
            for (int i = tid; i < p.fresh; i += THREADS) {
                const int v = i < 4 ? p.first[i] : __ldg(p.from + i), s = v - v0;
                if ((uint32_t)(v - low) >= span)
                    continue;
                const uint32_t bit = 1u << (s & 31);
                count(s, i < p.fresh_prompt, form);
                if (!(atomicOr(touch() + (s >> 5), bit) & bit)) {
                    const int at = atomicAdd(n, 1);
                    if (at < cap) list[at] = (uint16_t)s;
                }
            }
        } else if (p.q.history()) {
            constexpr int U = 8; // tokens in flight per thread
            const int32_t *from = R.tokens + p.q.hist_lo;
            int64_t left = p.q.hist_hi - p.q.hist_lo, prompt = p.q.hist_mid - p.q.hist_lo;
            for (; left > 0; left -= THREADS * U, prompt -= THREADS * U, from += THREADS * U) {
                const int here = (int)min(left, (int64_t)(THREADS * U)), first = (int)max((int64_t)0, min(prompt, (int64_t)(THREADS * U)));
                int v[U];
#pragma unroll
                for (int u = 0; u < U; ++u)
                    v[u] = u * THREADS + tid < here ? __ldg(from + u * THREADS + tid) : -1;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if ((uint32_t)(v[u] - low) < span) {
                        const int s = v[u] - v0;
                        atomicOr(touch() + (s >> 5), 1u << (s & 31));
                        count(s, u * THREADS + tid < first, form);
                    }
                }
            }
        }
        __syncthreads();
        if (clear || (follow && sorted && *n > before && *n <= cap)) order<THREADS>(bits, list, cap);
    }

    // Makes the list from the touch bits: a thread's words lie apart, as frequent tokens are neighbours.  Ends with the CTA synchronised.
    template <int THREADS> __device__ __forceinline__ void order(int bits, uint16_t *list, int cap) const
    {
        constexpr int W = (BITS + THREADS - 1) / THREADS;
        const int tid = threadIdx.x, lane = tid & 31;
        uint32_t w[W];
        int own = 0;
#pragma unroll
        for (int j = 0; j < W; ++j) {
            w[j] = tid + j * THREADS < bits ? touch()[tid + j * THREADS] : 0u;
            own += __popc(w[j]);
        }
        int at = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int below = __shfl_up_sync(0xFFFFFFFFu, at, o);
            if (lane >= o) at += below;
        }
        if (lane == 31) sums[tid >> 5] = (uint32_t)at;
        __syncthreads();
        at -= own;
        for (int k = 0; k < (tid >> 5); ++k)
            at += (int)sums[k];
        if (tid == THREADS - 1) *n = at + own;
#pragma unroll
        for (int j = 0; j < W; ++j)
            for (; w[j]; w[j] &= w[j] - 1, ++at)
                if (at < cap) list[at] = (uint16_t)((tid + j * THREADS) * 32 + __ffs((int)w[j]) - 1);
        __syncthreads();
    }

    // For every listed place: v = load(place), then use(place, v).  From the list where it is complete (a thread per entry),
    // otherwise from the bits (a thread per place).  Either way a place goes to the same thread in every call.  (Four or eight loads of a
    // thread in flight were slower: the copies of `use` cost the stream more than the waits.)
    template <int THREADS, typename Load, typename Use>
    __device__ __forceinline__ void each(int n_listed, int width, const uint16_t *list, int cap, const Load &load, const Use &use) const
    {
        const bool whole = n_listed <= cap;
        const int items = whole ? n_listed : (width + 31) & ~31;
#pragma unroll 1
        for (int i = threadIdx.x; i < items; i += THREADS) {
            const int p = whole ? list[i] : i;
            if (whole || (touch()[i >> 5] >> (i & 31) & 1u)) use(p, load(p));
        }
    }

    // Whether entry k of a short bias list is the last one that names its token (which bias_v has).
    __device__ __forceinline__ bool counts_as_bias(int k, int n_bias) const
    {
        const int v = bias_v()[k];
        if (v < 0)
            return false;
        if (*doubles == 0)
            return true;
        for (int j = k + 1; j < n_bias; ++j)
            if (bias_v()[j] == v)
                return false;
        return true;
    }
};

// The logit of a listed token under the penalties and its bias, before the temperature.
__device__ __forceinline__ float adjusted(float x, uint32_t count, float bias, const RowRules &q)
{
    if (count) {
        x = x > 0.0f ? x * q.inv_rep : x * q.rep;
        const uint32_t c = count & ~kSeen;
        if (c) x = x - fmaf(q.freq, (float)c, q.pres);
    }
    return x + bias;
}

// Value of entry `number` - 1 of the row's bias list; 0 for number 0.
__device__ __forceinline__ float bias_value(const hilore_logit_rules &R, const RowRules &q, uint32_t number)
{
    return number == 0u ? 0.0f : __ldg(R.bias_values + (q.bias_lo + (int64_t)number - 1));
}

// d(adjusted logit) / d(logit) of a listed token.
__device__ __forceinline__ float slope_of(float x, uint32_t count, const RowRules &q)
{
    return count ? (x > 0.0f ? q.inv_rep : q.rep) : 1.0f;
}

// ------------------------------------------------------------------------------------------ element-wise results of a row
// What all three element-wise calls share: out[v] = plain(in[v]) for every token, listed(...) for the listed ones, `off` where
// the grammar denies.  One CTA per (row, range of `width` positions).

struct MapApply { // z from x
    static constexpr bool kGrad = false;
    float inv_temp;
    static constexpr int target = -1;
    __device__ __forceinline__ float one(float in, bool) const { return in * inv_temp; }
    __device__ __forceinline__ float listed(float in, float, int, uint32_t c, float b, const RowRules &q) const
    {
        return adjusted(in, c, b, q) * inv_temp;
    }
    static __device__ __forceinline__ float off() { return -INFINITY; }
};

struct MapApplyGrad { // dx from dz; x is read at listed tokens only (the side of zero they are on)
    static constexpr bool kGrad = true;
    float inv_temp;
    static constexpr int target = -1;
    __device__ __forceinline__ float one(float in, bool) const { return in * inv_temp; }
    __device__ __forceinline__ float listed(float in, float x, int, uint32_t c, float, const RowRules &q) const
    {
        return in * slope_of(x, c, q) * inv_temp;
    }
    static __device__ __forceinline__ float off() { return 0.0f; }
};

struct MapLogpGrad { // omega (1[v = a] - exp(z - lse)) dz/dx from x
    static constexpr bool kGrad = false;
    float inv_temp, lse, scale; // scale = omega / temperature
    int target;                 // position of the target
    __device__ __forceinline__ float one(float z, bool hit) const
    {
        const float p = ex2_ftz(fmaf(z, inv_temp, -lse) * kLog2eF);
        return (hit ? 1.0f - p : -p) * scale;
    }
    __device__ __forceinline__ float listed(float in, float, int f, uint32_t c, float b, const RowRules &q) const
    {
        return one(adjusted(in, c, b, q), f == target) * slope_of(in, c, q);
    }
    static __device__ __forceinline__ float off() { return 0.0f; }
};

// Shapes of a CTA of THREADS threads.  A stage is 32 logits of every thread, in flight together.  Shared memory where tokens may be listed:
// bits, bias entries, and a pool for the table, the list and -- where the output is the input and everything has to be read before
// anything is stored -- the results of the listed tokens.  In that case a range is worked on as a whole where the row's lists cannot
// outgrow what the pool leaves beside the table, otherwise in parts whose every token may be listed.
//   hilore_logits_apply: 512 threads, two CTAs per SM (96 rows of 151936 fp32 logits, histories of up to 16384: with 256 threads, three
//   CTAs per SM, it took 70 us where this took 60; it takes 55 now).  The gradient of a log-probability holds more in registers: 256 (1500 x 32063 bf16
//   rows under prefixes 69 us; 94 with 512, 74 with 128, whose 12000 rows take 403 us for 416).
template <int THREADS> struct MapShape {
    static constexpr int kStage = THREADS * 32;
    static constexpr int kRange = THREADS == 512 ? 2 * kStage : 3 * kStage; // positions of a CTA's range at most: a table of 16-bit counts
    static constexpr int kBits = (kRange + kSlack + 127) / 128 * 4;
    static constexpr int kPool = THREADS == 512 ? 40 * 512 : 31 * 512; // words
    static constexpr int kCtas = THREADS == 512 ? 2 : 3;               // per SM
    using Table = Listed<kBits>;
    static constexpr size_t kShared = Table::kFixed + kPool * 4;
    static __host__ __device__ constexpr int words(int form, int step) { return (table_words(form, step + kSlack) + 3) & ~3; }
    static __host__ __device__ constexpr int capacity(int form, int step) { return (kPool - words(form, step)) * 4 / 6 & ~1; } // list and results
    static __host__ __device__ constexpr int most(int form) { return form == kCount16 ? kRange : form == kCount32 ? kRange / 2 : kRange / 4; }
    static __host__ __device__ constexpr int dense(int form) { return form == kCount16 ? 6144 : form == kCount32 ? 4864 : 3712; } // every token may be listed
    static_assert(words(kCount16, most(kCount16)) <= kPool && words(kCount32, most(kCount32)) <= kPool && words(kBiased, most(kBiased)) <= kPool, "tables fit");
};
static_assert(MapShape<256>::capacity(kCount16, MapShape<256>::dense(kCount16)) >= MapShape<256>::dense(kCount16) + kSlack + kBiasCap &&
                  MapShape<256>::capacity(kCount32, MapShape<256>::dense(kCount32)) >= MapShape<256>::dense(kCount32) + kSlack + kBiasCap &&
                  MapShape<256>::capacity(kBiased, MapShape<256>::dense(kBiased)) >= MapShape<256>::dense(kBiased) + kSlack,
              "lists of dense parts fit");
constexpr int kApplyThreads = 512, kGradThreads = 256;

// Positions [a, b) of a row as if no token were listed.
template <int THREADS, typename T, bool SHIFTED, typename Map>
__device__ __forceinline__ void map_vectors(const Row<T> &dst, const Source<T> &src, const Map &map, const uint32_t *mask, int n_words, int fa, int fb)
{
    constexpr int N = Lane<T>::N, U = 32 / N;
    constexpr uint32_t kAll = (1u << N) - 1u;
#pragma unroll 1
    for (int f0 = fa + (int)threadIdx.x * N; f0 < fb; f0 += THREADS * 32) {
        uint32_t w[U][8], deny[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int f = f0 + u * THREADS * N;
            deny[u] = f < fb && mask ? denied<N>(mask, n_words, f - dst.lead) : 0u;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int f = f0 + u * THREADS * N;
            if (f < fb && deny[u] != kAll) src.template load<SHIFTED>(f, w[u]); // a vector without an allowed token is not read
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int f = f0 + u * THREADS * N;
            if (f >= fb)
                break;
            float z[N];
            Lane<T>::unpack(w[u], z);
            const int at = map.target - f; // the target's place in this vector, if it is in it
#pragma unroll
            for (int i = 0; i < N; ++i)
                z[i] = map.one(z[i], i == at);
            if (deny[u]) {
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (deny[u] >> i & 1u) z[i] = Map::off();
            }
            dst.store(f, z);
        }
    }
}

template <int THREADS, typename T, typename Map>
__device__ __forceinline__ void map_plain(const Row<T> &dst, const T *in, const Map &map, const uint32_t *mask, int V, int a, int b)
{
    const Source<T> src(in, V, dst);
    const typename Row<T>::Parts p = src.parts(dst, a, b);
    const int n_words = (V + 31) >> 5;
    if (src.shift == 0) map_vectors<THREADS, T, false>(dst, src, map, mask, n_words, p.fa, p.fb);
    else map_vectors<THREADS, T, true>(dst, src, map, mask, n_words, p.fa, p.fb);
    each_edge<THREADS>(p, [&](int f) {
        const int v = f - dst.lead;
        Lane<T>::put(dst.origin + f, is_denied(mask, v) ? Map::off() : map.one(Lane<T>::one(in + v), f == map.target));
    });
}

// What the result of a listed token is made from; `ours`: it is this range's and allowed (otherwise the stream's result stays).
struct Pick {
    float in, x;
    bool ours;
};
template <bool GRAD, typename T> __device__ __forceinline__ Pick pick(const T *in, const T *x, const uint32_t *mask, int v, int lead, int a, int e)
{
    Pick k{0.0f, 0.0f, v + lead >= a && v + lead < e};
    if (k.ours) {
        k.in = Lane<T>::one(in + v);
        if (GRAD) k.x = Lane<T>::one(x + v);
        k.ours = !is_denied(mask, v);
    }
    return k;
}

// Asks L2 for positions [a, b) of the row that `row` points to, as far as whole 16-byte pieces of them go.
template <typename T> __device__ __forceinline__ void prefetch_range(const T *row, int V, int a, int b)
{
    const Row<T> own(row, V);
    const int lo = max(a, own.lead), hi = min(b, own.end);
    if (hi <= lo)
        return;
    const uintptr_t first = (reinterpret_cast<uintptr_t>(own.origin + lo) + 15) & ~(uintptr_t)15, last = reinterpret_cast<uintptr_t>(own.origin + hi) & ~(uintptr_t)15;
    if (last > first) prefetch_l2_bulk(reinterpret_cast<const void *>(first), (uint32_t)(last - first));
}

// Positions [a, b) of a row that may have listed tokens.  `in_place`: the output is the input.
template <int THREADS, typename T, typename Map>
__device__ __forceinline__ void map_listed(const Row<T> &dst, const T *in, const T *x, const Map &map, const RowPlan &plan, const hilore_logit_rules &R,
                                           int V, int a, int b, int range, bool in_place, const typename MapShape<THREADS>::Table &t, bool &intact)
{
    using Shape = MapShape<THREADS>;
    const RowRules &q = plan.q;
    const int tid = threadIdx.x, n_bias = plan.n_bias, form = plan.form, lead = dst.lead;
    const bool counts = q.history() || form == kBiased;
    const int64_t most = q.hist_hi - q.hist_lo + q.bias_hi - q.bias_lo; // different tokens of the row at most
    int step = min(range, Shape::most(form));
    if (in_place && most > Shape::capacity(form, step)) step = min(step, Shape::dense(form));
    const int cap = in_place ? Shape::capacity(form, step) : (Shape::kPool - Shape::words(form, step)) * 2; // without results the list has it all
    uint16_t *list = reinterpret_cast<uint16_t *>(t.word() + Shape::words(form, step));
    uint32_t *result = t.word() + Shape::words(form, step) + cap / 2;
    T *row = dst.origin + lead;
    for (; a < b; a += step) {
        const int e = min(b, a + step), v0 = a - kSlack, width = step + kSlack;
        if (q.listed()) t.template fill<THREADS>(R, plan, V, v0, width, form, plan.follows && intact && step == range, false, list, cap);
        const int n = counts ? *t.n : 0;
        const auto load = [&](int p) { return pick<Map::kGrad>(in, x, q.mask, v0 + p, lead, a, e); };
        const auto of_history = [&](int p, const Pick &k) {
            const float bias = form == kBiased ? bias_value(R, q, t.word()[2 * p + 1]) : 0.0f;
            return map.listed(k.in, k.x, v0 + p + lead, t.count_at(p, form), bias, q);
        };
        const auto of_bias = [&](int j, const Pick &k) {
            const int v = t.bias_v()[j];
            return map.listed(k.in, k.x, v + lead, counts ? t.count_of(v - v0, form) : 0u, t.bias_x()[j], q);
        };
        if (in_place) { // n entries and then those of the bias list: both fit, as `most` of them do
            for (int i = tid; i < n; i += THREADS) {
                const int p = list[i];
                const Pick k = load(p);
                const bool any = k.ours && !(n_bias > 0 && t.is_biased(p));
                if (any) result[i] = __float_as_uint(of_history(p, k));
                else list[i] = 0xFFFFu;
            }
            for (int j = tid; j < n_bias; j += THREADS) {
                const bool last = t.counts_as_bias(j, n_bias);
                const Pick k = last ? load(t.bias_v()[j] - v0) : Pick{0.0f, 0.0f, false};
                if (k.ours) result[n + j] = __float_as_uint(of_bias(j, k));
                list[n + j] = k.ours ? 0u : 0xFFFFu;
            }
            __syncthreads();
        } else if (Map::kGrad && n <= cap) {
            for (int i = tid; i < n; i += THREADS)
                prefetch_l2(x + max(v0 + (int)list[i], 0));
        }
        map_plain<THREADS>(dst, in, map, q.mask, V, a, e);
        if (!q.listed())
            continue;
        __syncthreads(); // the stream's results of listed tokens are there to be written over
        if (in_place) {
            for (int i = tid; i < n + n_bias; i += THREADS)
                if (list[i] != 0xFFFFu) Lane<T>::put(row + (i < n ? v0 + (int)list[i] : t.bias_v()[i - n]), __uint_as_float(result[i]));
            if (counts) intact = false; // its list has gaps
        } else {
            t.template each<THREADS>(n, width, list, cap, load, [&](int p, const Pick &k) {
                if (k.ours && !(n_bias > 0 && t.is_biased(p))) Lane<T>::put(row + (v0 + p), of_history(p, k));
            });
            for (int j = tid; j < n_bias; j += THREADS)
                if (t.counts_as_bias(j, n_bias)) {
                    const Pick k = load(t.bias_v()[j] - v0);
                    if (k.ours) Lane<T>::put(row + t.bias_v()[j], of_bias(j, k));
                }
            if (counts) intact = step == range && form != kBiased; // the table holds the last row with one, over the whole range
        }
        __syncthreads(); // the table may be changed
    }
}

// What a CTA keeps of the rows of its block.
struct RowLoss { // of the gradient of a log-probability
    int target;
    float omega, lse;
    bool live;
};

// One CTA per (block of rows, range).  2048 x 128256 bf16 rows of a gradient under prefixes: 248 us, 205 with an empty history (the
// bytes 163); 96 rows of 151936 fp32 logits with masks on half: 55 us with histories of up to 16384 tokens, 42 up to 4096, 39 up to 1024, 35
// without, 27 without lists (the bytes 19).  In place 124, 43, 39: lists of a long history go in parts, each with a scan of its own.  LISTS: rows may have listed tokens; otherwise a block is one row.
template <int THREADS, typename T, bool GRAD, bool LISTS>
__global__ void __launch_bounds__(THREADS, LISTS ? MapShape<THREADS>::kCtas : sizeof(T) == 2 ? 1024 / THREADS : 768 / THREADS)
    logits_apply_kernel(const T *x, int64_t ld, const T *in, int64_t ld_in, T *out, int64_t ld_out, int64_t n_rows, int V, int block_rows, int n_ranges,
                        int width, const __grid_constant__ hilore_logit_rules R)
{
    const int64_t row0 = (int64_t)(blockIdx.x / n_ranges) * block_rows;
    const int a = (int)(blockIdx.x % n_ranges) * width;
    if (!LISTS) {
        const RowRules q = row_rules(R, row0);
        const Row<T> dst(out + row0 * ld_out, V);
        if (a >= dst.end)
            return;
        if (GRAD) map_plain<THREADS>(dst, in + row0 * ld_in, MapApplyGrad{q.inv_temp}, q.mask, V, a, min(dst.end, a + width));
        else map_plain<THREADS>(dst, in + row0 * ld_in, MapApply{q.inv_temp}, q.mask, V, a, min(dst.end, a + width));
        return;
    }
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ RowPlan plan[kBlockRows];
    __shared__ uint32_t sums[THREADS / 32];
    __shared__ int count;
    __shared__ uint32_t doubles;
    const int rows = (int)min((int64_t)block_rows, n_rows - row0);
    if ((int)threadIdx.x < rows) {
        plan[threadIdx.x].q = row_rules(R, row0 + threadIdx.x);
        plan[threadIdx.x].used = a < Row<T>(out + (row0 + threadIdx.x) * ld_out, V).end;
    }
    plan_rows(plan, rows, R);
    const typename MapShape<THREADS>::Table t{smem, &count, &doubles, sums};
    bool intact = false;
    for (int i = 0; i < rows; ++i) {
        const RowRules &q = plan[i].q;
        const Row<T> dst(out + (row0 + i) * ld_out, V);
        const T *from = in + (row0 + i) * ld_in, *at = x + (row0 + i) * ld;
        const int b = min(dst.end, a + width);
        if (threadIdx.x == 0) { // the next row's input while this one is worked on (of a masked row, only what is allowed is read)
            if (i == 0 && q.mask == nullptr) prefetch_range(from, V, a, a + width);
            if (i + 1 < rows && plan[i + 1].q.mask == nullptr) prefetch_range(from + ld_in, V, a, a + width);
        }
        if (a >= b)
            continue;
        if (GRAD) map_listed<THREADS>(dst, from, at, MapApplyGrad{q.inv_temp}, plan[i], R, V, a, b, width, in == out, t, intact);
        else map_listed<THREADS>(dst, from, at, MapApply{q.inv_temp}, plan[i], R, V, a, b, width, in == out, t, intact);
    }
}

// The same for the gradient of a log-probability (three quarters of 4096 rows of 151936 bf16 logits 336 us, 6.5 TB/s, zeros of the others
// included; 1500 x 32063 under prefixes of up to 1200 tokens 69 us, 35 without rules).  Rows whose coefficient is zero, that have no token, whose token the grammar
// denies or that had nothing to choose from get zeros without being read.
__device__ __forceinline__ RowLoss row_loss(const RowRules &q, const int32_t *targets, const float *lse, const float *omega, int64_t row, int V)
{
    RowLoss p{targets[row], omega[row], lse[row], false};
    p.live = (uint32_t)p.target < (uint32_t)V && p.omega != 0.0f && !(p.lse <= kNothing) && !is_denied(q.mask, p.target);
    return p;
}

template <int THREADS, typename T> __device__ __forceinline__ void zero_range(const Row<T> &dst, int a, int b)
{
    const float zero[Lane<T>::N] = {};
    const typename Row<T>::Parts p = dst.parts(a, b);
#pragma unroll 4
    for (int f = p.fa + (int)threadIdx.x * Lane<T>::N; f < p.fb; f += THREADS * Lane<T>::N)
        dst.store(f, zero);
    each_edge<THREADS>(p, [&](int f) { Lane<T>::put(dst.origin + f, 0.0f); });
}

template <int THREADS, typename T, bool LISTS>
__global__ void __launch_bounds__(THREADS, LISTS ? MapShape<THREADS>::kCtas : sizeof(T) == 2 ? 1024 / THREADS : 768 / THREADS)
    token_logp_backward_kernel(const T *x, int64_t ld, int64_t n_rows, int V, int block_rows, int n_ranges, int width, const int32_t *targets,
                               const float *lse, const float *omega, T *grad, int64_t ld_grad, const __grid_constant__ hilore_logit_rules R)
{
    const int64_t row0 = (int64_t)(blockIdx.x / n_ranges) * block_rows;
    const int a = (int)(blockIdx.x % n_ranges) * width;
    if (!LISTS) {
        const RowRules q = row_rules(R, row0);
        const RowLoss p = row_loss(q, targets, lse, omega, row0, V);
        const Row<T> dst(grad + row0 * ld_grad, V);
        if (a >= dst.end)
            return;
        const int b = min(dst.end, a + width);
        if (p.live) map_plain<THREADS>(dst, x + row0 * ld, MapLogpGrad{softmax_factor(q.inv_temp), p.lse, p.omega * q.inv_temp, p.target + dst.lead}, q.mask, V, a, b);
        else zero_range<THREADS>(dst, a, b);
        return;
    }
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ RowPlan plan[kBlockRows];
    __shared__ RowLoss losses[kBlockRows];
    __shared__ uint32_t sums[THREADS / 32];
    __shared__ int count;
    __shared__ uint32_t doubles;
    const int rows = (int)min((int64_t)block_rows, n_rows - row0);
    if ((int)threadIdx.x < rows) {
        const RowRules q = row_rules(R, row0 + threadIdx.x);
        plan[threadIdx.x].q = q;
        losses[threadIdx.x] = row_loss(q, targets, lse, omega, row0 + threadIdx.x, V);
        plan[threadIdx.x].used = losses[threadIdx.x].live && a < Row<T>(grad + (row0 + threadIdx.x) * ld_grad, V).end;
    }
    plan_rows(plan, rows, R);
    const typename MapShape<THREADS>::Table t{smem, &count, &doubles, sums};
    bool intact = false;
    for (int i = 0; i < rows; ++i) {
        const RowRules &q = plan[i].q;
        const RowLoss p = losses[i];
        const Row<T> dst(grad + (row0 + i) * ld_grad, V);
        const T *from = x + (row0 + i) * ld;
        const int b = min(dst.end, a + width);
        if (threadIdx.x == 0) {
            if (i == 0 && p.live && q.mask == nullptr) prefetch_range(from, V, a, a + width);
            if (i + 1 < rows && losses[i + 1].live && plan[i + 1].q.mask == nullptr) prefetch_range(from + ld, V, a, a + width);
        }
        if (a >= b)
            continue;
        const MapLogpGrad map{softmax_factor(q.inv_temp), p.lse, p.omega * q.inv_temp, p.target + dst.lead};
        if (!p.live) zero_range<THREADS>(dst, a, b);
        else map_listed<THREADS>(dst, from, from, map, plan[i], R, V, a, b, width, x == grad, t, intact);
    }
}

// ---------------------------------------------------------------------------------------------- log-probability of a token
// Running statistics of a softmax in base 2: m the largest logit seen, s = sum 2^u, t = sum 2^u u with u = (z - m) c.
struct Soft {
    float m, s, t;
};

template <bool ENTROPY> __device__ __forceinline__ Soft soft_join(const Soft &a, const Soft &b, float c)
{
    Soft r;
    r.m = max_nan(a.m, b.m);
    const float da = fmaxf((a.m - r.m) * c, -256.0f), db = fmaxf((b.m - r.m) * c, -256.0f);
    const float ea = ex2_ftz(da), eb = ex2_ftz(db);
    r.s = a.s * ea + b.s * eb;
    r.t = ENTROPY ? ea * fmaf(da, a.s, a.t) + eb * fmaf(db, b.s, b.t) : 0.0f;
    return r;
}

// Adds N logits (already under the penalties and biases, -inf where denied) to the statistics.
template <int N, bool ENTROPY> __device__ __forceinline__ void soft_add(Soft &q, const float (&z)[N], float c)
{
    float m = z[0];
#pragma unroll
    for (int i = 1; i < N; ++i)
        m = max_nan(m, z[i]);
    m = max_nan(m, q.m);
    const float d = fmaxf((q.m - m) * c, -256.0f), e = ex2_ftz(d);
    if (ENTROPY) q.t = e * fmaf(d, q.s, q.t);
    q.s *= e;
    q.m = m;
    const uint64_t minus_m = f32x2_pack(-m, -m), cc = f32x2_pack(c, c);
    uint64_t sum = 0, mean = 0; // of pairs
#pragma unroll
    for (int i = 0; i < N; i += 2) {
        const uint64_t u = f32x2_mul(f32x2_add(f32x2_pack(z[i], z[i + 1]), minus_m), cc);
        float u0, u1;
        f32x2_unpack(u, u0, u1);
        if (ENTROPY) { // 2^-256 is zero in fp32: keeps -inf out of the product
            u0 = fmaxf(u0, -256.0f);
            u1 = fmaxf(u1, -256.0f);
        }
        const uint64_t e2 = f32x2_pack(ex2_ftz(u0), ex2_ftz(u1));
        sum = f32x2_add(sum, e2);
        if (ENTROPY) mean = f32x2_fma(e2, f32x2_pack(u0, u1), mean);
    }
    float lo, hi;
    f32x2_unpack(sum, lo, hi);
    q.s += lo + hi;
    if (ENTROPY) {
        f32x2_unpack(mean, lo, hi);
        q.t += lo + hi;
    }
}

// Adds one logit.
template <bool ENTROPY> __device__ __forceinline__ void soft_one(Soft &q, float z, float c)
{
    const float one[2] = {z, -INFINITY};
    soft_add<2, ENTROPY>(q, one, c);
}

constexpr int kLogpThreads = 256, kLogpWarps = kLogpThreads / 32, kMaxRowCtas = 8;

template <bool ENTROPY> __device__ __forceinline__ Soft warp_soft(Soft acc, float c)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        Soft other;
        other.m = __shfl_xor_sync(0xFFFFFFFFu, acc.m, o);
        other.s = __shfl_xor_sync(0xFFFFFFFFu, acc.s, o);
        other.t = ENTROPY ? __shfl_xor_sync(0xFFFFFFFFu, acc.t, o) : 0.0f;
        acc = soft_join<ENTROPY>(acc, other, c);
    }
    return acc;
}

// Results of a row from its statistics; z: the target's logit under penalties and bias, -inf where denied.
template <bool ENTROPY>
__device__ __forceinline__ void finish_row(const Soft &acc, float z, float inv_temp, int64_t row, float *logp, float *lse, float *entropy)
{
    const float ln_s = logf(acc.s);
    float l = fmaf(acc.m, inv_temp, ln_s), p = fmaf(z - acc.m, inv_temp, -ln_s), h = 0.0f;
    const bool nothing = acc.m == kLowest && acc.s == 0.0f;
    if (acc.m == INFINITY) { // the sum has no value (inf - inf); its logarithm has
        l = INFINITY;
        p = z - acc.m;
    } else if (nothing) {
        l = -INFINITY;
        p = -INFINITY;
    }
    if (ENTROPY) { // H = ln s - sum p u ln 2
        h = nothing ? 0.0f : fmaf(-acc.t / acc.s, 0.6931471805599453f, ln_s);
        if (acc.m != acc.m || acc.m == INFINITY) h = acc.m - acc.m;
        entropy[row] = h;
    }
    logp[row] = p;
    if (lse) lse[row] = l;
}

// Without rules beyond a temperature: one pass with the running maximum, sum and mean exponent of every thread, 32 logits in
// flight, exponentials in base 2 relative to the maximum, differences and sums in packed pairs (three quarters of 8192 rows of 151936 bf16 logits with
// entropy 298 us back to back, 6.3 TB/s, 364 among other work; the exponentials alone take 207 us of their units).  A row belongs to `row_ctas` CTAs (a thread-block cluster if more than one); each takes a
// share of its vectors.
template <typename T, bool ENTROPY>
__global__ void __launch_bounds__(kLogpThreads, 4)
    token_logp_kernel(const T *x, int64_t ld, int V, int row_ctas, const int32_t *targets, float *logp, float *lse, float *entropy,
                      const float *temperature)
{
    constexpr int N = Lane<T>::N, U = 32 / N;
    __shared__ Soft part[kLogpWarps];
    __shared__ Soft shares[kMaxRowCtas];
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x / row_ctas;
    const int rank = (int)(blockIdx.x - row * row_ctas);
    cg::cluster_group cl = cg::this_cluster();
    const int target = targets[row];
    if ((uint32_t)target >= (uint32_t)V) { // a slot without a token (the same for every CTA of the row)
        if (rank == 0 && tid == 0) {
            logp[row] = 0.0f;
            if (lse) lse[row] = 0.0f;
            if (ENTROPY) entropy[row] = 0.0f;
        }
        return;
    }
    if (row_ctas > 1) cl.barrier_arrive(); // once all have arrived, every CTA of the row runs
    const float inv_temp = softmax_factor(inverse_temperature(temperature, row)), c = kLog2eF * inv_temp;
    const Row<T> src(x + row * ld, V);
    const int n_vec = (src.end + N - 1) / N;
    const int a = (int)((int64_t)n_vec * rank / row_ctas) * N, b = (int)((int64_t)n_vec * (rank + 1) / row_ctas) * N;
    float z = 0.0f;
    if (rank == 0 && tid == 0) z = Lane<T>::one(x + row * ld + target);
    Soft acc{kLowest, 0.0f, 0.0f};
    const typename Row<T>::Parts p = src.parts(a, b);
    // L2 is asked for the next stage of bf16 logits, whose arithmetic takes long enough to wait for them (312 us without, 313 six stages ahead;
    // fp32 logits gain nothing from it).
    constexpr int kAhead = sizeof(T) == 2 ? kLogpThreads * 32 : 0;
    if (kAhead > 0 && tid == 0) prefetch_range(x + row * ld, V, a, min(b, a + kAhead));
    for (int f0 = p.fa + tid * N; f0 < p.fb; f0 += kLogpThreads * 32) {
        uint32_t w[U][8];
        if (kAhead > 0 && tid == 0 && f0 + kAhead < p.fb) prefetch_range(x + row * ld, V, f0 + kAhead, min(b, f0 + kAhead + kLogpThreads * 32));
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int f = f0 + u * kLogpThreads * N;
            if (f < p.fb) src.load(f, w[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int f = f0 + u * kLogpThreads * N;
            if (f < p.fb) {
                float v[N];
                Lane<T>::unpack(w[u], v);
                soft_add<N, ENTROPY>(acc, v, c);
            }
        }
    }
    each_edge<kLogpThreads>(p, [&](int f) { soft_one<ENTROPY>(acc, Lane<T>::one(src.origin + f), c); });
    acc = warp_soft<ENTROPY>(acc, c);
    if ((tid & 31) == 0) part[tid >> 5] = acc;
    __syncthreads();
    if (tid == 0)
        for (int w = 1; w < kLogpWarps; ++w)
            acc = soft_join<ENTROPY>(acc, part[w], c);
    if (row_ctas > 1) {
        cl.barrier_wait();
        if (tid == 0) *cl.map_shared_rank(&shares[rank], 0) = acc;
        cl.sync(); // the shares have arrived in the first CTA
    }
    if (rank != 0 || tid != 0)
        return;
    for (int r = 1; r < row_ctas; ++r)
        acc = soft_join<ENTROPY>(acc, shares[r], c);
    finish_row<ENTROPY>(acc, z, inv_temp, row, logp, lse, entropy);
}

// Under rules.  A cluster of `row_ctas` CTAs (or one CTA) walks a block of consecutive rows; each CTA owns `width` positions of
// every row, so that its table of counts serves one row after the other.  The statistics of every warp go to the first
// CTA, which joins them when the block is done.  Bound by the waits of a row's steps, not by bytes: 1021 rows of 50001 fp32 logits
// under prefixes of up to 900 tokens, 24 biases and masks on a third take 102 us (the bytes 29; 98 with a single fresh token left out of order), 60 without masks, biases and history.
constexpr int kLogpTokens = 32768; // tokens of a table of 16-bit counts at most: 8 CTAs take vocabularies up to 260000 in one part
constexpr int kLogpBits = kLogpTokens / 32 + 8, kLogpCap = 2048;
using LogpListed = Listed<kLogpBits>;
constexpr size_t kLogpFixed = LogpListed::kFixed; // bytes before the table; the list is in static shared memory

template <typename T, bool ENTROPY>
__global__ void __launch_bounds__(kLogpThreads, sizeof(T) == 4 ? 3 : 4)
    token_logp_rules_kernel(const T *x, int64_t ld, int64_t n_rows, int V, int block_rows, int row_ctas, int width, int words, const int32_t *targets,
                            float *logp, float *lse, float *entropy, const __grid_constant__ hilore_logit_rules R)
{
    constexpr int N = Lane<T>::N, U = 32 / N;
    constexpr uint32_t kAll = (1u << N) - 1u;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ RowPlan plan[kBlockRows];
    __shared__ int targets_of[kBlockRows];
    __shared__ int count;
    __shared__ uint32_t doubles;
    __shared__ uint16_t list[kLogpCap];
    __shared__ uint32_t sums[kLogpWarps];
    __shared__ Soft part[kBlockRows][kMaxRowCtas * kLogpWarps]; // in the first CTA: of all warps of the cluster
    __shared__ float target_z[kBlockRows];                      // in the first CTA: the targets' logits under penalties and bias
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int64_t row0 = (int64_t)(blockIdx.x / row_ctas) * block_rows;
    const int rank = (int)(blockIdx.x % row_ctas);
    const int rows = (int)min((int64_t)block_rows, n_rows - row0);
    cg::cluster_group cl = cg::this_cluster();
    if (row_ctas > 1) cl.barrier_arrive(); // once all have arrived, every CTA of the cluster runs
    if (tid < rows) {
        plan[tid].q = row_rules(R, row0 + tid);
        targets_of[tid] = targets[row0 + tid];
        plan[tid].used = (uint32_t)targets_of[tid] < (uint32_t)V;
    }
    plan_rows(plan, rows, R);
    if (row_ctas > 1) cl.barrier_wait();
    const LogpListed t{smem, &count, &doubles, sums};
    bool intact = false; // the table holds the last row with one, over the whole range
    Soft(*to_part)[kMaxRowCtas * kLogpWarps] = row_ctas > 1 ? cl.map_shared_rank(&part[0], 0) : &part[0];
    float *to_z = row_ctas > 1 ? cl.map_shared_rank(&target_z[0], 0) : &target_z[0];
    const int n_words = (V + 31) >> 5;
    for (int r = 0; r < rows; ++r) {
        const RowRules &q = plan[r].q;
        const int target = targets_of[r];
        if ((uint32_t)target >= (uint32_t)V)
            continue;
        const T *xrow = x + (row0 + r) * ld;
        const Row<T> src(xrow, V);
        const float c = kLog2eF * softmax_factor(q.inv_temp);
        const uint32_t *mask = q.mask;
        int a = rank * width;
        const int b = min(src.end, a + width);
        const int form = plan[r].form, n_bias = plan[r].n_bias;
        const bool lists = q.listed(), counts = q.history() || form == kBiased;
        const int room = (form == kCount16 ? 2 * words : form == kCount32 ? words : words / 2) - kSlack;
        const int step = lists && width > room ? room & ~127 : width;
        Soft acc{kLowest, 0.0f, 0.0f};
        for (; a < b; a += step) {
            const int e = min(b, a + step), v0 = a - kSlack, ft = target + src.lead;
            int n = 0;
            if (lists) {
                __syncthreads(); // the last range or row is done with the table
                const bool follow = plan[r].follows && intact && step == width;
                t.template fill<kLogpThreads>(R, plan[r], V, v0, step + kSlack, form, follow, true, list, kLogpCap);
                n = counts ? count : 0;
                if (counts) intact = step == width && form != kBiased;
            }
            const bool touched = counts, biased = n_bias > 0;
            const typename Row<T>::Parts parts = src.parts(a, e);
            for (int f0 = parts.fa + tid * N; f0 < parts.fb; f0 += kLogpThreads * 32) {
                uint32_t w[U][8], off[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int f = f0 + u * kLogpThreads * N;
                    off[u] = kAll;
                    if (f < parts.fb) {
                        const int p = f - src.lead - v0;
                        off[u] = mask ? denied<N>(mask, n_words, f - src.lead) : 0u;
                        if (touched) off[u] |= __funnelshift_r(t.touch()[p >> 5], t.touch()[(p >> 5) + 1], p & 31) & kAll;
                        if (biased) off[u] |= __funnelshift_r(t.biased()[p >> 5], t.biased()[(p >> 5) + 1], p & 31) & kAll;
                    }
                }
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (off[u] != kAll) src.load(f0 + u * kLogpThreads * N, w[u]); // a vector without an allowed token is not read
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (off[u] == kAll)
                        continue;
                    float z[N];
                    Lane<T>::unpack(w[u], z);
                    if (off[u]) {
#pragma unroll
                        for (int i = 0; i < N; ++i)
                            if (off[u] >> i & 1u) z[i] = -INFINITY;
                    }
                    soft_add<N, ENTROPY>(acc, z, c);
                }
            }
            each_edge<kLogpThreads>(parts, [&](int f) {
                const int p = f - src.lead - v0;
                if (is_denied(mask, f - src.lead) || (touched && (t.touch()[p >> 5] >> (p & 31) & 1u)) || (biased && t.is_biased(p)))
                    return;
                soft_one<ENTROPY>(acc, Lane<T>::one(src.origin + f), c);
            });
            // listed tokens after the stream: most of them are in L2 by now
            const auto load = [&](int p) { return pick<false>(xrow, xrow, mask, v0 + p, src.lead, a, e); };
            t.template each<kLogpThreads>(n, step + kSlack, list, kLogpCap, load, [&](int p, const Pick &k) {
                const int v = v0 + p;
                if (v + src.lead < a || v + src.lead >= e || (biased && t.is_biased(p)))
                    return;
                const float bias = form == kBiased ? bias_value(R, q, t.word()[2 * p + 1]) : 0.0f;
                const float z = k.ours ? adjusted(k.in, t.count_at(p, form), bias, q) : -INFINITY;
                if (v == target) to_z[r] = z;
                soft_one<ENTROPY>(acc, z, c);
            });
            for (int j = tid; j < n_bias; j += kLogpThreads)
                if (t.counts_as_bias(j, n_bias)) {
                    const int v = t.bias_v()[j];
                    if (v + src.lead < a || v + src.lead >= e)
                        continue;
                    const Pick k = load(v - v0);
                    const float z = k.ours ? adjusted(k.in, counts ? t.count_of(v - v0, form) : 0u, t.bias_x()[j], q) : -INFINITY;
                    if (v == target) to_z[r] = z;
                    soft_one<ENTROPY>(acc, z, c);
                }
            if (tid == 0 && ft >= a && ft < e) {
                const int p = target - v0;
                if (!(touched && (t.touch()[p >> 5] >> (p & 31) & 1u)) && !(biased && t.is_biased(p)))
                    to_z[r] = is_denied(mask, target) ? -INFINITY : Lane<T>::one(xrow + target);
            }
        }
        acc = warp_soft<ENTROPY>(acc, c);
        if (lane == 0) to_part[r][rank * kLogpWarps + warp] = acc;
    }
    if (row_ctas > 1) cl.sync(); // everything has arrived in the first CTA
    else __syncthreads();
    if (rank != 0)
        return;
    for (int r = warp; r < rows; r += kLogpWarps) {
        const int target = targets_of[r];
        const int64_t row = row0 + r;
        if ((uint32_t)target >= (uint32_t)V) { // a slot without a token
            if (lane == 0) {
                logp[row] = 0.0f;
                if (lse) lse[row] = 0.0f;
                if (ENTROPY) entropy[row] = 0.0f;
            }
            continue;
        }
        const float inv_temp = softmax_factor(plan[r].q.inv_temp), c = kLog2eF * inv_temp;
        Soft acc{kLowest, 0.0f, 0.0f};
        for (int k = lane; k < row_ctas * kLogpWarps; k += 32)
            acc = soft_join<ENTROPY>(acc, part[r][k], c);
        acc = warp_soft<ENTROPY>(acc, c);
        if (lane == 0) finish_row<ENTROPY>(acc, target_z[r], inv_temp, row, logp, lse, entropy);
    }
}

// ------------------------------------------------------------------------------------------------------------ host side
static int check_rules(const hilore_logit_rules *r, int64_t n_rows, int64_t V)
{
    if (r->n_tokens < 0 || r->n_bias < 0 || r->n_bias > 0x7FFFFFFE)
        return HILORE_INVALID_ARG;
    if (r->tokens ? !r->hist_begin || !r->resp_begin || !r->hist_end : r->n_tokens > 0)
        return HILORE_INVALID_ARG;
    if (r->bias_tokens ? !r->bias_values || !r->bias_offsets : r->n_bias > 0)
        return HILORE_INVALID_ARG;
    if (r->allow) {
        if (r->n_allow < 0 || (!r->allow_row && r->n_allow < n_rows))
            return HILORE_INVALID_ARG;
        if (r->allow_ld < (V + 31) / 32)
            return HILORE_SHAPE;
    }
    const void *four[] = {r->temperature, r->repetition, r->frequency, r->presence, r->tokens, r->bias_tokens, r->bias_values, r->allow, r->allow_row};
    const void *eight[] = {r->hist_begin, r->resp_begin, r->hist_end, r->bias_offsets};
    for (const void *p : four)
        if (!aligned(p, 4)) return HILORE_ALIGN;
    for (const void *p : eight)
        if (!aligned(p, 8)) return HILORE_ALIGN;
    return HILORE_OK;
}

// Arguments that all calls share; `rules` may be NULL where the call allows it.
static int check_rows(int32_t dtype, int64_t n_rows, int64_t V, int64_t ld)
{
    if ((dtype != HILORE_BF16 && dtype != HILORE_F32) || n_rows < 0 || V <= 0)
        return HILORE_INVALID_ARG;
    if (ld < V || V > 0x7FFF0000 || n_rows > 0x7FFF0000)
        return HILORE_SHAPE;
    return HILORE_OK;
}

static hilore_logit_rules used_rules(const hilore_logit_rules *r)
{
    hilore_logit_rules q{};
    if (r) q = *r;
    if (!q.repetition && !q.frequency && !q.presence) q.tokens = nullptr; // a history that nothing asks about is not read
    return q;
}

static bool more_than_temperature(const hilore_logit_rules &q) { return q.tokens || q.bias_tokens || q.allow; }

// More than 48 KB of shared memory, the kernels' own 12 KB at most included, needs an opt-in.  It is always one for `most`, the
// largest size that any call gives the kernel: the attribute belongs to the process, and a smaller one set by another thread
// between this call's opt-in and its launch would have the launch refused.
template <typename K> static bool allow_smem(K kernel, size_t bytes, size_t most)
{
    return bytes <= 32 * 1024 || cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most) == cudaSuccess;
}

static bool has_lists(const hilore_logit_rules &q) { return q.tokens || q.bias_tokens; }

// Work split.  A CTA takes a block of rows and a range of positions; its time is taken as proportional to
// rows * (positions + per-row overhead) + start, the start being the scan of a history, and the split is the one with the least number of
// rounds times that.  Overheads in positions, from fits to measured times.  The scan is charged once per block, as for the prefixes of
// one sequence; the caller knows the mean length only where rows share no tokens, and there every row is scanned, which makes blocks look
// cheaper than they are.
struct Split {
    int64_t block_rows, width, n_ranges, grid;
};
static Split best_split(int64_t n_rows, int64_t positions, int64_t slots, int max_block, int64_t max_width, int64_t min_width, int64_t per_row, int64_t start)
{
    Split best{1, max_width, 0, 0};
    double least = 1e300;
    const int64_t fewest = (positions + max_width - 1) / max_width, most = (positions + min_width - 1) / min_width;
    for (int64_t n = fewest; n <= most; n += n < 16 ? 1 : n / 8) {
        const int64_t width = ((positions + n - 1) / n + 127) / 128 * 128, ranges = (positions + width - 1) / width;
        for (int b = 1; b <= max_block && b <= n_rows; ++b) {
            const int64_t grid = (n_rows + b - 1) / b * ranges, rounds = (grid + slots - 1) / slots;
            // the last round's CTAs run among fewer others
            const double time = ((double)(rounds - 1) + 0.5 + 0.5 * (double)(grid - (rounds - 1) * slots) / (double)slots) * (double)(b * (width + per_row) + start);
            if (time < least) {
                least = time;
                best = Split{b, width, ranges, grid};
            }
        }
    }
    return best;
}

template <int THREADS> static Split map_split(int64_t n_rows, int64_t V, const hilore_logit_rules &R, bool lists)
{
    const int64_t sms = sm_count(), positions = V + 15;
    if (lists) {
        const int64_t history = R.n_tokens / n_rows;
        return best_split(n_rows, positions, MapShape<THREADS>::kCtas * sms, kBlockRows, MapShape<THREADS>::kRange, 2048, 8192, 8192 + (history < 65536 ? history : 65536));
    }
    Split p{1, 16384, 0, 0}; // one row, less of it while SMs are left without four CTAs
    const auto ranges = [&] { return (positions + p.width - 1) / p.width; };
    while (p.width > 2048 && n_rows * ranges() < 4 * sms)
        p.width /= 2;
    p.n_ranges = ranges();
    p.grid = n_rows * p.n_ranges;
    return p;
}

template <typename T, bool GRAD, bool LISTS>
static int launch_apply_as(const T *x, int64_t ld, const T *in, int64_t ld_in, T *out, int64_t ld_out, int64_t n_rows, int64_t V,
                           const hilore_logit_rules &R, cudaStream_t st)
{
    // Without listed tokens one CTA shape serves all.
    constexpr int THREADS = LISTS ? kApplyThreads : kGradThreads;
    const Split p = map_split<THREADS>(n_rows, V, R, LISTS);
    if (p.grid > 0x7FFFFFFF)
        return HILORE_SHAPE;
    auto kernel = logits_apply_kernel<THREADS, T, GRAD, LISTS>;
    const size_t smem = LISTS ? MapShape<THREADS>::kShared : 0;
    if (!allow_smem(kernel, smem, smem))
        return HILORE_CUDA;
    kernel<<<(unsigned)p.grid, THREADS, smem, st>>>(x, ld, in, ld_in, out, ld_out, n_rows, (int)V, (int)p.block_rows, (int)p.n_ranges, (int)p.width, R);
    return cudaGetLastError() == cudaSuccess ? HILORE_OK : HILORE_CUDA;
}

template <typename T, bool GRAD>
static int launch_apply(const T *x, int64_t ld, const T *in, int64_t ld_in, T *out, int64_t ld_out, int64_t n_rows, int64_t V,
                        const hilore_logit_rules &R, cudaStream_t st)
{
    return has_lists(R) ? launch_apply_as<T, GRAD, true>(x, ld, in, ld_in, out, ld_out, n_rows, V, R, st)
                        : launch_apply_as<T, GRAD, false>(x, ld, in, ld_in, out, ld_out, n_rows, V, R, st);
}

static bool clusters_on()
{
    const char *off = std::getenv("HILORE_DISABLE_CLUSTER_LAUNCH");
    return off == nullptr || off[0] == '\0' || (off[0] == '0' && off[1] == '\0');
}

// CTAs of a row: as many as keep the SMs busy with two each, at most a portable cluster, none with less than 2048 logits.
static int row_ctas_for(int64_t n_rows, int64_t V)
{
    int k = 1;
    if (clusters_on())
        while (k < kMaxRowCtas && n_rows * k < 2 * (int64_t)sm_count() && V / (2 * k) >= 2048)
            k *= 2;
    return k;
}

template <typename... KArgs, typename... Args>
static int launch_rows(void (*kernel)(KArgs...), int64_t grid, int cluster, size_t smem, cudaStream_t st, Args... args)
{
    if (grid > 0x7FFFFFFF)
        return HILORE_SHAPE;
    if (!allow_smem(kernel, smem, kLogpFixed + kLogpTokens * 2))
        return HILORE_CUDA;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(kLogpThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)cluster;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 1 : 0;
    if (cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...) != cudaSuccess)
        return HILORE_CUDA;
    return cudaGetLastError() == cudaSuccess ? HILORE_OK : HILORE_CUDA;
}

template <typename T, bool ENTROPY>
static int launch_logp(const T *x, int64_t ld, int64_t n_rows, int64_t V, const int32_t *targets, float *logp, float *lse, float *entropy,
                       const hilore_logit_rules &R, cudaStream_t st)
{
    int k = row_ctas_for(n_rows, V);
    if (!more_than_temperature(R))
        return launch_rows(token_logp_kernel<T, ENTROPY>, n_rows * k, k, 0, st, x, ld, (int)V, k, targets, logp, lse, entropy, R.temperature);
    // Enough CTAs for a row that a table of 16-bit counts takes a share of it.
    if (clusters_on() && has_lists(R))
        while (k < kMaxRowCtas && V / k > kLogpTokens - 256)
            k *= 2;
    const int64_t width = ((V + 15 + k - 1) / k + 127) / 128 * 128;
    int64_t words = (width + kSlack) / 2; // 16-bit counts; at least two words for 128 tokens and the slack, the narrowest part of a range
    words = words < 512 ? 512 : words > kLogpTokens / 2 ? kLogpTokens / 2 : (words + 3) & ~(int64_t)3;
    const int64_t block = has_lists(R) ? best_split(n_rows, width * k, 3 * (int64_t)sm_count(), kBlockRows, width, width, 8192, 8192).block_rows : 1;
    const int64_t grid = (n_rows + block - 1) / block * k;
    const size_t smem = has_lists(R) ? kLogpFixed + (size_t)words * 4 : 0;
    return launch_rows(token_logp_rules_kernel<T, ENTROPY>, grid, k, smem, st, x, ld, n_rows, (int)V, (int)block, k, (int)width, (int)words, targets, logp,
                       lse, entropy, R);
}

template <typename T, bool LISTS>
static int launch_logp_backward_as(const T *x, int64_t ld, int64_t n_rows, int64_t V, const int32_t *targets, const float *lse, const float *omega,
                                   T *grad, int64_t ld_grad, const hilore_logit_rules &R, cudaStream_t st)
{
    constexpr int THREADS = kGradThreads;
    const Split p = map_split<THREADS>(n_rows, V, R, LISTS);
    if (p.grid > 0x7FFFFFFF)
        return HILORE_SHAPE;
    auto kernel = token_logp_backward_kernel<THREADS, T, LISTS>;
    const size_t smem = LISTS ? MapShape<THREADS>::kShared : 0;
    if (!allow_smem(kernel, smem, smem))
        return HILORE_CUDA;
    kernel<<<(unsigned)p.grid, THREADS, smem, st>>>(x, ld, n_rows, (int)V, (int)p.block_rows, (int)p.n_ranges, (int)p.width, targets, lse, omega, grad,
                                                       ld_grad, R);
    return cudaGetLastError() == cudaSuccess ? HILORE_OK : HILORE_CUDA;
}

template <typename T>
static int launch_logp_backward(const T *x, int64_t ld, int64_t n_rows, int64_t V, const int32_t *targets, const float *lse, const float *omega,
                                T *grad, int64_t ld_grad, const hilore_logit_rules &R, cudaStream_t st)
{
    return has_lists(R) ? launch_logp_backward_as<T, true>(x, ld, n_rows, V, targets, lse, omega, grad, ld_grad, R, st)
                        : launch_logp_backward_as<T, false>(x, ld, n_rows, V, targets, lse, omega, grad, ld_grad, R, st);
}

} // namespace hilore

using namespace hilore;

extern "C" int hilore_logits_apply(const void *logits, int32_t dtype, int64_t n_rows, int64_t V, int64_t ld,
                                   const hilore_logit_rules *rules, void *out, int64_t ld_out, void *stream)
{
    if (!rules)
        return HILORE_INVALID_ARG;
    int bad = check_rows(dtype, n_rows, V, ld);
    if (!bad) bad = check_rules(rules, n_rows, V);
    if (bad)
        return bad;
    if (ld_out < V)
        return HILORE_SHAPE;
    if (n_rows == 0)
        return HILORE_OK;
    if (!logits || !out)
        return HILORE_INVALID_ARG;
    const size_t es = dtype == HILORE_BF16 ? 2 : 4;
    if (!aligned(logits, es) || !aligned(out, es))
        return HILORE_ALIGN;
    if (out == logits && ld_out != ld && n_rows > 1)
        return HILORE_SHAPE;
    const hilore_logit_rules R = used_rules(rules);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dtype == HILORE_BF16) {
        const uint16_t *p = static_cast<const uint16_t *>(logits);
        return launch_apply<uint16_t, false>(p, ld, p, ld, static_cast<uint16_t *>(out), ld_out, n_rows, V, R, st);
    }
    const float *p = static_cast<const float *>(logits);
    return launch_apply<float, false>(p, ld, p, ld, static_cast<float *>(out), ld_out, n_rows, V, R, st);
}

extern "C" int hilore_logits_apply_backward(const void *logits, int32_t dtype, int64_t n_rows, int64_t V, int64_t ld,
                                            const hilore_logit_rules *rules, const void *grad_out, int64_t ld_grad_out, void *grad_in,
                                            int64_t ld_grad_in, void *stream)
{
    if (!rules)
        return HILORE_INVALID_ARG;
    int bad = check_rows(dtype, n_rows, V, ld);
    if (!bad) bad = check_rules(rules, n_rows, V);
    if (bad)
        return bad;
    if (ld_grad_out < V || ld_grad_in < V)
        return HILORE_SHAPE;
    if (n_rows == 0)
        return HILORE_OK;
    if (!logits || !grad_out || !grad_in)
        return HILORE_INVALID_ARG;
    const size_t es = dtype == HILORE_BF16 ? 2 : 4;
    if (!aligned(logits, es) || !aligned(grad_out, es) || !aligned(grad_in, es))
        return HILORE_ALIGN;
    if (grad_in == logits) // the side of zero that a listed logit is on would be lost
        return HILORE_INVALID_ARG;
    if (grad_in == grad_out && ld_grad_in != ld_grad_out && n_rows > 1)
        return HILORE_SHAPE;
    const hilore_logit_rules R = used_rules(rules);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dtype == HILORE_BF16)
        return launch_apply<uint16_t, true>(static_cast<const uint16_t *>(logits), ld, static_cast<const uint16_t *>(grad_out), ld_grad_out,
                                            static_cast<uint16_t *>(grad_in), ld_grad_in, n_rows, V, R, st);
    return launch_apply<float, true>(static_cast<const float *>(logits), ld, static_cast<const float *>(grad_out), ld_grad_out,
                                     static_cast<float *>(grad_in), ld_grad_in, n_rows, V, R, st);
}

extern "C" int hilore_token_logp(const void *logits, int32_t dtype, int64_t n_rows, int64_t V, int64_t ld, const hilore_logit_rules *rules,
                                 const int32_t *targets, float *logp, float *lse, float *entropy, void *stream)
{
    int bad = check_rows(dtype, n_rows, V, ld);
    if (!bad && rules) bad = check_rules(rules, n_rows, V);
    if (bad)
        return bad;
    if (n_rows == 0)
        return HILORE_OK;
    if (!logits || !targets || !logp)
        return HILORE_INVALID_ARG;
    if (!aligned(logits, dtype == HILORE_BF16 ? 2 : 4) || !aligned(targets, 4) || !aligned(logp, 4) || !aligned(lse, 4) || !aligned(entropy, 4))
        return HILORE_ALIGN;
    const hilore_logit_rules R = used_rules(rules);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
#define HILORE_PICK(T)                                                                                                                          \
    const T *p = static_cast<const T *>(logits);                                                                                                \
    return entropy ? launch_logp<T, true>(p, ld, n_rows, V, targets, logp, lse, entropy, R, st)                                                 \
                   : launch_logp<T, false>(p, ld, n_rows, V, targets, logp, lse, entropy, R, st)
    if (dtype == HILORE_BF16) { HILORE_PICK(uint16_t); }
    HILORE_PICK(float);
#undef HILORE_PICK
}

extern "C" int hilore_token_logp_backward(const void *logits, int32_t dtype, int64_t n_rows, int64_t V, int64_t ld,
                                          const hilore_logit_rules *rules, const int32_t *targets, const float *lse, const float *omega,
                                          void *grad, int64_t ld_grad, void *stream)
{
    int bad = check_rows(dtype, n_rows, V, ld);
    if (!bad && rules) bad = check_rules(rules, n_rows, V);
    if (bad)
        return bad;
    if (ld_grad < V)
        return HILORE_SHAPE;
    if (n_rows == 0)
        return HILORE_OK;
    if (!logits || !targets || !lse || !omega || !grad)
        return HILORE_INVALID_ARG;
    const size_t es = dtype == HILORE_BF16 ? 2 : 4;
    if (!aligned(logits, es) || !aligned(grad, es) || !aligned(targets, 4) || !aligned(lse, 4) || !aligned(omega, 4))
        return HILORE_ALIGN;
    if (grad == logits && ld_grad != ld && n_rows > 1)
        return HILORE_SHAPE;
    const hilore_logit_rules R = used_rules(rules);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
#define HILORE_PICK(T)                                                                                                                          \
    const T *p = static_cast<const T *>(logits);                                                                                                \
    T *g = static_cast<T *>(grad);                                                                                                              \
    return launch_logp_backward<T>(p, ld, n_rows, V, targets, lse, omega, g, ld_grad, R, st)
    if (dtype == HILORE_BF16) { HILORE_PICK(uint16_t); }
    HILORE_PICK(float);
#undef HILORE_PICK
}
