// The vocabulary end of an actor update: rules on logits (penalties for repeated tokens, biases, grammar masks,
// temperature), log-probabilities of the sampled tokens under them, and the gradient of the logits from the update
// coefficients omega_t = dL/dlogp_t that the coefficient pass writes.
//
// All of it streams rows of V logits once, so HBM is the bound; what a row's rules say about single tokens is kept
// off that stream.  A CTA owns a range of 8192 tokens of a row.  It scans the row's history and bias list into a table with
// one word per token in shared memory, with a list of the tokens that occur; the stream runs as if no token were listed,
// the listed ones are worked out on their own, one per thread, and written over the stream's results or, where a sum is
// wanted, left out of the stream by one bit per token.  (Counts in global memory would cost 4 bytes per logit, twice the
// bf16 logits themselves.  Asking the table inside the stream serialises a warp over its listed tokens: gradients of
// 2048 x 128256 bf16 rows under prefixes of up to 1536 tokens took 329 us that way.  A hash table over a larger range needs
// fewer scans but probes and overflows: 96 rows of 151936 fp32 logits with histories up to 16384 took 320 us, 111 before.)
#include "common.cuh"

#include <cooperative_groups.h>
#include <cstdlib>

namespace cg = cooperative_groups;

namespace hilore {

constexpr float kLog2eF = 1.4426950408889634f;
constexpr float kLowest = -3.402823466e38f; // the running maximum of a row starts here: a row of -inf keeps a finite one
constexpr float kNothing = -1e30f;          // an lse at or below this belongs to a row without a token to choose from
constexpr uint32_t kSeen = 0x80000000u;     // bit of a count: the token occurs in the prompt part of the history

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
// leading dimension is.  Only the first and the last vector of a row can hold positions of other rows; their elements
// are loaded and stored one by one.
template <typename T> struct Row {
    T *origin; // address of position 0; never dereferenced outside [lead, end)
    int lead, end;
    __device__ __forceinline__ Row(const T *row, int V)
    {
        lead = (int)((reinterpret_cast<uintptr_t>(row) & 31) / sizeof(T));
        origin = const_cast<T *>(row) - lead;
        end = lead + V;
    }
    __device__ __forceinline__ bool whole(int f) const { return f >= lead && f + Lane<T>::N <= end; }
    __device__ __forceinline__ uint32_t valid(int f) const // bit i: position f + i belongs to the row
    {
        constexpr int N = Lane<T>::N;
        uint32_t m = (1u << N) - 1u;
        if (f < lead) m &= m << (lead - f);
        if (f + N > end) m = (f >= end) ? 0u : m & ((1u << (end - f)) - 1u);
        return m;
    }
    __device__ __forceinline__ void load(int f, uint32_t (&w)[8]) const
    {
        if (whole(f)) ld_global_256(origin + f, w);
        else load_part(origin, valid(f), f, w);
    }
    // Elements f .. f + N - 1 of `m` from base + f.
    static __device__ __forceinline__ void load_part(const T *base, uint32_t m, int f, uint32_t (&w)[8])
    {
        float z[Lane<T>::N];
#pragma unroll
        for (int i = 0; i < Lane<T>::N; ++i)
            z[i] = (m >> i & 1u) ? Lane<T>::one(base + f + i) : 0.0f;
        Lane<T>::pack(z, w);
    }
    __device__ __forceinline__ void store(int f, const float (&z)[Lane<T>::N]) const
    {
        if (whole(f)) {
            uint32_t w[8];
            Lane<T>::pack(z, w);
            st_global_256(origin + f, w);
            return;
        }
        const uint32_t m = valid(f);
#pragma unroll
        for (int i = 0; i < Lane<T>::N; ++i)
            if (m >> i & 1u) Lane<T>::put(origin + f + i, z[i]);
    }
};

// Reads of a row in the frame of another one (the row that is written).  Where the two addresses differ modulo 32 bytes, a
// vector is put together from two neighbouring aligned ones by a shift of whole words and, for bf16, of half a word; the
// second one hits L1.  (Element-wise stores instead, as a first version had, took 8.6 times as long as the bytes.)
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
    template <bool SHIFTED> __device__ __forceinline__ void load(const Row<T> &frame, int f, uint32_t (&w)[8]) const
    {
        constexpr int N = Lane<T>::N;
        if (!SHIFTED) {
            frame.whole(f) ? ld_global_256(exact + f, w) : Row<T>::load_part(exact, frame.valid(f), f, w);
            return;
        }
        const int lo = (int)(aligned - own.origin) + f; // position of the first aligned vector in the read row's own frame
        if (!own.whole(lo) || !own.whole(lo + N)) {
            Row<T>::load_part(exact, frame.valid(f), f, w);
            return;
        }
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
    __device__ __forceinline__ bool listed() const { return hist_lo < hist_hi || bias_lo < bias_hi; }
};

__device__ __forceinline__ RowRules row_rules(const hilore_logit_rules &R, int64_t row)
{
    RowRules q;
    const float t = R.temperature ? R.temperature[row] : 1.0f;
    q.inv_temp = t > 0.0f ? __fdiv_rn(1.0f, t) : 1.0f; // 0 (greedy) and what is no temperature: not scaled
    q.rep = R.repetition ? R.repetition[row] : 1.0f;
    q.inv_rep = __fdiv_rn(1.0f, q.rep);
    q.freq = R.frequency ? R.frequency[row] : 0.0f;
    q.pres = R.presence ? R.presence[row] : 0.0f;
    q.hist_lo = q.hist_hi = q.hist_mid = q.bias_lo = q.bias_hi = 0;
    if (R.tokens && !(q.rep == 1.0f && q.freq == 0.0f && q.pres == 0.0f)) {
        q.hist_lo = max((int64_t)0, R.hist_begin[row]);
        q.hist_hi = min(R.n_tokens, R.hist_end[row]);
        q.hist_mid = R.resp_begin[row];
    }
    if (R.bias_tokens) {
        q.bias_lo = max((int64_t)0, R.bias_offsets[row]);
        q.bias_hi = min(R.n_bias, R.bias_offsets[row + 1]);
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

// The listed tokens of a range [first, last) of positions: a table with one word per position -- kSeen if the token occurs
// in the prompt part of the history, 11 bits of the number of the last bias entry that names it, 20 bits of its occurrences
// in the generated part -- and the places that are not zero, in the order they were found.
// A row with a longer bias list or a longer generated part takes two words per position and ranges of half the width.
constexpr int kWords = 8192;
constexpr int kCountBits = 20, kBiasBits = 11;

struct Listed {
    uint32_t *word;  // [kWords]
    uint16_t *list;  // [kWords]
    uint32_t *touch; // [kWords / 32] bit f - first: the token at position f is listed; nullptr where the stream does not ask
    int *n;          // entries of the list
    int first;
    bool wide;
};

constexpr size_t kListedBytes = kWords * 6 + kWords / 8;

__device__ __forceinline__ Listed listed_at(unsigned char *smem, const RowRules &q, bool bits, int *n)
{
    Listed t;
    t.word = reinterpret_cast<uint32_t *>(smem);
    t.touch = bits ? t.word + kWords : nullptr;
    t.list = reinterpret_cast<uint16_t *>(t.word + kWords + kWords / 32);
    t.n = n;
    t.first = 0;
    t.wide = q.hist_hi - q.hist_mid >= (1 << kCountBits) || q.bias_hi - q.bias_lo >= (1 << kBiasBits);
    return t;
}

__device__ __forceinline__ void list_place(const Listed &t, uint32_t s)
{
    t.list[atomicAdd(t.n, 1)] = (uint16_t)s;
    if (t.touch) atomicOr(t.touch + (s >> 5), 1u << (s & 31));
}

constexpr int kScan = 8; // history tokens in flight per thread

// Up to kScan * THREADS tokens of the history from i0 on (-1 past its end).
template <int THREADS> __device__ __forceinline__ void history_load(const hilore_logit_rules &R, const RowRules &q, int64_t i0, int (&v)[kScan])
{
#pragma unroll
    for (int u = 0; u < kScan; ++u) {
        const int64_t i = i0 + u * THREADS + threadIdx.x;
        v[u] = i < q.hist_hi ? __ldg(R.tokens + i) : -1;
    }
}

// Fills table and list for positions [t.first, last).  `head`: the first kScan * THREADS tokens of the history, which a
// caller with several ranges keeps in registers.  Ends with the CTA synchronised.
template <int THREADS>
__device__ __forceinline__ void fill_listed(const hilore_logit_rules &R, const RowRules &q, int V, int lead, int last, const Listed &t,
                                            const int (&head)[kScan])
{
    const int tid = threadIdx.x;
    const int words = kWords + (t.touch ? kWords / 32 : 0);
    for (int i = tid; i < words / 4; i += THREADS)
        reinterpret_cast<uint4 *>(t.word)[i] = make_uint4(0, 0, 0, 0);
    if (tid == 0) *t.n = 0;
    __syncthreads();
    const int v0 = t.first - lead;
    const uint32_t width = (uint32_t)(last - t.first);
    if (q.bias_lo < q.bias_hi) { // before the counts: the largest number of a word is that of the last entry
        for (int64_t i = q.bias_lo + tid; i < q.bias_hi; i += THREADS) {
            const int v = __ldg(R.bias_tokens + i);
            const uint32_t s = (uint32_t)(v - v0), k = (uint32_t)(i - q.bias_lo) + 1u;
            if (s < width && (uint32_t)v < (uint32_t)V) {
                const uint32_t old = t.wide ? atomicMax(t.word + 2 * s + 1, k) : atomicMax(t.word + s, k << kCountBits);
                if (old == 0) list_place(t, s);
            }
        }
        __syncthreads();
    }
    for (int64_t i0 = q.hist_lo; i0 < q.hist_hi; i0 += THREADS * kScan) {
        int v[kScan];
        if (i0 == q.hist_lo) {
#pragma unroll
            for (int u = 0; u < kScan; ++u)
                v[u] = head[u];
        } else {
            history_load<THREADS>(R, q, i0, v);
        }
#pragma unroll
        for (int u = 0; u < kScan; ++u) {
            const uint32_t s = (uint32_t)(v[u] - v0);
            if (s < width && (uint32_t)v[u] < (uint32_t)V) {
                uint32_t *w = t.word + (t.wide ? 2 * s : s);
                const uint32_t old = i0 + u * THREADS + tid < q.hist_mid ? atomicOr(w, kSeen) : atomicAdd(w, 1u);
                if (old == 0 && !(t.wide && w[1] != 0)) list_place(t, s);
            }
        }
    }
    __syncthreads();
}

// Puts the list in the order of positions, from the touch bits: a sum over listed tokens must not depend on the order in which
// atomics found them.  `sums`: one word per warp.  Ends with the CTA synchronised.
template <int THREADS> __device__ __forceinline__ void order_listed(const Listed &t, uint32_t *sums)
{
    static_assert(THREADS == kWords / 32, "one word of touch bits per thread");
    const int tid = threadIdx.x, lane = tid & 31;
    uint32_t w = t.touch[tid];
    uint32_t at = (uint32_t)__popc(w);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t below = __shfl_up_sync(0xFFFFFFFFu, at, o);
        if (lane >= o) at += below;
    }
    if (lane == 31) sums[tid >> 5] = at;
    __syncthreads();
    at -= (uint32_t)__popc(w);
    for (int k = 0; k < (tid >> 5); ++k)
        at += sums[k];
    for (; w; w &= w - 1)
        t.list[at++] = (uint16_t)(tid * 32 + __ffs((int)w) - 1);
    __syncthreads();
}

// Place, count and bias entry of the i-th listed token.
__device__ __forceinline__ int listed_token(const Listed &t, int i, uint32_t &count, uint32_t &bias)
{
    const int s = t.list[i];
    if (t.wide) {
        count = t.word[2 * s];
        bias = t.word[2 * s + 1];
    } else {
        const uint32_t w = t.word[s];
        count = w & (kSeen | ((1u << kCountBits) - 1u));
        bias = w >> kCountBits & ((1u << kBiasBits) - 1u);
    }
    return s;
}

// The logit of a listed token under the penalties and its bias, before the temperature.
__device__ __forceinline__ float adjusted(float x, uint32_t count, uint32_t bias, const RowRules &q, const hilore_logit_rules &R)
{
    if (count) {
        x = x > 0.0f ? x * q.inv_rep : x * q.rep;
        const uint32_t c = count & ~kSeen;
        if (c) x = x - fmaf(q.freq, (float)c, q.pres);
    }
    if (bias) x += __ldg(R.bias_values + q.bias_lo + bias - 1);
    return x;
}

// d(adjusted logit) / d(logit) of a listed token.
__device__ __forceinline__ float slope_of(float x, uint32_t count, const RowRules &q)
{
    return count ? (x > 0.0f ? q.inv_rep : q.rep) : 1.0f;
}

// ------------------------------------------------------------------------------------------ element-wise results of a row
// What all three element-wise calls share: out[v] = plain(in[v]) for every token, listed(...) for the listed ones, `off` where
// the grammar denies.  One CTA per (row, range of `width` positions).
constexpr int kMapThreads = 256;

struct MapApply { // z from x
    static constexpr bool kGrad = false;
    float inv_temp;
    template <int N> __device__ __forceinline__ void plain(float (&z)[N], int) const
    {
#pragma unroll
        for (int i = 0; i < N; ++i)
            z[i] *= inv_temp;
    }
    __device__ __forceinline__ float listed(float in, float, int, uint32_t c, uint32_t b, const RowRules &q, const hilore_logit_rules &R) const
    {
        return adjusted(in, c, b, q, R) * inv_temp;
    }
    static __device__ __forceinline__ float off() { return -INFINITY; }
};

struct MapApplyGrad { // dx from dz; x is read at listed tokens only (the side of zero they are on)
    static constexpr bool kGrad = true;
    float inv_temp;
    template <int N> __device__ __forceinline__ void plain(float (&z)[N], int) const
    {
#pragma unroll
        for (int i = 0; i < N; ++i)
            z[i] *= inv_temp;
    }
    __device__ __forceinline__ float listed(float in, float x, int, uint32_t c, uint32_t, const RowRules &q, const hilore_logit_rules &) const
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
    template <int N> __device__ __forceinline__ void plain(float (&z)[N], int f) const
    {
        const int at = target - f;
#pragma unroll
        for (int i = 0; i < N; ++i)
            z[i] = one(z[i], i == at);
    }
    __device__ __forceinline__ float listed(float in, float, int f, uint32_t c, uint32_t b, const RowRules &q, const hilore_logit_rules &R) const
    {
        return one(adjusted(in, c, b, q, R), f == target) * slope_of(in, c, q);
    }
    static __device__ __forceinline__ float off() { return 0.0f; }
};

// 32 logits of every thread: the vectors of kMapThreads * 32 positions from `f0` on, in flight together.
constexpr int kMapStage = kMapThreads * 32;
static_assert(kMapStage == kWords, "a range with listed tokens is one stage of the stream");

template <typename T> struct Stage {
    static constexpr int N = Lane<T>::N, U = 32 / N;
    static constexpr uint32_t kAll = (1u << N) - 1u;
    uint32_t w[U][8], deny[U];
    template <bool SHIFTED>
    __device__ __forceinline__ void load(const Row<T> &dst, const Source<T> &src, const uint32_t *mask, int n_words, int f0, int b)
    {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int f = f0 + (u * kMapThreads + (int)threadIdx.x) * N;
            deny[u] = f < b && mask ? denied<N>(mask, n_words, f - dst.lead) : 0u;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int f = f0 + (u * kMapThreads + (int)threadIdx.x) * N;
            if (f < b && deny[u] != kAll) src.template load<SHIFTED>(dst, f, w[u]); // a vector without an allowed token is not read
        }
    }
    template <typename Map> __device__ __forceinline__ void store(const Row<T> &dst, const Map &map, int f0, int b)
    {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int f = f0 + (u * kMapThreads + (int)threadIdx.x) * N;
            if (f >= b)
                break;
            float z[N];
            Lane<T>::unpack(w[u], z);
            map.plain(z, f);
            if (deny[u]) {
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (deny[u] >> i & 1u) z[i] = Map::off();
            }
            dst.store(f, z);
        }
    }
};

template <typename T, bool SHIFTED, typename Map>
__device__ __forceinline__ void map_range(const Row<T> &dst, const Source<T> &src, const T *in, const T *x, const Map &map, const RowRules &q,
                                          const hilore_logit_rules &R, int V, int a, int b, unsigned char *smem, int *n)
{
    const int n_words = (V + 31) >> 5;
    Stage<T> stage;
    if (!q.listed()) {
        for (; a < b; a += kMapStage) {
            stage.template load<SHIFTED>(dst, src, q.mask, n_words, a, b);
            stage.store(dst, map, a, b);
        }
        return;
    }
    Listed t = listed_at(smem, q, false, n);
    int head[kScan];
    history_load<kMapThreads>(R, q, q.hist_lo, head);
    for (; a < b; a += t.wide ? kWords / 2 : kWords) {
        const int e = min(b, a + (t.wide ? kWords / 2 : kWords));
        stage.template load<SHIFTED>(dst, src, q.mask, n_words, a, e);
        t.first = a;
        fill_listed<kMapThreads>(R, q, V, dst.lead, e, t, head);
        // their results take the place of their words; all are read before anything is stored, as `out` may be `in`
        for (int i = threadIdx.x; i < *n; i += kMapThreads) {
            uint32_t c, k;
            const int s = listed_token(t, i, c, k), f = a + s, v = f - dst.lead;
            const float r = is_denied(q.mask, v) ? Map::off() : map.listed(Lane<T>::one(in + v), Map::kGrad ? Lane<T>::one(x + v) : 0.0f, f, c, k, q, R);
            t.word[t.wide ? 2 * s : s] = __float_as_uint(r);
        }
        __syncthreads();
        stage.store(dst, map, a, e);
        __syncthreads(); // the stream's results of listed tokens are there to be written over
        for (int i = threadIdx.x; i < *n; i += kMapThreads) {
            const int s = t.list[i];
            Lane<T>::put(dst.origin + (a + s), __uint_as_float(t.word[t.wide ? 2 * s : s]));
        }
        if (e < b) __syncthreads();
    }
}

template <typename T, typename Map>
__device__ __forceinline__ void map_row(const Row<T> &dst, const T *in, const T *x, const Map &map, const RowRules &q, const hilore_logit_rules &R,
                                        int V, int a, int b, unsigned char *smem, int *n)
{
    const Source<T> src(in, V, dst);
    if (src.shift == 0) map_range<T, false>(dst, src, in, x, map, q, R, V, a, b, smem, n);
    else map_range<T, true>(dst, src, in, x, map, q, R, V, a, b, smem, n);
}

// One CTA per (row, range).
template <typename T, bool GRAD>
__global__ void __launch_bounds__(kMapThreads, sizeof(T) == 2 ? 4 : 3)
    logits_apply_kernel(const T *x, int64_t ld, const T *in, int64_t ld_in, T *out, int64_t ld_out, int V, int n_ranges, int width,
                        const __grid_constant__ hilore_logit_rules R)
{
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ int n_listed;
    const int64_t row = blockIdx.x / n_ranges;
    const int a = (int)(blockIdx.x - row * n_ranges) * width;
    const Row<T> dst(out + row * ld_out, V);
    if (a >= dst.end)
        return;
    const int b = min(dst.end, a + width);
    const RowRules q = row_rules(R, row);
    if (GRAD) map_row(dst, in + row * ld_in, x + row * ld, MapApplyGrad{q.inv_temp}, q, R, V, a, b, smem, &n_listed);
    else map_row(dst, in + row * ld_in, x + row * ld, MapApply{q.inv_temp}, q, R, V, a, b, smem, &n_listed);
}

// One CTA per (row, range); rows whose coefficient is zero, that have no token, whose token the grammar denies or that had
// nothing to choose from get zeros without being read.
template <typename T>
__global__ void __launch_bounds__(kMapThreads, sizeof(T) == 2 ? 4 : 3)
    token_logp_backward_kernel(const T *x, int64_t ld, int V, int n_ranges, int width, const int32_t *targets, const float *lse,
                               const float *omega, T *grad, int64_t ld_grad, const __grid_constant__ hilore_logit_rules R)
{
    constexpr int N = Lane<T>::N;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ int n_listed;
    const int64_t row = blockIdx.x / n_ranges;
    const int a = (int)(blockIdx.x - row * n_ranges) * width;
    const Row<T> dst(grad + row * ld_grad, V);
    if (a >= dst.end)
        return;
    const int b = min(dst.end, a + width);
    const int target = targets[row];
    const float om = omega[row], l = lse[row];
    const RowRules q = row_rules(R, row);
    if ((uint32_t)target >= (uint32_t)V || om == 0.0f || l <= kNothing || is_denied(q.mask, target)) {
        const float zero[N] = {};
        for (int f = a + (int)threadIdx.x * N; f < b; f += kMapThreads * N)
            dst.store(f, zero);
        return;
    }
    map_row(dst, x + row * ld, x + row * ld, MapLogpGrad{q.inv_temp, l, om * q.inv_temp, target + dst.lead}, q, R, V, a, b, smem, &n_listed);
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
    float s0 = 0.0f, s1 = 0.0f, t0 = 0.0f, t1 = 0.0f;
#pragma unroll
    for (int i = 0; i < N; i += 2) {
        float u0 = (z[i] - m) * c, u1 = (z[i + 1] - m) * c;
        if (ENTROPY) { // 2^-256 is zero in fp32: keeps -inf out of the product
            u0 = fmaxf(u0, -256.0f);
            u1 = fmaxf(u1, -256.0f);
        }
        const float e0 = ex2_ftz(u0), e1 = ex2_ftz(u1);
        s0 += e0;
        s1 += e1;
        if (ENTROPY) {
            t0 = fmaf(e0, u0, t0);
            t1 = fmaf(e1, u1, t1);
        }
    }
    q.s += s0 + s1;
    if (ENTROPY) q.t += t0 + t1;
}

// Adds one logit.
template <bool ENTROPY> __device__ __forceinline__ void soft_one(Soft &q, float z, float c)
{
    const float one[2] = {z, -INFINITY};
    soft_add<2, ENTROPY>(q, one, c);
}

constexpr int kLogpThreads = 256, kMaxRowCtas = 8;

// A row belongs to `row_ctas` CTAs (a thread-block cluster if more than one); each takes a share of its vectors.  RULES: more
// than a temperature.
template <typename T, bool RULES, bool ENTROPY>
__global__ void __launch_bounds__(kLogpThreads, RULES && sizeof(T) == 4 ? 3 : 4)
    token_logp_kernel(const T *x, int64_t ld, int V, int row_ctas, const int32_t *targets, float *logp, float *lse, float *entropy,
                      const __grid_constant__ hilore_logit_rules R)
{
    constexpr int N = Lane<T>::N, U = 32 / N;
    constexpr uint32_t kAll = (1u << N) - 1u;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ Soft part[kLogpThreads / 32];
    __shared__ uint32_t sums[kLogpThreads / 32];
    __shared__ Soft shares[kMaxRowCtas];
    __shared__ float target_z; // the target's logit under penalties and bias; in the cluster's first CTA
    __shared__ int n_listed;
    const int tid = threadIdx.x, lane = tid & 31;
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
    const T *xrow = x + row * ld;
    const RowRules q = row_rules(R, row);
    if (rank == 0 && tid == 0) target_z = is_denied(q.mask, target) ? -INFINITY : Lane<T>::one(xrow + target);
    if (row_ctas > 1)
        cl.sync(); // every CTA of the row runs, and target_z is set, before anything is sent to the first one
    float *first_z = row_ctas > 1 ? cl.map_shared_rank(&target_z, 0) : &target_z;

    const Row<T> src(xrow, V);
    const int n_vec = (src.end + N - 1) / N, n_words = (V + 31) >> 5;
    int a = (int)((int64_t)n_vec * rank / row_ctas) * N;
    const int b = (int)((int64_t)n_vec * (rank + 1) / row_ctas) * N;
    const float c = kLog2eF * q.inv_temp;
    Soft acc{kLowest, 0.0f, 0.0f};
    if (!RULES) {
        for (int f0 = a + tid * N; f0 < b; f0 += kLogpThreads * 32) {
            uint32_t w[U][8];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int f = f0 + u * kLogpThreads * N;
                if (f < b) src.load(f, w[u]);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int f = f0 + u * kLogpThreads * N;
                if (f < b) {
                    float z[N];
                    Lane<T>::unpack(w[u], z);
                    if (!src.whole(f)) {
                        const uint32_t ok = src.valid(f);
#pragma unroll
                        for (int i = 0; i < N; ++i)
                            if (!(ok >> i & 1u)) z[i] = -INFINITY;
                    }
                    soft_add<N, ENTROPY>(acc, z, c);
                }
            }
        }
    } else {
        const bool lists = q.listed();
        Listed t = listed_at(smem, q, true, &n_listed);
        int head[kScan];
        if (lists) history_load<kLogpThreads>(R, q, q.hist_lo, head);
        const int width = lists && t.wide ? kWords / 2 : kWords;
        for (; a < b; a += width) {
            const int e = min(b, a + width);
            uint32_t w[U][8], off[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int f = a + (u * kLogpThreads + tid) * N;
                off[u] = f < e && q.mask ? denied<N>(q.mask, n_words, f - src.lead) : 0u;
                off[u] |= f < e ? ~src.valid(f) & kAll : kAll;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int f = a + (u * kLogpThreads + tid) * N;
                if (off[u] != kAll) src.load(f, w[u]); // a vector without an allowed token is not read
            }
            if (lists) {
                t.first = a;
                __syncthreads(); // the previous range is done with the table
                fill_listed<kLogpThreads>(R, q, V, src.lead, e, t, head);
                order_listed<kLogpThreads>(t, sums);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int s = (u * kLogpThreads + tid) * N;
                    off[u] |= t.touch[s >> 5] >> (s & 31) & kAll;
                }
                for (int i = tid; i < n_listed; i += kLogpThreads) {
                    uint32_t n, k;
                    const int v = a + listed_token(t, i, n, k) - src.lead;
                    if (is_denied(q.mask, v))
                        continue;
                    const float z = adjusted(Lane<T>::one(xrow + v), n, k, q, R);
                    if (v == target) *first_z = z;
                    soft_one<ENTROPY>(acc, z, c);
                }
            }
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
    }

#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        Soft other;
        other.m = __shfl_xor_sync(0xFFFFFFFFu, acc.m, o);
        other.s = __shfl_xor_sync(0xFFFFFFFFu, acc.s, o);
        other.t = ENTROPY ? __shfl_xor_sync(0xFFFFFFFFu, acc.t, o) : 0.0f;
        acc = soft_join<ENTROPY>(acc, other, c);
    }
    if (lane == 0) part[tid >> 5] = acc;
    __syncthreads();
    if (tid == 0) {
        for (int w = 1; w < kLogpThreads / 32; ++w)
            acc = soft_join<ENTROPY>(acc, part[w], c);
        if (row_ctas > 1) *cl.map_shared_rank(&shares[rank], 0) = acc;
    }
    if (row_ctas > 1)
        cl.sync(); // the shares have arrived in the first CTA
    if (rank != 0 || tid != 0)
        return;
    for (int r = 1; r < row_ctas; ++r)
        acc = soft_join<ENTROPY>(acc, shares[r], c);
    const float ln_s = logf(acc.s);
    float l = fmaf(acc.m, q.inv_temp, ln_s), p = fmaf(target_z - acc.m, q.inv_temp, -ln_s), h = 0.0f;
    if (acc.m == INFINITY) { // the sum has no value (inf - inf); its logarithm has
        l = INFINITY;
        p = target_z - acc.m;
    } else if (acc.m == kLowest && acc.s == 0.0f) { // nothing to choose from
        l = -INFINITY;
        p = -INFINITY;
    }
    if (ENTROPY) { // H = ln s - sum p u ln 2
        h = acc.m == kLowest && acc.s == 0.0f ? 0.0f : fmaf(-acc.t / acc.s, 0.6931471805599453f, ln_s);
        if (acc.m != acc.m || acc.m == INFINITY) h = acc.m - acc.m;
        entropy[row] = h;
    }
    logp[row] = p;
    if (lse) lse[row] = l;
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

// Dynamic shared memory beyond 48 KB (with the kernels' static few hundred bytes) needs an opt-in.
template <typename K> static bool allow_smem(K kernel, size_t bytes)
{
    return bytes <= 47 * 1024 || cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == cudaSuccess;
}

// Positions of a CTA's range in the element-wise calls: one table of listed tokens, twice that where there are none, and less
// while that leaves SMs without four CTAs.
static int64_t range_width(int64_t n_rows, int64_t V, const hilore_logit_rules &R)
{
    int64_t width = R.tokens || R.bias_tokens ? kWords : 2 * kWords;
    while (width > 2048 && n_rows * ((V + width - 1) / width) < 4 * (int64_t)sm_count())
        width /= 2;
    return width;
}

template <typename T, bool GRAD>
static int launch_apply(const T *x, int64_t ld, const T *in, int64_t ld_in, T *out, int64_t ld_out, int64_t n_rows, int64_t V,
                        const hilore_logit_rules &R, cudaStream_t st)
{
    const int64_t width = range_width(n_rows, V, R), n = (V + Lane<T>::N - 1 + width - 1) / width;
    if (n * n_rows > 0x7FFFFFFF)
        return HILORE_SHAPE;
    auto kernel = logits_apply_kernel<T, GRAD>;
    const size_t smem = R.tokens || R.bias_tokens ? kListedBytes : 0;
    if (!allow_smem(kernel, smem))
        return HILORE_CUDA;
    kernel<<<(unsigned)(n * n_rows), kMapThreads, smem, st>>>(x, ld, in, ld_in, out, ld_out, (int)V, (int)n, (int)width, R);
    return cudaGetLastError() == cudaSuccess ? HILORE_OK : HILORE_CUDA;
}

static bool clusters_on()
{
    const char *off = std::getenv("HILORE_DISABLE_CLUSTER_LAUNCH");
    return off == nullptr || off[0] == '\0' || (off[0] == '0' && off[1] == '\0');
}

template <typename T, bool RULES, bool ENTROPY>
static int launch_logp(const T *x, int64_t ld, int64_t n_rows, int64_t V, const int32_t *targets, float *logp, float *lse, float *entropy,
                       const hilore_logit_rules &R, cudaStream_t st)
{
    auto kernel = token_logp_kernel<T, RULES, ENTROPY>;
    // CTAs per row: as many as keep the SMs busy with two each, at most a portable cluster, none with less than 2048 logits
    int row_ctas = 1;
    if (clusters_on())
        while (row_ctas < kMaxRowCtas && n_rows * row_ctas < 2 * (int64_t)sm_count() && V / (2 * row_ctas) >= 2048)
            row_ctas *= 2;
    if (n_rows * row_ctas > 0x7FFFFFFF)
        return HILORE_SHAPE;
    const size_t smem = R.tokens || R.bias_tokens ? kListedBytes : 0;
    if (!allow_smem(kernel, smem))
        return HILORE_CUDA;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(n_rows * row_ctas));
    cfg.blockDim = dim3(kLogpThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)row_ctas;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = row_ctas > 1 ? 1 : 0;
    if (cudaLaunchKernelEx(&cfg, kernel, x, ld, (int)V, row_ctas, targets, logp, lse, entropy, R) != cudaSuccess)
        return HILORE_CUDA;
    return cudaGetLastError() == cudaSuccess ? HILORE_OK : HILORE_CUDA;
}

template <typename T>
static int launch_logp_backward(const T *x, int64_t ld, int64_t n_rows, int64_t V, const int32_t *targets, const float *lse, const float *omega,
                                T *grad, int64_t ld_grad, const hilore_logit_rules &R, cudaStream_t st)
{
    const int64_t width = range_width(n_rows, V, R), n = (V + Lane<T>::N - 1 + width - 1) / width;
    if (n * n_rows > 0x7FFFFFFF)
        return HILORE_SHAPE;
    auto kernel = token_logp_backward_kernel<T>;
    const size_t smem = R.tokens || R.bias_tokens ? kListedBytes : 0;
    if (!allow_smem(kernel, smem))
        return HILORE_CUDA;
    kernel<<<(unsigned)(n * n_rows), kMapThreads, smem, st>>>(x, ld, (int)V, (int)n, (int)width, targets, lse, omega, grad, ld_grad, R);
    return cudaGetLastError() == cudaSuccess ? HILORE_OK : HILORE_CUDA;
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
    if (more_than_temperature(R))                                                                                                                        \
        return entropy ? launch_logp<T, true, true>(p, ld, n_rows, V, targets, logp, lse, entropy, R, st)                                       \
                       : launch_logp<T, true, false>(p, ld, n_rows, V, targets, logp, lse, entropy, R, st);                                     \
    return entropy ? launch_logp<T, false, true>(p, ld, n_rows, V, targets, logp, lse, entropy, R, st)                                          \
                   : launch_logp<T, false, false>(p, ld, n_rows, V, targets, logp, lse, entropy, R, st)
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
