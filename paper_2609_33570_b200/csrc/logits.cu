// The vocabulary end of an actor update: rules on logits (penalties for repeated tokens, biases, grammar masks,
// temperature), log-probabilities of the sampled tokens under them, and the gradient of the logits from the update
// coefficients omega_t = dL/dlogp_t that the coefficient pass writes.
//
// All of it streams rows of V logits once, so HBM is the bound; what a row's rules say about single tokens is kept
// off that stream.  A CTA owns a segment of a row.  It scans the row's history once and keeps, in shared memory, a
// bit per token of the segment that the rules touch, a bit per token that the grammar denies, and a count for the
// touched ones; the loop over the logits then asks one 32-bit word per 16 tokens, and only vectors with a bit set leave
// the plain path.  (Dense counts in global memory would cost 4 bytes per logit, twice the bf16 logits themselves.)
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
        if (whole(f)) {
            ld_global_256(origin + f, w);
            return;
        }
        const uint32_t m = valid(f);
        float z[Lane<T>::N];
#pragma unroll
        for (int i = 0; i < Lane<T>::N; ++i)
            z[i] = (m >> i & 1u) ? Lane<T>::one(origin + f + i) : 0.0f;
        Lane<T>::pack(z, w);
    }
    __device__ __forceinline__ void store(int f, const float (&z)[Lane<T>::N], bool vectors) const
    {
        if (vectors && whole(f)) {
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

// What the rules of one row say, in registers.
struct RowRules {
    float inv_temp, rep, inv_rep, freq, pres;
    const float *bias; // values of the row's list; entry k of the list has number k + 1
};

__device__ __forceinline__ float inverse_temperature(const hilore_logit_rules &R, int64_t row)
{
    const float t = R.temperature ? R.temperature[row] : 1.0f;
    return t > 0.0f ? __fdiv_rn(1.0f, t) : 1.0f; // 0 (greedy) and what is no temperature: not scaled
}

__device__ __forceinline__ RowRules row_rules(const hilore_logit_rules &R, int64_t row)
{
    RowRules q;
    q.inv_temp = inverse_temperature(R, row);
    q.rep = R.repetition ? R.repetition[row] : 1.0f;
    q.inv_rep = __fdiv_rn(1.0f, q.rep);
    q.freq = R.frequency ? R.frequency[row] : 0.0f;
    q.pres = R.presence ? R.presence[row] : 0.0f;
    q.bias = nullptr;
    return q;
}

// Words of the row's grammar mask, or nullptr where no mask applies.
__device__ __forceinline__ const uint32_t *row_mask(const hilore_logit_rules &R, int64_t row)
{
    if (R.allow == nullptr)
        return nullptr;
    const int64_t a = R.allow_row ? (int64_t)R.allow_row[row] : row;
    return (a < 0 || a >= R.n_allow) ? nullptr : reinterpret_cast<const uint32_t *>(R.allow) + a * R.allow_ld;
}

// Shared-memory tables of one segment (positions [f0, f0 + SEG) of a row's frame):
//   bits  [SEG / 16]  low half: the rules touch the token; high half: the grammar denies it
//   count [SEG]       occurrences in the generated part of the history, kSeen if in the prompt part as well or alone
//   bias  [SEG]       number of the last entry of the row's bias list that names the token
// count and bias hold zeros outside of touched tokens; whoever consumes a touched token puts the zero back.
struct Tables {
    uint32_t *bits, *count, *bias;
};

template <int SEG>
__device__ __forceinline__ Tables tables_at(unsigned char *smem, const hilore_logit_rules &R)
{
    Tables t;
    t.bits = reinterpret_cast<uint32_t *>(smem);
    t.count = t.bits + SEG / 16;
    t.bias = t.count + (R.tokens ? SEG : 0);
    return t;
}

template <int SEG> static size_t tables_bytes(const hilore_logit_rules &R)
{
    return (size_t)(SEG / 16 + (R.tokens ? SEG : 0) + (R.bias_tokens ? SEG : 0)) * 4;
}

template <int SEG, int THREADS> __device__ __forceinline__ void clear_tables(const Tables &t, const hilore_logit_rules &R)
{
    const int words = (R.tokens ? SEG : 0) + (R.bias_tokens ? SEG : 0);
    uint4 *p = reinterpret_cast<uint4 *>(t.count);
    for (int i = threadIdx.x; i < words / 4; i += THREADS)
        p[i] = make_uint4(0, 0, 0, 0);
}

// 16 mask bits from token v on (bits of tokens outside the vocabulary are arbitrary).
__device__ __forceinline__ uint32_t mask_bits16(const uint32_t *words, int n_words, int v)
{
    const int i = v >> 5, sh = v & 31;
    const uint32_t lo = (i >= 0 && i < n_words) ? __ldg(words + i) : 0u;
    const uint32_t hi = (sh > 16 && i + 1 >= 0 && i + 1 < n_words) ? __ldg(words + i + 1) : 0u;
    return __funnelshift_r(lo, hi, sh) & 0xFFFFu;
}

// Fills the tables for the segment; ends with the CTA synchronised.  `t.bits` may still be in use by the previous
// segment's loop when this is entered (it synchronises first).
template <int SEG, int THREADS>
__device__ __forceinline__ void fill_tables(const hilore_logit_rules &R, int64_t row, const uint32_t *mask, int V, int lead, int f0,
                                            const Tables &t)
{
    const int tid = threadIdx.x, n_words = (V + 31) >> 5;
    __syncthreads();
    for (int w = tid; w < SEG / 16; w += THREADS)
        t.bits[w] = mask ? (~mask_bits16(mask, n_words, f0 - lead + 16 * w) & 0xFFFFu) << 16 : 0u;
    __syncthreads();
    const int v0 = f0 - lead;
    if (R.tokens) {
        const int64_t lo = max((int64_t)0, R.hist_begin[row]), hi = min(R.n_tokens, R.hist_end[row]), mid = R.resp_begin[row];
        for (int64_t i = lo + tid; i < hi; i += THREADS) {
            const int v = __ldg(R.tokens + i);
            const uint32_t s = (uint32_t)(v - v0);
            if (s < (uint32_t)SEG && (uint32_t)v < (uint32_t)V) {
                if (i < mid) atomicOr(t.count + s, kSeen);
                else atomicAdd(t.count + s, 1u);
                atomicOr(t.bits + (s >> 4), 1u << (s & 15));
            }
        }
    }
    if (R.bias_tokens) {
        const int64_t lo = max((int64_t)0, R.bias_offsets[row]), hi = min(R.n_bias, R.bias_offsets[row + 1]);
        for (int64_t i = lo + tid; i < hi; i += THREADS) {
            const int v = __ldg(R.bias_tokens + i);
            const uint32_t s = (uint32_t)(v - v0);
            if (s < (uint32_t)SEG && (uint32_t)v < (uint32_t)V) {
                atomicMax(t.bias + s, (uint32_t)(i - lo) + 1u);
                atomicOr(t.bits + (s >> 4), 1u << (s & 15));
            }
        }
    }
    __syncthreads();
}

__device__ __forceinline__ const float *row_bias(const hilore_logit_rules &R, int64_t row)
{
    return R.bias_tokens ? R.bias_values + max((int64_t)0, R.bias_offsets[row]) : nullptr;
}

// Bits of the vector at segment position s (a multiple of N): touched in the low half, denied in the high half.
template <int N> __device__ __forceinline__ uint32_t vector_bits(const uint32_t *bits, int s)
{
    const uint32_t w = bits[s >> 4];
    return N == 16 ? w : (w >> (s & 8)) & 0x00FF00FFu;
}

// A touched token's count and bias entry; leaves zeros behind.
__device__ __forceinline__ void take_entry(const Tables &t, const hilore_logit_rules &R, int s, uint32_t &count, uint32_t &bias)
{
    count = 0;
    bias = 0;
    if (R.tokens) {
        count = t.count[s];
        t.count[s] = 0;
    }
    if (R.bias_tokens) {
        bias = t.bias[s];
        t.bias[s] = 0;
    }
}

// The logit of a touched token under the penalties and its bias, before the temperature.
__device__ __forceinline__ float adjusted(float x, uint32_t count, uint32_t bias, const RowRules &q)
{
    if (count) {
        x = x > 0.0f ? x * q.inv_rep : x * q.rep;
        const uint32_t c = count & ~kSeen;
        if (c) x = x - fmaf(q.freq, (float)c, q.pres);
    }
    if (bias) x += __ldg(q.bias + bias - 1);
    return x;
}

// d(adjusted logit) / d(logit) of a touched token.
__device__ __forceinline__ float slope_of(float x, uint32_t count, const RowRules &q)
{
    return count ? (x > 0.0f ? q.inv_rep : q.rep) : 1.0f;
}

// ------------------------------------------------------------------------------------------------ rules and their gradient
// One CTA per (row, segment).  GRAD: in = gradient of the processed logits, out = gradient of the logits; x is read at
// touched tokens only (the side of zero they are on).
template <typename T, bool GRAD, int THREADS, int K>
__global__ void __launch_bounds__(THREADS)
    logits_apply_kernel(const T *x, int64_t ld, const T *in, int64_t ld_in, T *out, int64_t ld_out, int V, int n_seg,
                        const __grid_constant__ hilore_logit_rules R)
{
    constexpr int N = Lane<T>::N, SEG = THREADS * K * N;
    extern __shared__ __align__(16) unsigned char smem[];
    const int64_t row = blockIdx.x / n_seg;
    const int f0 = (int)(blockIdx.x - row * n_seg) * SEG;
    const Row<T> src(in + row * ld_in, V);
    if (f0 >= src.end)
        return;
    const T *xrow = x + row * ld;
    T *orow = out + row * ld_out;
    Row<T> dst(orow, V);
    const bool vectors = dst.lead == src.lead;
    dst.origin = orow - src.lead; // the frame of the input; whole 32-byte stores only where both agree
    dst.lead = src.lead;
    dst.end = src.end;
    const Tables t = tables_at<SEG>(smem, R);
    const uint32_t *mask = row_mask(R, row);
    RowRules q = row_rules(R, row);
    q.bias = row_bias(R, row);
    clear_tables<SEG, THREADS>(t, R);
    fill_tables<SEG, THREADS>(R, row, mask, V, src.lead, f0, t);
#pragma unroll 1
    for (int k = 0; k < K; ++k) {
        const int s = (k * THREADS + threadIdx.x) * N, f = f0 + s;
        if (f >= src.end)
            break;
        const uint32_t b = vector_bits<N>(t.bits, s);
        const uint32_t deny = b >> 16, touch = b & 0xFFFFu;
        float z[N];
        if (deny == (1u << N) - 1u) { // nothing of this vector is read
#pragma unroll
            for (int i = 0; i < N; ++i)
                z[i] = GRAD ? 0.0f : -INFINITY;
        } else {
            uint32_t w[8];
            src.load(f, w);
            Lane<T>::unpack(w, z);
            if (touch) {
                const uint32_t ok = src.valid(f);
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (touch & ok & (1u << i)) {
                        uint32_t c, e;
                        take_entry(t, R, s + i, c, e);
                        z[i] = GRAD ? z[i] * slope_of(Lane<T>::one(xrow + (f + i - src.lead)), c, q) : adjusted(z[i], c, e, q);
                    }
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                z[i] *= q.inv_temp;
                if (deny & (1u << i)) z[i] = GRAD ? 0.0f : -INFINITY;
            }
        }
        dst.store(f, z, vectors);
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

constexpr int kLogpThreads = 256, kMaxRowCtas = 8;

// A row belongs to `row_ctas` CTAs (a thread-block cluster if more than one); each takes a share of its vectors.
template <typename T, bool TABLES, bool ENTROPY>
__global__ void __launch_bounds__(kLogpThreads)
    token_logp_kernel(const T *x, int64_t ld, int V, int row_ctas, const int32_t *targets, float *logp, float *lse, float *entropy,
                      const __grid_constant__ hilore_logit_rules R)
{
    constexpr int N = Lane<T>::N, K = 32 / N, SEG = kLogpThreads * K * N; // 8192 positions
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ Soft part[kLogpThreads / 32];
    __shared__ Soft shares[kMaxRowCtas];
    __shared__ float target_z; // the target's logit under penalties and bias; in the cluster's first CTA
    const int tid = threadIdx.x, lane = tid & 31;
    const int64_t row = blockIdx.x / row_ctas;
    const int rank = (int)(blockIdx.x - row * row_ctas);
    cg::cluster_group cl = cg::this_cluster();
    const int a = targets[row];
    if ((uint32_t)a >= (uint32_t)V) { // a slot without a token (the same for every CTA of the row)
        if (rank == 0 && tid == 0) {
            logp[row] = 0.0f;
            if (lse) lse[row] = 0.0f;
            if (ENTROPY) entropy[row] = 0.0f;
        }
        return;
    }
    if (rank == 0 && tid == 0) target_z = -INFINITY;
    if (row_ctas > 1)
        cl.sync(); // every CTA of the row runs, and target_z is set, before anything is sent to the first one
    else
        __syncthreads();
    float *first_z = row_ctas > 1 ? cl.map_shared_rank(&target_z, 0) : &target_z;

    const Row<T> src(x + row * ld, V);
    const int n_vec = (src.end + N - 1) / N;
    const int j_begin = (int)((int64_t)n_vec * rank / row_ctas), j_end = (int)((int64_t)n_vec * (rank + 1) / row_ctas);
    RowRules q = row_rules(R, row);
    const float c = kLog2eF * q.inv_temp;
    const int fa = a + src.lead;
    Soft acc{kLowest, 0.0f, 0.0f};
    if (!TABLES) {
        if (rank == 0 && tid == 0) target_z = Lane<T>::one(x + row * ld + a);
        for (int j0 = j_begin; j0 < j_end; j0 += kLogpThreads * K) {
            uint32_t w[K][8];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int j = j0 + k * kLogpThreads + tid;
                if (j < j_end) src.load(j * N, w[k]);
            }
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int j = j0 + k * kLogpThreads + tid;
                if (j < j_end) {
                    float z[N];
                    Lane<T>::unpack(w[k], z);
                    if (!src.whole(j * N)) {
                        const uint32_t ok = src.valid(j * N);
#pragma unroll
                        for (int i = 0; i < N; ++i)
                            if (!(ok >> i & 1u)) z[i] = -INFINITY;
                    }
                    soft_add<N, ENTROPY>(acc, z, c);
                }
            }
        }
    } else {
        const Tables t = tables_at<SEG>(smem, R);
        const uint32_t *mask = row_mask(R, row);
        q.bias = row_bias(R, row);
        clear_tables<SEG, kLogpThreads>(t, R);
        // segments start on multiples of 16 positions, as the words of the bit table do
        for (int f0 = j_begin * N & ~15; f0 < j_end * N; f0 += SEG) {
            fill_tables<SEG, kLogpThreads>(R, row, mask, V, src.lead, f0, t);
#pragma unroll 1
            for (int k = 0; k < K; ++k) {
                const int s = (k * kLogpThreads + tid) * N, f = f0 + s, j = f / N;
                const bool mine = j >= j_begin && j < j_end;
                if (f >= src.end)
                    continue;
                const uint32_t b = vector_bits<N>(t.bits, s);
                const uint32_t ok = src.valid(f), touch = b & ok, deny = (b >> 16) | ~ok;
                float z[N];
                const bool read = mine && (deny & ((1u << N) - 1u)) != (1u << N) - 1u;
                if (read) {
                    uint32_t w[8];
                    src.load(f, w);
                    Lane<T>::unpack(w, z);
                }
                if (touch) {
#pragma unroll
                    for (int i = 0; i < N; ++i)
                        if (touch & (1u << i)) {
                            uint32_t n, e;
                            take_entry(t, R, s + i, n, e);
                            if (read) z[i] = adjusted(z[i], n, e, q);
                        }
                }
                if (!read)
                    continue;
                if (deny & ((1u << N) - 1u)) {
#pragma unroll
                    for (int i = 0; i < N; ++i)
                        if (deny & (1u << i)) z[i] = -INFINITY;
                }
                if (j == fa / N) {
#pragma unroll
                    for (int i = 0; i < N; ++i)
                        if (i == fa % N) *first_z = z[i];
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

// grad_v = omega (1[v = a] - exp(z_v - lse)) dz_v/dx_v.  One CTA per (row, segment); rows whose coefficient is zero, that
// have no token, whose token the grammar denies or that had nothing to choose from get zeros without being read.
template <typename T, bool TABLES, int THREADS, int K>
__global__ void __launch_bounds__(THREADS)
    token_logp_backward_kernel(const T *x, int64_t ld, int V, int n_seg, const int32_t *targets, const float *lse, const float *omega,
                               T *grad, int64_t ld_grad, const __grid_constant__ hilore_logit_rules R)
{
    constexpr int N = Lane<T>::N, SEG = THREADS * K * N;
    extern __shared__ __align__(16) unsigned char smem[];
    const int64_t row = blockIdx.x / n_seg;
    const int f0 = (int)(blockIdx.x - row * n_seg) * SEG;
    const Row<T> src(x + row * ld, V);
    if (f0 >= src.end)
        return;
    Row<T> dst(grad + row * ld_grad, V);
    const bool vectors = dst.lead == src.lead;
    dst.origin = grad + row * ld_grad - src.lead;
    dst.lead = src.lead;
    dst.end = src.end;
    const int a = targets[row];
    const float om = omega[row], l = lse[row];
    const uint32_t *mask = row_mask(R, row);
    bool live = (uint32_t)a < (uint32_t)V && om != 0.0f && !(l <= kNothing);
    if (live && mask != nullptr) live = (__ldg(mask + (a >> 5)) >> (a & 31)) & 1u;
    const int fa = a + src.lead;
    if (!live) {
        const float zero[N] = {};
#pragma unroll 1
        for (int k = 0; k < K; ++k) {
            const int f = f0 + (k * THREADS + threadIdx.x) * N;
            if (f < src.end) dst.store(f, zero, vectors);
        }
        return;
    }
    RowRules q = row_rules(R, row);
    const Tables t = tables_at<SEG>(smem, R);
    if (TABLES) {
        q.bias = row_bias(R, row);
        clear_tables<SEG, THREADS>(t, R);
        fill_tables<SEG, THREADS>(R, row, mask, V, src.lead, f0, t);
    }
    const float scale = om * q.inv_temp;
#pragma unroll 1
    for (int k = 0; k < K; ++k) {
        const int s = (k * THREADS + threadIdx.x) * N, f = f0 + s;
        if (f >= src.end)
            break;
        const uint32_t b = TABLES ? vector_bits<N>(t.bits, s) : 0u;
        const uint32_t deny = b >> 16, touch = b & 0xFFFFu;
        float z[N];
        if (deny == (1u << N) - 1u) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                z[i] = 0.0f;
        } else {
            uint32_t w[8];
            src.load(f, w);
            Lane<T>::unpack(w, z);
            float slope[N];
            if (TABLES) {
#pragma unroll
                for (int i = 0; i < N; ++i)
                    slope[i] = 1.0f;
                if (touch) {
                    const uint32_t ok = src.valid(f);
#pragma unroll
                    for (int i = 0; i < N; ++i)
                        if (touch & ok & (1u << i)) {
                            uint32_t n, e;
                            take_entry(t, R, s + i, n, e);
                            slope[i] = slope_of(z[i], n, q);
                            z[i] = adjusted(z[i], n, e, q);
                        }
                }
            }
            const int at = fa - f; // the target's place in this vector, if it is in it
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float p = ex2_ftz(fmaf(z[i], q.inv_temp, -l) * kLog2eF);
                float g = (i == at ? 1.0f - p : -p) * scale;
                if (TABLES) {
                    g *= slope[i];
                    if (deny & (1u << i)) g = 0.0f;
                }
                z[i] = g;
            }
        }
        dst.store(f, z, vectors);
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

static bool needs_tables(const hilore_logit_rules &q) { return q.tokens || q.bias_tokens || q.allow; }

template <typename K> static bool allow_smem(K kernel, size_t bytes)
{
    return bytes <= 48 * 1024 || cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == cudaSuccess;
}

template <typename T, bool GRAD>
static int launch_apply(const T *x, int64_t ld, const T *in, int64_t ld_in, T *out, int64_t ld_out, int64_t n_rows, int64_t V,
                        const hilore_logit_rules &R, cudaStream_t st)
{
    constexpr int N = Lane<T>::N, THREADS = 256, K = 32 / N, SEG = THREADS * K * N;
    const int64_t n_seg = (V + N - 1 + SEG - 1) / SEG;
    if (n_seg * n_rows > 0x7FFFFFFF)
        return HILORE_SHAPE;
    auto kernel = logits_apply_kernel<T, GRAD, THREADS, K>;
    const size_t smem = tables_bytes<SEG>(R);
    if (!allow_smem(kernel, smem))
        return HILORE_CUDA;
    kernel<<<(unsigned)(n_seg * n_rows), THREADS, smem, st>>>(x, ld, in, ld_in, out, ld_out, (int)V, (int)n_seg, R);
    return cudaGetLastError() == cudaSuccess ? HILORE_OK : HILORE_CUDA;
}

static bool clusters_on()
{
    const char *off = std::getenv("HILORE_DISABLE_CLUSTER_LAUNCH");
    return off == nullptr || off[0] == '\0' || (off[0] == '0' && off[1] == '\0');
}

template <typename T, bool TABLES, bool ENTROPY>
static int launch_logp(const T *x, int64_t ld, int64_t n_rows, int64_t V, const int32_t *targets, float *logp, float *lse, float *entropy,
                       const hilore_logit_rules &R, cudaStream_t st)
{
    auto kernel = token_logp_kernel<T, TABLES, ENTROPY>;
    const size_t smem = TABLES ? tables_bytes<8192>(R) : 0;
    if (!allow_smem(kernel, smem))
        return HILORE_CUDA;
    // CTAs per row: as many as keep the SMs busy with two each, at most a portable cluster, none with less than 2048 logits
    int row_ctas = 1;
    if (clusters_on())
        while (row_ctas < kMaxRowCtas && n_rows * row_ctas < 2 * (int64_t)sm_count() && V / (2 * row_ctas) >= 2048)
            row_ctas *= 2;
    if (n_rows * row_ctas > 0x7FFFFFFF)
        return HILORE_SHAPE;
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

template <typename T, bool TABLES>
static int launch_logp_backward(const T *x, int64_t ld, int64_t n_rows, int64_t V, const int32_t *targets, const float *lse, const float *omega,
                                T *grad, int64_t ld_grad, const hilore_logit_rules &R, cudaStream_t st)
{
    constexpr int N = Lane<T>::N, THREADS = 256, K = 32 / N, SEG = THREADS * K * N;
    const int64_t n_seg = (V + N - 1 + SEG - 1) / SEG;
    if (n_seg * n_rows > 0x7FFFFFFF)
        return HILORE_SHAPE;
    auto kernel = token_logp_backward_kernel<T, TABLES, THREADS, K>;
    const size_t smem = TABLES ? tables_bytes<SEG>(R) : 0;
    if (!allow_smem(kernel, smem))
        return HILORE_CUDA;
    kernel<<<(unsigned)(n_seg * n_rows), THREADS, smem, st>>>(x, ld, (int)V, (int)n_seg, targets, lse, omega, grad, ld_grad, R);
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
    if (needs_tables(R))                                                                                                                        \
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
    return needs_tables(R) ? launch_logp_backward<T, true>(p, ld, n_rows, V, targets, lse, omega, g, ld_grad, R, st)                            \
                           : launch_logp_backward<T, false>(p, ld, n_rows, V, targets, lse, omega, g, ld_grad, R, st)
    if (dtype == HILORE_BF16) { HILORE_PICK(uint16_t); }
    HILORE_PICK(float);
#undef HILORE_PICK
}
