// Tokens of back-to-back sequences: where sequences lie, accesses of eight neighbouring tokens a lane and of blocks of 256 a warp, masks,
// and scans over the lanes of a warp.  Shared by advantages.cu and objective.cu.
#pragma once

#include <initializer_list>

#include "common.cuh"

namespace hilore {

// The sequences of a call: packed with their boundaries, or rows of T slots (cu == nullptr).  Whatever `cu` holds, boundaries
// lie in [0, n_tok]; tokens from bound(n_seq) on belong to no sequence.
struct Sequences {
    const int32_t *cu;
    int64_t n_seq, n_tok, T;

    __device__ __forceinline__ int bound(int s) const // s in [0, n_seq]
    {
        if (cu == nullptr)
            return (int)((int64_t)s * T);
        if (s == 0)
            return 0;
        const int64_t b = __ldg(cu + s);
        return (int)(b < 0 ? 0 : (b > n_tok ? n_tok : b));
    }
    __device__ __forceinline__ int live() const { return bound((int)n_seq); }

    // The sequence in [first, last] that holds token p: the last one that begins at or before it.
    __device__ __forceinline__ int owner(int p, int first, int last) const
    {
        if (cu == nullptr)
            return (int)((uint32_t)p / (uint32_t)T);
        while (first < last) {
            const int mid = first + (last - first + 1) / 2;
            if (bound(mid) <= p) first = mid;
            else last = mid - 1;
        }
        return first;
    }

    // The same over all sequences, of two tokens at once, by a whole warp: 32 probes for each at a time.
    __device__ __forceinline__ void owner_warp2(int p0, int p1, int lane, int &s0, int &s1) const
    {
        if (cu == nullptr) {
            s0 = (int)((uint32_t)p0 / (uint32_t)T);
            s1 = (int)((uint32_t)p1 / (uint32_t)T);
            return;
        }
        // the answers lie in [f0, f0 + count) and [f1, f1 + count), as far as these are in [0, n_seq)
        int64_t f0 = 0, f1 = 0, count = n_seq;
        while (count > 1) {
            const int64_t step = (count + 31) / 32, a0 = f0 + lane * step, a1 = f1 + lane * step;
            const int b0 = lane * step < count && a0 < n_seq ? bound((int)a0) : 0x7FFFFFFF;
            const int b1 = lane * step < count && a1 < n_seq ? bound((int)a1) : 0x7FFFFFFF;
            const uint32_t h0 = ~__ballot_sync(0xFFFFFFFFu, lane == 0 || b0 <= p0), h1 = ~__ballot_sync(0xFFFFFFFFu, lane == 0 || b1 <= p1);
            // the leading run of hits: with boundaries in order that is every hit
            f0 += (h0 ? __ffs(h0) - 2 : 31) * step;
            f1 += (h1 ? __ffs(h1) - 2 : 31) * step;
            count = step;
        }
        s0 = (int)f0;
        s1 = (int)f1;
    }
    __device__ __forceinline__ int owner_warp(int p, int lane) const
    {
        int s0, s1;
        owner_warp2(p, p, lane, s0, s1);
        return s0;
    }
};

// ---- a thread's eight tokens, from token k on; those at or beyond `hi` count as masked and read as zero ----
__device__ __forceinline__ void load8(const float *p, int k, int hi, bool vec, float (&x)[8])
{
    if (vec && k + 8 <= hi) {
        uint32_t w[8];
        ld_global_256(p + k, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(w[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = k + e < hi ? p[k + e] : 0.0f;
    }
}

// A bit for each of eight bytes that is not zero.
__device__ __forceinline__ uint32_t mask_bits(uint2 w)
{
    // the top bit of every byte that is not zero; these, 8 apart, gathered in four neighbouring bits
    const uint32_t a = (((w.x & 0x7F7F7F7Fu) + 0x7F7F7F7Fu) | w.x) & 0x80808080u, b = (((w.y & 0x7F7F7F7Fu) + 0x7F7F7F7Fu) | w.y) & 0x80808080u;
    return (a * 0x00204081u) >> 28 | ((b * 0x00204081u) >> 28) << 4;
}

__device__ __forceinline__ void zero8(float (&x)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = 0.0f;
}

__device__ __forceinline__ void store8(float *p, const float (&x)[8])
{
    uint32_t w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = __float_as_uint(x[e]);
    st_global_256(p, w);
}

// Those of the eight tokens that lie in [lo, hi).
__device__ __forceinline__ void store8(float *p, int k, int lo, int hi, bool vec, const float (&x)[8])
{
    if (vec && k >= lo && k + 8 <= hi) {
        uint32_t w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = __float_as_uint(x[e]);
        st_global_256(p + k, w);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (k + e >= lo && k + e < hi) p[k + e] = x[e];
    }
}

// ---- blocks of 256 tokens on their way through shared memory ----
// cp.async holds no registers while the data is on its way, so a warp can have several blocks in flight.  Every instruction copies
// 512 neighbouring bytes (sixteen bytes of every thirty-two would ask L2 for each sector twice), so lanes read what others asked
// for.  Pieces of four numbers are swapped in pairs in every other row of eight, which lets lanes read their two without conflicts.
constexpr int kBlock = 256;
struct Stage {
    float4 x[kBlock / 4];
};
__device__ __forceinline__ int swapped(int c) { return c ^ (c >> 3 & 1); }
__device__ __forceinline__ void copy_async(void *to, const void *from, int bytes) // 4, 8 or 16
{
    const uint32_t d = (uint32_t)__cvta_generic_to_shared(to);
    if (bytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(d), "l"(from) : "memory");
    else if (bytes == 8) asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(d), "l"(from) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(d), "l"(from) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

// Tokens base .. base + 255, those in [0, n).  whole: all of them, at an address that moves eight at a time.
__device__ __forceinline__ void fetch_block(Stage &to, int lane, const float *p, int base, int n, bool whole)
{
    if (whole) {
#pragma unroll
        for (int j = 0; j < 2; ++j) copy_async(&to.x[swapped(32 * j + lane)], p + base + 128 * j + 4 * lane, 16);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int t = 32 * j + lane;
            if (base + t < n) copy_async(reinterpret_cast<float *>(&to.x[swapped(t >> 2)]) + (t & 3), p + base + t, 4);
        }
    }
}
__device__ __forceinline__ void fetch_block(Stage &to, int lane, const uint16_t *p, int base, int n, bool whole) // bf16
{
    if (whole) {
        copy_async(&to.x[lane], p + base + 8 * lane, 16);
    } else {
        uint16_t *h = reinterpret_cast<uint16_t *>(to.x);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int t = 32 * j + lane;
            if (base + t < n) h[t] = p[base + t];
        }
    }
}
// Tokens 8 at .. 8 at + 7 of the block.
__device__ __forceinline__ void read8(const Stage &from, int at, float (&x)[8])
{
    const float4 a = from.x[swapped(2 * at)], b = from.x[swapped(2 * at + 1)];
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}
__device__ __forceinline__ void read8_bf16(const Stage &from, int at, float (&x)[8])
{
    const float4 w = from.x[at];
    const uint32_t v[4] = {__float_as_uint(w.x), __float_as_uint(w.y), __float_as_uint(w.z), __float_as_uint(w.w)};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[2 * e] = bf16_lo(v[e]);
        x[2 * e + 1] = bf16_hi(v[e]);
    }
}

// The eight mask bytes from token k on, those at or behind n as zeros.
__device__ __forceinline__ uint2 mask_bytes(const uint8_t *p, int k, int n)
{
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (k + e < n) w[e >> 2] |= (uint32_t)p[k + e] << (8 * (e & 3));
    return make_uint2(w[0], w[1]);
}
// The mask of eight tokens in two steps: read, and, a while later, made bits, since nothing that follows in a warp's program starts before
// the first step that needs what has been read.
struct Mask8 {
    uint2 bytes;
    __device__ __forceinline__ void read(const uint8_t *p, int k, int hi, bool vec)
    {
        bytes = make_uint2(0u, 0u);
        if (k >= hi) return;
        if (p == nullptr) bytes = make_uint2(0x01010101u, 0x01010101u);
        else if (vec && k + 8 <= hi) bytes = ld_global_64_stream(p + k);
        else bytes = mask_bytes(p, k, hi);
    }
    __device__ __forceinline__ uint32_t bits(int k, int hi) const
    {
        const uint32_t v = mask_bits(bytes);
        return k + 8 <= hi ? v : (k < hi ? v & ((1u << (hi - k)) - 1) : 0u);
    }
};

// Bits of the tokens k .. k + 7 that lie in [lo, hi).
__device__ __forceinline__ uint32_t range_bits(int k, int lo, int hi)
{
    if (k >= lo && k + 8 <= hi) return 0xFFu;
    if (k + 8 <= lo || k >= hi) return 0u;
    const uint32_t from = k < lo ? 0xFFu << (lo - k) : 0xFFu, to = k + 8 > hi ? 0xFFu >> (k + 8 - hi) : 0xFFu;
    return from & to & 0xFFu;
}

// yes ? a : b with both worked out, where the compiler would make a branch of it.
__device__ __forceinline__ double pick(bool yes, double a, double b)
{
    double r;
    asm("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %3, 0;\n\tselp.f64 %0, %1, %2, p;\n\t}" : "=d"(r) : "d"(a), "d"(b), "r"((uint32_t)yes));
    return r;
}

// ---- scans over the lanes of a warp ----
// Op::Map is what a run of tokens does to the state that comes in; Op::then(a, b) is a followed by b, Op::apply(m, s) the state
// behind the run.  A run that holds the start of a sequence does not depend on what comes in, and says so in its flag.
template <typename T> __device__ __forceinline__ T shfl_up_words(const T &v, int by)
{
    static_assert(sizeof(T) % 4 == 0, "whole words");
    T r;
    const uint32_t *a = reinterpret_cast<const uint32_t *>(&v);
    uint32_t *b = reinterpret_cast<uint32_t *>(&r);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 4); ++i) b[i] = __shfl_up_sync(0xFFFFFFFFu, a[i], by);
    return r;
}

template <typename T> __device__ __forceinline__ T shfl_words(const T &v, int from)
{
    T r;
    const uint32_t *a = reinterpret_cast<const uint32_t *>(&v);
    uint32_t *b = reinterpret_cast<uint32_t *>(&r);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 4); ++i) b[i] = __shfl_sync(0xFFFFFFFFu, a[i], from);
    return r;
}

// The map of the lanes before this one, and in `all` (last lane) that of the warp.
template <typename Op> __device__ __forceinline__ typename Op::Map warp_scan(typename Op::Map mine, int lane, typename Op::Map &all)
{
#pragma unroll
    for (int by = 1; by < 32; by *= 2) {
        const typename Op::Map before = shfl_up_words(mine, by);
        if (lane >= by) mine = Op::then(before, mine);
    }
    all = mine;
    const typename Op::Map before = shfl_up_words(mine, 1);
    return lane == 0 ? Op::identity() : before;
}

// ---- host side ----
constexpr int64_t kMaxTokens = (int64_t(1) << 31) - (int64_t(1) << 16); // token numbers some blocks behind the last stay in 31 bits

// The sequences of a call, or why there are none.
inline int check_sequences(const int32_t *cu, int64_t n_seq, int64_t n_tok, Sequences &q)
{
    if (n_seq < 0 || n_tok < 0)
        return HILORE_INVALID_ARG;
    if (n_seq > kMaxTokens || n_tok > kMaxTokens || (n_seq == 0 && n_tok > 0) || (!cu && n_seq > 0 && n_tok % n_seq != 0))
        return HILORE_SHAPE;
    if (!aligned(cu, 4))
        return HILORE_ALIGN;
    q = Sequences{cu, n_seq, n_tok, n_seq > 0 ? n_tok / n_seq : 0};
    return HILORE_OK;
}

// Whether tokens can move eight at a time.
inline bool vectors(std::initializer_list<const float *> tensors, const uint8_t *mask)
{
    for (const float *p : tensors)
        if (!aligned(p, 32)) return false;
    return aligned(mask, 8);
}

} // namespace hilore
