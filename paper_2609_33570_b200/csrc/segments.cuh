// Tokens of back-to-back sequences in tiles of 2048: which sequences a tile holds, where they end, and scans over a tile's
// tokens that start anew at every sequence.  Shared by the kernels of objective.cu.
#pragma once

#include <initializer_list>

#include "common.cuh"

namespace hilore {

constexpr int kSegThreads = 256;             // threads of a CTA
constexpr int kSegEach = 8;                  // consecutive tokens of a thread: one 256-bit access per fp32 tensor
constexpr int kSegTile = kSegThreads * kSegEach;
constexpr int kSegWarps = kSegThreads / 32;

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
            return (int)(p / T);
        while (first < last) {
            const int mid = first + (last - first + 1) / 2;
            if (bound(mid) <= p) first = mid;
            else last = mid - 1;
        }
        return first;
    }

    // The same over all sequences by a whole warp: 32 probes at a time.
    __device__ __forceinline__ int owner_warp(int p, int lane) const
    {
        if (cu == nullptr)
            return (int)(p / T);
        int64_t first = 0, count = n_seq; // the answer lies in [first, first + count)
        while (count > 1) {
            const int64_t step = (count + 31) / 32, at = first + lane * step;
            const bool le = lane == 0 || (at < first + count && bound((int)at) <= p);
            const uint32_t hit = __ballot_sync(0xFFFFFFFFu, le);
            // the leading run of hits: with boundaries in order that is every hit
            const int k = __ffs(~hit) == 0 ? 31 : __ffs(~hit) - 2;
            const int64_t begin = first + k * step;
            count = (first + count - begin) < step ? (first + count - begin) : step;
            first = begin;
        }
        return (int)first;
    }
};

// What a CTA knows of its tile: tokens [lo, hi), sequences s0 .. s1 of them, and a bit for every token that ends its sequence.
struct TileShared {
    uint32_t ends[kSegTile / 32];
    int s0, s1;
};

// All threads; `hi` > `lo`.  Ends with a barrier; a barrier must lie between a tile's last use of `sh` and the next call.
__device__ __forceinline__ void tile_sequences(const Sequences &q, int lo, int hi, TileShared &sh)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid < kSegTile / 32)
        sh.ends[tid] = 0;
    if (warp == 2 || warp == 3) { // the first and the last sequence at the same time
        const int s = q.owner_warp(warp == 2 ? lo : hi - 1, lane);
        if (lane == 0) {
            if (warp == 2) sh.s0 = s;
            else sh.s1 = s;
        }
    }
    __syncthreads();
    for (int s = sh.s0 + tid; s <= sh.s1; s += kSegThreads) {
        const int e = q.bound(s + 1) - 1 - lo;
        if (e >= 0 && e < hi - lo)
            atomicOr(&sh.ends[e >> 5], 1u << (e & 31));
    }
    __syncthreads();
}

// The end bits of the eight tokens of block `b` (0 .. 255) of the tile.
__device__ __forceinline__ uint32_t block_ends(const TileShared &sh, int b) { return (sh.ends[b >> 2] >> (8 * (b & 3))) & 0xFFu; }

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

__device__ __forceinline__ void load8(const uint16_t *p, int k, int hi, bool vec, float (&x)[8]) // bf16
{
    if (vec && k + 8 <= hi) {
        const uint4 w = ld_global_128_stream(p + k);
        const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[2 * e] = bf16_lo(v[e]);
            x[2 * e + 1] = bf16_hi(v[e]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = k + e < hi ? __uint_as_float((uint32_t)p[k + e] << 16) : 0.0f;
    }
}

__device__ __forceinline__ uint32_t load_mask8(const uint8_t *p, int k, int hi, bool vec)
{
    const int n = hi - k;
    if (n <= 0)
        return 0;
    if (p == nullptr)
        return n >= 8 ? 0xFFu : (1u << n) - 1;
    uint32_t m = 0;
    if (vec && n >= 8) {
        const uint2 w = ld_global_64_stream(p + k);
        // every byte that is not zero to 0xFF, then the top bits gathered
        const uint32_t a = __vcmpne4(w.x, 0u) & 0x08040201u, b = __vcmpne4(w.y, 0u) & 0x80402010u;
        m = ((a | b) * 0x01010101u) >> 24;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n && p[k + e] != 0) m |= 1u << e;
    }
    return m;
}

__device__ __forceinline__ void store8(float *p, int k, int hi, bool vec, const float (&x)[8])
{
    if (vec && k + 8 <= hi) {
        uint32_t w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = __float_as_uint(x[e]);
        st_global_256(p + k, w);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (k + e < hi) p[k + e] = x[e];
    }
}

// ---- scans over the threads of a CTA ----
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
constexpr int64_t kMaxTokens = (int64_t(1) << 31) - (int64_t(1) << 16); // token numbers of a whole tile stay in 31 bits

// The sequences and tiles of a call, or why there are none.
inline int check_sequences(const int32_t *cu, int64_t n_seq, int64_t n_tok, Sequences &q, int &tiles)
{
    if (n_seq < 0 || n_tok < 0)
        return HILORE_INVALID_ARG;
    if (n_seq > kMaxTokens || n_tok > kMaxTokens || (n_seq == 0 && n_tok > 0) || (!cu && n_seq > 0 && n_tok % n_seq != 0))
        return HILORE_SHAPE;
    if (!aligned(cu, 4))
        return HILORE_ALIGN;
    q = Sequences{cu, n_seq, n_tok, n_seq > 0 ? n_tok / n_seq : 0};
    tiles = (int)((n_tok + kSegTile - 1) / kSegTile);
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
