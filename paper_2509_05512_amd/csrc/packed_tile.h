// Device helpers shared by the kernels of packed sequences (gfx950): blocks of 128
// tokens and the sequences that they belong to.
#pragma once

#include <hip/hip_runtime.h>

#include "cache_tile.h"

namespace quan {
namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves, kBlock = 32 * kWaves;  // a wave per 32 tokens of a block

// A block of a sequence's tokens; at >= len: none.
struct Block {
    int seq, at;
};

// Block `id` of packed_blocks(): those of sequence i are the first of numbers
// first[i] / 128 + i ..; the next sequence's begin (first[i + 1] - first[i]) / 128
// + 1 later at least, and it has no more blocks.  Numbers that are none of a
// sequence's blocks are idle.  The sequences are counted that begin at or below
// `id`, which the host does not have to know.
__device__ __forceinline__ Block locate(const Sequences &s, int id, int *lds)
{
    if (s.first == nullptr) {
        const int per = (s.tokens + kBlock - 1) / kBlock, seq = id / per;
        return {seq, (id - seq * per) * kBlock};
    }
    int below = 0;
    for (int i0 = 0; i0 < s.count; i0 += kThreads) {
        const int i = i0 + threadIdx.x;
        below += __popcll(__ballot(i < s.count && min(max(s.first[min(i, s.count - 1)], 0), s.tokens) / kBlock + i <= id));
    }
    if ((threadIdx.x & 63) == 0)
        lds[threadIdx.x >> 6] = below;
    __syncthreads();
    int seq = -1;
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
        seq += lds[w];
    if (seq < 0)
        return {0, s.tokens};
    // (out of order, a sequence may be counted before its own number)
    const int block = id - (min(max(s.first[seq], 0), s.tokens) / kBlock + seq);
    return {seq, block < 0 || block > s.tokens / kBlock ? s.tokens : block * kBlock};
}

// A block's walk over `mine` tiles, dealt out to work-groups: `count` of them take
// `per` tiles each, the last the rest, where the sequence's longest walk has `longest`
// tiles and `splits` work-groups, so that all take about as many.  (Two tiles at
// least.)
struct Walk {
    int per, count;
};
__device__ __forceinline__ Walk walk_of(int longest, int mine, int splits)
{
    const int per = max(2, (longest + splits - 1) / splits);
    return {per, max(1, (mine + per - 1) / per)};
}

// Infinities and NaN in rows of a tile that not all of the work-group's lanes see:
// a product's masked factor 0 would make NaN of them.  Such rows (rare, and looked
// for in the tiles at a walk's edge alone) are zeroed on their way to LDS and added
// one by one to the lanes that see them, from memory.
template <typename F> __device__ __forceinline__ bool any_not_finite(const F &v)
{
    const f32x8 t = to_f32(v);
    unsigned top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        top = max(top, __float_as_uint(t[e]) & 0x7fffffffu);
    return top >= 0x7f800000u;
}
// Zeros this thread's chunks of the rows that are not finite in a or b (which may
// be the same); flags[row]: whether the row was.
template <typename Tile> __device__ __forceinline__ void zero_not_finite(Tile &a, Tile &b, int *flags)
{
    constexpr int kChunks = Tile::kChunks;
    const int row = threadIdx.x / kChunks, lane = threadIdx.x & 63;
    if (Tile::kStep > Tile::kTokens && row >= Tile::kTokens)
        return;
#pragma unroll
    for (int i = 0; i < Tile::kCount; ++i) {
        const bool bad = any_not_finite(a.r[i]) || (&a != &b && any_not_finite(b.r[i]));
        const bool zero = __ballot(bad) >> (lane & ~(kChunks - 1)) & ((1ull << kChunks) - 1);
        if (zero) {
            a.r[i] = typename Tile::frag{};
            b.r[i] = typename Tile::frag{};
        }
        if (threadIdx.x % kChunks == 0)
            flags[row + i * Tile::kStep] = zero;
    }
}
// The rows of a tile that zero_not_finite() has flagged, one bit each.
__device__ __forceinline__ unsigned long long flagged(const int *flags, int rows)
{
    const int lane = threadIdx.x & 63;
    return __ballot(lane < rows && flags[min(lane, rows - 1)] != 0);
}
// 0 in the accumulators of part `sub` that belong to flagged rows.
template <int TOKENS> __device__ __forceinline__ void clear_flagged(f32x16 &s, unsigned long long rows, int sub)
{
    const unsigned mine = unsigned(rows >> (TOKENS / 2 * ((threadIdx.x & 63) >> 5) + 16 * sub));
#pragma unroll
    for (int r = 0; r < 16; ++r)
        s[r] = mine >> r & 1 ? 0.0f : s[r];
}
// A row's inner product with the row that the lane and its partner hold.
template <typename T, int DQP>
__device__ __forceinline__ float row_dot(const WholeMap<T, DQP> &m, int64_t token, const typename Elem<T>::frag (&x)[DQP / 4])
{
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < DQP / 4; ++i) {
        const f32x8 a = to_f32(m.load(token, 16 * i + 8 * ((threadIdx.x & 63) >> 5), true)), b = to_f32(x[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            s = fmaf(a[e], b[e], s);
    }
    return half_sum(s);
}
// A row times `by`, added to the accumulators of the lanes that see it.
template <typename T, int DQP>
__device__ __forceinline__ void row_add(f32x16 (&acc)[DQP / 8], const WholeMap<T, DQP> &m, int64_t token, float by, bool sees)
{
#pragma unroll
    for (int i = 0; i < DQP / 8; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const T *p = m.at(token, 32 * i + 8 * g + 4 * ((threadIdx.x & 63) >> 5));
#pragma unroll
            for (int t = 0; t < 4; ++t)
                acc[i][4 * g + t] = sees ? fmaf(by, float(p[t]), acc[i][4 * g + t]) : acc[i][4 * g + t];
        }
}

// A D x 32 tile of accumulators, transposed, to a row of fp32.
template <int DP> __device__ __forceinline__ void store_part(float *dst, const f32x16 (&v)[DP / 32], bool here)
{
    if (!here)
        return;
#pragma unroll
    for (int i = 0; i < DP / 32; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const f32x4 t = {v[i][4 * g], v[i][4 * g + 1], v[i][4 * g + 2], v[i][4 * g + 3]};
            *reinterpret_cast<f32x4 *>(dst + 32 * i + 8 * g + 4 * ((threadIdx.x & 63) >> 5)) = t;
        }
}

// Work-groups of a launch that joins: each takes 1024 / D rows of a block.
constexpr int join_groups(int dp) { return kBlock * dp / 1024; }

}  // namespace
}  // namespace quan
