// Device helpers shared by the kernels of packed sequences (gfx950): blocks of 128
// tokens and the sequences that they belong to.
#pragma once

#include <hip/hip_runtime.h>

#include "cache_tile.h"

namespace quan {
namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kBlock = 32 * kWaves;  // tokens of a block: 32 to a wave (or in blocks twice as large 64)

// A block of a sequence's tokens; at >= len: none.
struct Block {
    int seq, at;
};

// Block `id` of packed_blocks(), of `size` tokens: those of sequence i are the first
// of numbers first[i] / size + i ..; the next sequence's begin (first[i + 1] -
// first[i]) / size + 1 later at least, and it has no more blocks.  Numbers that are none of a
// sequence's blocks are idle.  The sequences are counted that begin at or below
// `id`, which the host does not have to know.
template <int SIZE = kBlock> __device__ __forceinline__ Block locate(const Sequences &s, int id, int *lds)
{
    if (s.first == nullptr) {
        const int per = (s.tokens + SIZE - 1) / SIZE, seq = id / per;
        return {seq, (id - seq * per) * SIZE};
    }
    int below = 0;
    for (int i0 = 0; i0 < s.count; i0 += kThreads) {
        const int i = i0 + threadIdx.x;
        below += __popcll(__ballot(i < s.count && min(max(s.first[min(i, s.count - 1)], 0), s.tokens) / SIZE + i <= id));
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
    const int block = id - (min(max(s.first[seq], 0), s.tokens) / SIZE + seq);
    return {seq, block < 0 || block > s.tokens / SIZE ? s.tokens : block * SIZE};
}

// Sum and maximum over a wave.
__device__ __forceinline__ int wave_sum(int x)
{
#define QUAN_DPP(v, ctrl) __builtin_amdgcn_update_dpp(0, v, ctrl, 0xf, 0xf, false)
    x += QUAN_DPP(x, 0xB1);   // lane ^ 1
    x += QUAN_DPP(x, 0x4E);   // lane ^ 2
    x += QUAN_DPP(x, 0x141);  // 7 - lane of 8
    x += QUAN_DPP(x, 0x140);  // 15 - lane of 16
    const auto a = __builtin_amdgcn_permlane16_swap(unsigned(x), unsigned(x), false, false);
    x = int(a[0] + a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(unsigned(x), unsigned(x), false, false);
    return __builtin_amdgcn_readfirstlane(int(b[0] + b[1]));
}
__device__ __forceinline__ int wave_max(int x)
{
    x = max(x, QUAN_DPP(x, 0xB1));
    x = max(x, QUAN_DPP(x, 0x4E));
    x = max(x, QUAN_DPP(x, 0x141));
    x = max(x, QUAN_DPP(x, 0x140));
#undef QUAN_DPP
    const auto a = __builtin_amdgcn_permlane16_swap(unsigned(x), unsigned(x), false, false);
    x = max(int(a[0]), int(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(unsigned(x), unsigned(x), false, false);
    return __builtin_amdgcn_readfirstlane(max(int(b[0]), int(b[1])));
}

// The blocks in an order that begins with the longest walks: of 64 sequences at a
// time, first the blocks that are `level` from their sequence's one end, then those
// that are one less, down to 0 (whose walks are the shortest).  at is SIZE * level,
// or with from_end the block that many before the last.
template <int SIZE> __device__ __forceinline__ Block locate_longest(const Sequences &s, int id, bool from_end)
{
    const int lane = threadIdx.x & 63;
    if (s.first == nullptr) {
        const int per = (s.tokens + SIZE - 1) / SIZE, down = id / s.count;  // (equal lengths)
        return {id - down * s.count, (from_end ? down : per - 1 - down) * SIZE};
    }
    // the 64 sequences, counted as in locate()
    int set = 0;
    for (int i0 = 0; i0 + 64 < s.count; i0 += 64 * 64) {
        const int i = i0 + 64 * lane + 64;
        set += __popcll(__ballot(i < s.count && min(max(s.first[min(i, s.count)], 0), s.tokens) / SIZE + i <= id));
    }
    set *= 64;
    const int at0 = min(max(s.first[set], 0), s.tokens), rank = id - (at0 / SIZE + set);
    const int seq = min(set + lane, s.count - 1);
    const int a = min(max(s.first[seq], 0), s.tokens), len = min(max(s.first[seq + 1], a), s.tokens) - a;
    const int blocks = set + lane < s.count ? (len + SIZE - 1) / SIZE : 0;
    // the largest level with more than `rank` blocks at or above it
    int low = 0, high = wave_max(blocks);
    if (rank < 0 || rank >= wave_sum(blocks))
        return {0, s.tokens};
    while (high - low > 1) {
        const int mid = (low + high) >> 1;
        if (wave_sum(max(0, blocks - mid)) > rank)
            low = mid;
        else
            high = mid;
    }
    const int skip = rank - wave_sum(max(0, blocks - low - 1));
    const auto here = __ballot(blocks > low);
    const auto mine = __ballot(blocks > low && __popcll(here & ((1ull << lane) - 1)) == skip);
    const int l = mine != 0 ? __builtin_ctzll(mine) : 0;
    const int of = __builtin_amdgcn_readlane(blocks, l);
    return {min(set + l, s.count - 1), (from_end ? of - 1 - low : low) * SIZE};
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
// a product's masked factor 0 would make NaN of them.  Tiles at a walk's edge, and
// they alone, are looked over as they are staged; one with such a row (rare) is left
// out of the walk and taken row by row after it, from memory.
template <typename F> __device__ __forceinline__ bool not_finite(const F &v)
{
    const f32x8 t = to_f32(v);
    unsigned top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        top = max(top, __float_as_uint(t[e]) & 0x7fffffffu);
    return top >= 0x7f800000u;
}
// Whether this thread's chunks of a tile have one; to flags[wave].
template <typename Tile> __device__ __forceinline__ bool staged_not_finite(const Tile &t)
{
    bool bad = false;
#pragma unroll
    for (int i = 0; i < Tile::kCount; ++i)
        bad = bad || not_finite(t.r[i]);
    return bad;
}
__device__ __forceinline__ void flag_wave(int *flags, bool bad)
{
    const bool any = __ballot(bad) != 0;
    if ((threadIdx.x & 63) == 0)
        flags[threadIdx.x >> 6] = any;
}
template <int WAVES> __device__ __forceinline__ bool flagged(const int *flags)
{
    int any = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w)
        any |= flags[w];
    return __builtin_amdgcn_readfirstlane(any) != 0;
}
// Whether tokens [token, end) of a map's tile have one: the same for every wave.
template <typename T, int DQP> __device__ __forceinline__ bool rows_not_finite(const WholeMap<T, DQP> &m, int token, int end)
{
    constexpr int kChunks = DQP / 2;
    const int lane = threadIdx.x & 63;
    bool bad = false;
    for (int t = token + lane / kChunks; t < end; t += 64 / kChunks)
        bad = bad || not_finite(m.load(t, 8 * (lane % kChunks), true));
    return __ballot(bad) != 0;
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
// A row times `by`, added to the accumulators (from the row's tile `first` on) of the
// lanes that see it.
template <typename T, int DQP, int N>
__device__ __forceinline__ void row_add(f32x16 (&acc)[N], const WholeMap<T, DQP> &m, int64_t token, float by, bool sees,
                                        int first = 0)
{
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const T *p = m.at(token, 32 * (first + i) + 8 * g + 4 * ((threadIdx.x & 63) >> 5));
#pragma unroll
            for (int t = 0; t < 4; ++t)
                acc[i][4 * g + t] = sees ? fmaf(by, float(p[t]), acc[i][4 * g + t]) : acc[i][4 * g + t];
        }
}

// A D x 32 tile of accumulators, transposed, to a row of fp32.
template <int N> __device__ __forceinline__ void store_part(float *dst, const f32x16 (&v)[N], bool here)
{
    if (!here)
        return;
#pragma unroll
    for (int i = 0; i < N; ++i)
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
