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

// The work-group's head and its number among that head's.  Work-groups go round the
// 8 XCDs, and each XCD has an L2 of its own with lines of 128 bytes, in which a map has
// the same component of up to 4 or 8 heads side by side: `near` such heads go one after
// another to one XCD, other heads and other blocks to others.  (7200 tokens in nine
// sequences, 8 heads of 64 bf16 reals: 41 and 50 us for the queries' and the keys'
// gradient, 50 and 62 with every head on an XCD of its own, which read 186 and 247 MB
// from beyond its L2 for maps of 30.)
struct Unit {
    int head, id;
};
__device__ __forceinline__ Unit unit_of(int block, int heads, int near)
{
    const int turn = block / 8, set = turn / near * 8 + block % 8, sets = heads / near;
    return {set % sets * near + turn % near, set / sets};
}
// Work-groups of a launch with `ids` numbers; some at the end have larger ones.
inline int64_t unit_blocks(int64_t ids, int heads, int near)
{
    return (ids * (heads / near) + 7) / 8 * 8 * near;
}
// Heads that share lines of a map whose elements have `size` bytes.
inline int near_heads(const AttnMap &m, int heads, int dq, int size)
{
    int near = 1;
    while (m.s_h == dq && heads % (2 * near) == 0 && 2 * near * dq * size <= 128)
        near *= 2;
    return near;
}

// Sum and maximum over a wave.
#define QUAN_DPP(v, ctrl) __builtin_amdgcn_update_dpp(0, v, ctrl, 0xf, 0xf, false)
__device__ __forceinline__ float wave_sum(float x)
{
    x += __int_as_float(QUAN_DPP(__float_as_int(x), 0xB1));
    x += __int_as_float(QUAN_DPP(__float_as_int(x), 0x4E));
    x += __int_as_float(QUAN_DPP(__float_as_int(x), 0x141));
    x += __int_as_float(QUAN_DPP(__float_as_int(x), 0x140));
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = half_sum(__uint_as_float(a[0]) + __uint_as_float(a[1]));
    return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x)));
}
__device__ __forceinline__ int wave_sum(int x)
{
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

// Tiles of keys that queries up to `last` (counted from 1) of a sequence see.
template <int TILE> __device__ __forceinline__ int key_tiles(bool causal, int lq, int lk, int last)
{
    return (max(0, causal ? min(lk, min(last, lq) + lk - lq) : lk) + TILE - 1) / TILE;
}
// The first tile of queries that sees a key at `at` or behind it, and how many from
// it on.
struct Span {
    int from, count;
};
template <int TILE> __device__ __forceinline__ Span query_tiles(bool causal, int lq, int lk, int at)
{
    const int from = causal ? max(0, at - (lk - lq)) / TILE : 0;
    return {from, max(0, (lq + TILE - 1) / TILE - from)};
}

// A walk is dealt out to `count` work-groups, `per` tiles to each (the last has the
// rest).
struct Walk {
    int per, count;
};
// Tiles of all walks of a sequence, KEYS: of blocks of keys over the queries that see
// them, else of blocks of queries over their keys.  (A rule of thumb: halves of the
// first and the last.)
template <int SIZE, int TILE, bool KEYS> __device__ __forceinline__ float walks_of(bool causal, int lq, int lk)
{
    const int blocks = ((KEYS ? lk : lq) + SIZE - 1) / SIZE;
    const int first = KEYS ? query_tiles<TILE>(causal, lq, lk, 0).count : key_tiles<TILE>(causal, lq, lk, SIZE);
    const int last = KEYS ? query_tiles<TILE>(causal, lq, lk, max(0, lk - 1)).count : key_tiles<TILE>(causal, lq, lk, lq);
    return 0.5f * float(blocks) * float(first + last);
}
// That of a block with `mine` tiles in its sequence (`times`: walks over the heads of
// a group one after another): to as many as have the share of one of kSlots
// work-groups of all walks, and what it costs to start one, each, where the
// sequence's longest walk is more than twice that; to `splits` at most, which is what
// the launch has.  (One sequence of 6400 tokens, 4 heads of 128 reals, a training
// step: 368 us, 384 with shares of 1 / 400, 409 of 1 / 300, 405 with starts of 3 tiles
// at 1 / 512; without shares 1569.)  all: the sum of walks_of() over the lanes' sequences.
// (Two to a compute unit, which is what heads of up to 64 bf16 reals and the wide
// forward pass have; registers and LDS leave the wide gradients one, so that there it
// is a share of what runs in two turns.)
constexpr int kSlots = 512;
constexpr int start_of(int tile) { return tile == 64 ? 4 : 1; }  // tiles' worth: bf16, fp32
template <int TILE, bool KEYS>
__device__ __forceinline__ Walk walk_of(const PackedCall &c, int lq, int lk, int mine, int splits, float all)
{
    const int times = KEYS ? c.heads / c.kv_heads : 1;
    const int longest = times * (((KEYS ? lq : lk) + TILE - 1) / TILE);
    const int share = int(fminf(wave_sum(all) * float(c.heads) / kSlots, 1e9f)) + start_of(TILE);
    if (longest <= 2 * share)
        return {max(1, times * mine), 1};
    const int per = max(share, (longest + splits - 1) / splits);
    return {per, max(1, (times * mine + per - 1) / per)};
}
template <int SIZE, int TILE, bool KEYS> __device__ __forceinline__ float all_walks(const PackedCall &c)
{
    float all = 0.0f;
    for (int i0 = 0; i0 < c.qs.count; i0 += 64) {
        const int seq = i0 + int(threadIdx.x & 63), at = min(seq, c.qs.count - 1);
        const float w = walks_of<SIZE, TILE, KEYS>(c.causal, tokens_of(c.qs, c.qs.first, at).len, tokens_of(c.ks, c.ks.first, at).len);
        all += seq < c.qs.count ? w : 0.0f;
    }
    return all;
}

// Block `id` of a launch, its sequence and its walk.  The blocks come in an order that
// begins with the longest walks: of 64 sequences at a time, first the blocks that are
// `level` from their sequence's one end, then those one less, down to 0 (whose walks
// are the shortest); queries' blocks from the last, of keys from the first.  at >= the
// sequence's length: none.  (What a wave needs it reads at once: a work-group has
// little to do before its first tile but to wait for memory.)
struct Place {
    Tokens q, k;
    int at;
    Walk walk;
};
template <int SIZE, int TILE, bool KEYS> __device__ __forceinline__ Place place_of(const PackedCall &c, int id, int splits)
{
    const int lane = threadIdx.x & 63;
    const Sequences &mine = KEYS ? c.ks : c.qs;
    Place p;
    float all = 0.0f;
    if (mine.first == nullptr) {
        const int per = (mine.tokens + SIZE - 1) / SIZE, down = id / mine.count;  // (equal lengths)
        const int seq = id - down * mine.count;
        p.q = {seq, 0, c.qs.tokens};
        p.k = {seq, 0, c.ks.tokens};
        p.at = (KEYS ? down : per - 1 - down) * SIZE;
        if (splits > 1)
            all = lane == 0 ? float(mine.count) * walks_of<SIZE, TILE, KEYS>(c.causal, p.q.len, p.k.len) : 0.0f;
    } else {
        const int n = mine.count;
        auto clamp = [&](int v, const Sequences &s) { return min(max(v, 0), s.tokens); };
        // the 64 sequences, counted as in locate()
        int set = 0;
        for (int i0 = 0; i0 + 64 < n; i0 += 64 * 64) {
            const int i = i0 + 64 * lane + 64;
            set += __popcll(__ballot(i < n && clamp(mine.first[min(i, n)], mine) / SIZE + i <= id));
        }
        set *= 64;
        const int seq = min(set + lane, n - 1);
        const int qa = clamp(c.qs.first[seq], c.qs), q_len = max(clamp(c.qs.first[seq + 1], c.qs) - qa, 0);
        // (one array for maps of two sizes: each map's tokens end with it)
        int ka = qa, k_len = q_len;
        if (c.ks.first != c.qs.first || c.ks.tokens != c.qs.tokens) {
            ka = clamp(c.ks.first[seq], c.ks);
            k_len = max(clamp(c.ks.first[seq + 1], c.ks) - ka, 0);
        }
        const int blocks = set + lane < n ? ((KEYS ? k_len : q_len) + SIZE - 1) / SIZE : 0;
        const int rank = id - (__builtin_amdgcn_readfirstlane(KEYS ? ka : qa) / SIZE + set);
        // the largest level with more than `rank` blocks at or above it
        int low = 0, high = wave_max(blocks);
        if (rank < 0 || rank >= wave_sum(blocks))
            return {{0, 0, 0}, {0, 0, 0}, 0, {1, 1}};
        while (high - low > 1) {
            const int mid = (low + high) >> 1;
            if (wave_sum(max(0, blocks - mid)) > rank)
                low = mid;
            else
                high = mid;
        }
        const int skip = rank - wave_sum(max(0, blocks - low - 1));
        const auto here = __ballot(blocks > low);
        const auto one = __ballot(blocks > low && __popcll(here & ((1ull << lane) - 1)) == skip);
        const int l = one != 0 ? __builtin_ctzll(one) : 0;
        p.q = {0, __builtin_amdgcn_readlane(qa, l), __builtin_amdgcn_readlane(q_len, l)};
        p.k = {0, __builtin_amdgcn_readlane(ka, l), __builtin_amdgcn_readlane(k_len, l)};
        const int of = ((KEYS ? p.k.len : p.q.len) + SIZE - 1) / SIZE;
        p.at = (KEYS ? of - 1 - low : low) * SIZE;
        if (splits > 1 && n > 64)
            all = all_walks<SIZE, TILE, KEYS>(c);
        else if (splits > 1)
            all = set + lane < n ? walks_of<SIZE, TILE, KEYS>(c.causal, q_len, k_len) : 0.0f;
    }
    const int tiles = KEYS ? query_tiles<TILE>(c.causal, p.q.len, p.k.len, p.at).count
                           : key_tiles<TILE>(c.causal, p.q.len, p.k.len, p.at + SIZE);
    if (splits > 1)
        p.walk = walk_of<TILE, KEYS>(c, p.q.len, p.k.len, tiles, splits, all);
    else
        p.walk = {max(1, (KEYS ? c.heads / c.kv_heads : 1) * tiles), 1};
    return p;
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
