// Causal attention of packed sequences on gfx950, forward.
//
// As in the attention between all pixels of a map, a work-group of four waves
// takes 128 queries of one head and sequence and walks over the keys in tiles of LDS
// with the running maximum and sum of a softmax; the transposed scores S^T = K Q^T
// leave a query's scores in two lanes.  The walk ends with the keys that the block's
// last query sees.
//
// Where there are 512 blocks of 256 queries, a wave has 64: a tile's operands are read
// from LDS once for two products.  (Nine sequences of up to 6400 tokens, 8 heads of 64
// reals on 2: 179 to 183 us on one card, 740 TFLOP/s, 245 with 32 queries a wave and the
// blocks in order; 213 on another card.)  Its SIMDs are then 31 % of the time in matrix
// instructions and 53 % in vector ones, with two waves each that overlap little
// (waiting 29 %).  No faster, each on its own: scores
// without the running maximum where a tile's sum shows that none is far ahead (a fifth
// fewer vector instructions), raised wave priorities for either half of a tile, walks
// that begin in different places, tiles dealt to two sets of waves in a work-group.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "packed_tile.h"

namespace quan {
namespace {

constexpr float kAhead = 8.0f;  // probabilities of 2^8 at most

struct Forward {
    PackedCall c;
    AttnMap out, rest;  // (rest.data may be NULL)
    float *stats;
    int blocks, splits, near;
    float *part, *part_stats;  // [split][head][token][D], [split][head][token][2]; splits > 1
};

// QN: sets of 32 queries that a wave holds.  PARTS: bf16 numbers that a probability
// meets v in, the second what the first leaves of it (see cut()).  At inference one will do: it is
// off by 2^-8 of a term at most, as out is of the sum once it is rounded.  In a
// training step (with rest) there are two: the rows' sums of dout out go into every
// dS, and with probabilities of 8 bits and the rounded out the queries' gradient was
// 0.0025 to 0.005 of its norm off (sequences of 1600 and of 2 tokens; bf16's own
// rounding is 0.0017).
template <typename T, int DQP, int QN, int PARTS>
__global__ void __launch_bounds__(kThreads, 2) packed_forward_kernel(Forward f)
{
    constexpr int DP = 4 * DQP;
    typedef Stage<T, DP, kThreads> Tile;
    typedef typename Elem<T>::frag frag;
    constexpr int KT = Tile::kTokens, SUBS = KT / 32, SIZE = kBlock * QN;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds_raw[];
    __shared__ int flags[2 * kWaves];
    T *k_lds = reinterpret_cast<T *>(lds_raw), *v_lds = k_lds + 2 * Tile::kElems;

    const PackedCall &c = f.c;
    // the blocks that see most keys first; of the shares of walks all first ones, then
    // all second ones: in between, those that are none would leave the same compute
    // units idle
    const auto [head, id] = unit_of(blockIdx.x, c.heads, f.near);
    const int kv_head = head / (c.heads / c.kv_heads), split = id / f.blocks;
    if (split >= f.splits)
        return;
    const Place b = place_of<SIZE, KT, false>(c, id - split * f.blocks, f.splits);
    const Tokens &qt = b.q, &kt = b.k;
    const Walk &walk = b.walk;
    if (b.at >= qt.len || split >= walk.count)
        return;
    const int all = c.causal ? min(kt.len, min(b.at + SIZE, qt.len) + kt.len - qt.len) : kt.len;
    const int begin = split * walk.per * KT, end = min(all, begin + walk.per * KT);

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
    const int half_at = KT / 2 * half;  // the lane's half of a tile
    const int wave_at = b.at + 32 * QN * wave, query = wave_at + (lane & 31);  // the first of the lane's queries
    // keys that a query sees: those below query + shift
    const int shift = c.causal ? kt.len - qt.len + 1 : 0;
    const int wave_end = wave_at >= qt.len ? 0 : c.causal ? min(end, wave_at + 32 * QN - 1 + shift) : end;

    const WholeMap<T, DQP> qm(c.q, qt.img, head), km(c.k, kt.img, kv_head), vm(c.v, kt.img, kv_head);
    Tile k_tile, v_tile;
    if (begin < end) {
        k_tile.fetch(km, kt.at + begin, kt.at + end);
        v_tile.fetch(vm, kt.at + begin, kt.at + end);
    }
    // scores are taken with the scale's magnitude, its sign goes to q (0: q is 0)
    const float sign = c.scale < 0.0f ? -1.0f : c.scale > 0.0f ? 1.0f : 0.0f;
    const float scale = c.scale != 0.0f ? fabsf(c.scale) * kLog2e : 1.0f;
    frag q[QN][DP / 16];
#pragma unroll
    for (int n = 0; n < QN; ++n)
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) {
            q[n][i] = qm.load(qt.at + query + 32 * n, 16 * i + 8 * half, query + 32 * n < qt.len);
            if (sign != 1.0f)
                q[n][i] = to_frag<T>(to_f32(q[n][i]) * sign);
        }

    f32x16 o[QN][DP / 32];
    float base[QN], ahead[QN], sum[QN];
#pragma unroll
    for (int n = 0; n < QN; ++n) {
#pragma unroll
        for (int i = 0; i < DP / 32; ++i)
            o[n][i] = 0.0f;
        base[n] = sum[n] = 0.0f;
        ahead[n] = -INFINITY;
    }

    // tiles from here on are not seen by all of the block's queries
    const int edge = c.causal ? max(0, b.at + shift) / KT * KT : all;
    bool left = false;
    int buf = 0;
    for (int j0 = begin; j0 < end; j0 += KT, buf ^= 1) {
        T *kb = k_lds + buf * Tile::kElems, *vb = v_lds + buf * Tile::kElems;
        if (j0 >= edge)
            flag_wave(flags + buf * kWaves, staged_not_finite(v_tile));
        k_tile.put(kb);
        v_tile.put(vb);
        __syncthreads();
        if (j0 + KT < end) {
            k_tile.fetch(km, kt.at + j0 + KT, kt.at + end);
            v_tile.fetch(vm, kt.at + j0 + KT, kt.at + end);
        }
        if (j0 >= edge && flagged<kWaves>(flags + buf * kWaves)) {
            left = true;
            continue;
        }
        if (j0 >= wave_end)
            continue;  // (none of the wave's queries sees the tile)
        f32x16 s[QN][SUBS];
#pragma unroll
        for (int sub = 0; sub < SUBS; ++sub) {
#pragma unroll
            for (int n = 0; n < QN; ++n)
                s[n][sub] = 0.0f;
#pragma unroll
            for (int i = 0; i < DP / 16; ++i) {
                const frag row = row_frag<T, DP>(kb, sub, i);
#pragma unroll
                for (int n = 0; n < QN; ++n)
                    s[n][sub] = mma(row, q[n][i], s[n][sub]);
            }
        }
#pragma unroll
        for (int n = 0; n < QN; ++n) {
            // tiles that reach past what the first of the queries sees
            if (j0 + KT > min(end, c.causal ? wave_at + 32 * n + shift : end)) {
                const int seen = c.causal ? min(query + 32 * n + shift, end) : end;
#pragma unroll
                for (int sub = 0; sub < SUBS; ++sub)
                    clear_behind(s[n][sub], seen - j0 - half_at, sub, -INFINITY);
            }
            // in units of log 2 from `base`, which follows the row's maximum where that
            // is kAhead above it (and first of all)
            float most = -INFINITY;
#pragma unroll
            for (int sub = 0; sub < SUBS; ++sub)
#pragma unroll
                for (int r = 0; r < 16; r += 2) {
                    s[n][sub][r] = fmaf(s[n][sub][r], scale, -base[n]);
                    s[n][sub][r + 1] = fmaf(s[n][sub][r + 1], scale, -base[n]);
                    most = fmaxf(most, fmaxf(s[n][sub][r], s[n][sub][r + 1]));
                }
            most = half_max(most);
            if (__any(most > ahead[n])) {
                const float up = most > ahead[n] ? most : 0.0f;
                const float back = ahead[n] == -INFINITY ? 0.0f : exp2_fast(-up);  // (nothing before)
                base[n] += up;
                ahead[n] = most > ahead[n] ? kAhead : ahead[n];
                sum[n] *= back;
#pragma unroll
                for (int i = 0; i < DP / 32; ++i)
                    o[n][i] *= back;
#pragma unroll
                for (int sub = 0; sub < SUBS; ++sub)
                    s[n][sub] -= up;
            }
#pragma unroll
            for (int sub = 0; sub < SUBS; ++sub)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    s[n][sub][r] = exp2_fast(s[n][sub][r]);
                    sum[n] += s[n][sub][r];
                }
        }
#pragma unroll
        for (int sub = 0; sub < SUBS; ++sub)
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                frag p[QN][PARTS];
#pragma unroll
                for (int n = 0; n < QN; ++n) {
                    if constexpr (PARTS == 2) {
                        f32x8 t;
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            t[e] = s[n][sub][8 * st + e];
                        p[n][0] = cut(t);
                        p[n][1] = to_frag<T>(t);
                    } else {
                        p[n][0] = acc_frag<T>(s[n][sub], st);
                    }
                }
#pragma unroll
                for (int i = 0; i < DP / 32; ++i) {
                    const frag column = col_frag<DP>(vb, sub, st, i);
#pragma unroll
                    for (int n = 0; n < QN; ++n)
#pragma unroll
                        for (int part = 0; part < PARTS; ++part)
                            o[n][i] = mma(column, p[n][part], o[n][i]);
                }
            }
    }
#pragma unroll
    for (int n = 0; n < QN; ++n)
        sum[n] = half_sum(sum[n]);
    if (left)
        for (int j0 = max(begin, edge); j0 < end; j0 += KT) {
            if (!rows_not_finite(vm, kt.at + j0, kt.at + min(j0 + KT, end)))
                continue;
            for (int j = j0; j < min(j0 + KT, end); ++j)
#pragma unroll
                for (int n = 0; n < QN; ++n) {
                    const bool sees = j < query + 32 * n + shift;
                    const float t = row_dot(km, kt.at + j, q[n]) * scale;
                    const bool up = sees && t > base[n] + ahead[n];
                    const float back = !up ? 1.0f : ahead[n] == -INFINITY ? 0.0f : exp2_fast(base[n] - t);
                    base[n] = up ? t : base[n];
                    ahead[n] = up ? kAhead : ahead[n];
                    const float p = exp2_fast(t - base[n]);
                    sum[n] = sees ? fmaf(sum[n], back, p) : sum[n];
#pragma unroll
                    for (int i = 0; i < DP / 32; ++i)
                        o[n][i] *= back;
                    row_add(o[n], vm, kt.at + j, p, sees);
                }
        }
    const HeadMap<T, DQP> om(f.out, qt.img, head, c.dq);
#pragma unroll
    for (int n = 0; n < QN; ++n) {
        const int token = qt.at + query + 32 * n;
        const bool here = query + 32 * n < qt.len;
        const int64_t row = head * c.q_tokens() + int64_t(qt.img) * c.qs.tokens + token;
        if (walk.count > 1) {
            const int64_t at = split * (c.heads * c.q_tokens()) + row;
            store_part<DP / 32>(f.part + at * DP, o[n], here);
            if (half == 0 && here) {
                f.part_stats[2 * at] = ahead[n] == -INFINITY ? -INFINITY : base[n];
                f.part_stats[2 * at + 1] = sum[n];
            }
            continue;
        }
        const float inv = sum[n] > 0.0f || sum[n] != sum[n] ? 1.0f / sum[n] : 0.0f;
#pragma unroll
        for (int i = 0; i < DP / 32; ++i) {
            o[n][i] *= inv;
            om.store(token, i, half, o[n][i], here);
        }
        if constexpr (PARTS > 1) {
            const HeadMap<T, DQP> rm(f.rest, qt.img, head, c.dq);
#pragma unroll
            for (int i = 0; i < DP / 32; ++i)
#pragma unroll
                for (int gq = 0; gq < 4; ++gq) {
                    const int d = 32 * i + 8 * gq + 4 * half;
                    const f32x4 v = {o[n][i][4 * gq], o[n][i][4 * gq + 1], o[n][i][4 * gq + 2], o[n][i][4 * gq + 3]};
                    if (here)
                        store_rest(rm.at(token, d), v, rm.valid(d, 4), rm.vec);
                }
        }
        if (f.stats != nullptr && half == 0 && here) {
            f.stats[2 * row] = base[n];
            f.stats[2 * row + 1] = sum[n];
        }
    }
}

// The results of work-groups that shared a block's keys, joined: D / 4 lanes for a
// query, 4 reals each.
template <typename T, int DQP> __global__ void __launch_bounds__(kThreads) packed_join_kernel(Forward f)
{
    constexpr int DP = 4 * DQP, KT = Elem<T>::kTile, kLanes = DP / 4, kGroups = join_groups(DP);
    __shared__ int counts[kWaves];
    const PackedCall &c = f.c;
    const auto [head, id] = unit_of(blockIdx.x, c.heads, f.near);
    if (id >= f.blocks * kGroups)
        return;
    const Block b = locate(c.qs, id / kGroups, counts);
    const Tokens qt = tokens_of(c.qs, c.qs.first, b.seq), kt = tokens_of(c.ks, c.ks.first, b.seq);
    const int query = b.at + id % kGroups * (kThreads / kLanes) + threadIdx.x / kLanes, d = 4 * (threadIdx.x % kLanes);
    const int tiles = key_tiles<KT>(c.causal, qt.len, kt.len, b.at + kBlock);
    const Walk walk = walk_of<KT, false>(c, qt.len, kt.len, tiles, f.splits, all_walks<kBlock, KT, false>(c));
    if (walk.count == 1 || query >= qt.len)
        return;
    const int64_t row = head * c.q_tokens() + int64_t(qt.img) * c.qs.tokens + qt.at + query;
    float top = -INFINITY, sum = 0.0f;
    f32x4 o = 0.0f;
#pragma unroll 4
    for (int s = 0; s < walk.count; ++s) {
        const int64_t at = s * (c.heads * c.q_tokens()) + row;
        const float t = f.part_stats[2 * at], l = f.part_stats[2 * at + 1];
        const f32x4 v = *reinterpret_cast<const f32x4 *>(f.part + at * DP + d);
        const float now = fmaxf(top, t), m = now == -INFINITY ? 0.0f : now;
        const float back = exp2_fast(top - m), w = exp2_fast(t - m);
        top = now;
        sum = sum * back + l * w;
        o = o * back + v * w;
    }
    o *= sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
    const HeadMap<T, DQP> om(f.out, qt.img, head, c.dq);
    store_quad(om.at(qt.at + query, d), o, om.valid(d, 4), om.vec);
    if constexpr (sizeof(T) == 2) {
        if (f.rest.data != nullptr) {
            const HeadMap<T, DQP> rm(f.rest, qt.img, head, c.dq);
            store_rest(rm.at(qt.at + query, d), o, rm.valid(d, 4), rm.vec);
        }
    }
    if (f.stats != nullptr && d == 0) {
        f.stats[2 * row] = top == -INFINITY ? 0.0f : top;
        f.stats[2 * row + 1] = sum;
    }
}

constexpr int64_t kMaxExtra = int64_t(64) << 20;

// Work-groups that share a block's walk where there are few blocks.
int forward_splits(const PackedCall &c, DType dt, bool may_split)
{
    const int64_t groups = packed_blocks(c.qs) * c.heads;
    const int tiles = (c.ks.tokens + (dt == DType::BF16 ? 63 : 31)) / (dt == DType::BF16 ? 64 : 32);
    if (!may_split || groups >= kSlots)
        return 1;
    const int64_t room = kMaxExtra / (c.heads * c.q_tokens() * (4 * padded_dq(c.dq) + 2) * int64_t(sizeof(float)));
    return int(std::max<int64_t>(1, std::min({(2 * kSlots + groups - 1) / groups, int64_t(tiles) / 4, room})));
}

template <typename T, int DQP, int PARTS> hipError_t launch(Forward f, hipStream_t s)
{
    constexpr int kTile = Elem<T>::kTile;
    const size_t lds = size_t(4) * kTile * Lds<T, 4 * DQP>::kRow * sizeof(T);
    // blocks twice as large where there are enough of them
    constexpr bool kWide = sizeof(T) == 2 && DQP <= 16;
    if constexpr (kWide) {
        const int64_t wide = packed_blocks(f.c.qs, 2 * kBlock);
        if (f.splits == 1 && wide * f.c.heads >= 512) {
            f.blocks = int(wide);
            packed_forward_kernel<T, DQP, 2, PARTS><<<unsigned(unit_blocks(wide, f.c.heads, f.near)), kThreads, lds, s>>>(f);
            return hipGetLastError();
        }
    }
    const auto grid = [&](int64_t ids) { return unsigned(unit_blocks(ids, f.c.heads, f.near)); };
    packed_forward_kernel<T, DQP, 1, PARTS><<<grid(int64_t(f.blocks) * f.splits), kThreads, lds, s>>>(f);
    if (hipError_t e = hipGetLastError())
        return e;
    if (f.splits > 1)
        packed_join_kernel<T, DQP><<<grid(int64_t(f.blocks) * join_groups(4 * DQP)), kThreads, 0, s>>>(f);
    return hipGetLastError();
}
template <typename T, int DQP> hipError_t launch_parts(const Forward &f, hipStream_t s)
{
    if constexpr (sizeof(T) == 2)
        if (f.rest.data != nullptr)
            return launch<T, DQP, 2>(f, s);
    return launch<T, DQP, 1>(f, s);
}
template <typename T> hipError_t launch_dq(const Forward &f, hipStream_t s)
{
    switch (padded_dq(f.c.dq)) {
    case 8:
        return launch_parts<T, 8>(f, s);
    case 16:
        return launch_parts<T, 16>(f, s);
    default:
        return launch_parts<T, 32>(f, s);
    }
}

}  // namespace

size_t packed_copy_bytes(int64_t tokens, int heads, int dq, DType dt)
{
    return (size_t(tokens) * heads * 4 * padded_dq(dq) * (dt == DType::BF16 ? 2 : 4) + 255) & ~size_t(255);
}

void packed_copy_add(AttnPack &pack, AttnMap &m, int images, int tokens, int heads, int dq, DType dt, unsigned char *&at)
{
    const int i = pack.maps++;
    const int64_t d = 4 * padded_dq(dq);
    pack.src[i] = m;
    pack.kv_len[i] = nullptr;
    pack.heads[i] = heads;
    pack.by_heads[i] = FastDiv(heads);
    pack.tokens[i] = tokens;
    pack.dst[i] = at;
    m = {at, int64_t(heads) * tokens * d, d, d / 4, true, tokens * d};
    at += packed_copy_bytes(int64_t(images) * tokens, heads, dq, dt);
}

size_t packed_forward_work_bytes(const PackedCall &c, DType dt)
{
    if (c.q.vec && c.k.vec && c.v.vec && padded_dq(c.dq) == c.dq)
        return 0;
    return packed_copy_bytes(c.q_tokens(), c.heads, c.dq, dt) + 2 * packed_copy_bytes(c.k_tokens(), c.kv_heads, c.dq, dt);
}

size_t packed_forward_extra_bytes(const PackedCall &c, DType dt)
{
    const int splits = forward_splits(c, dt, true);
    return splits == 1 ? 0 : size_t(splits) * c.heads * c.q_tokens() * (4 * padded_dq(c.dq) + 2) * sizeof(float);
}

hipError_t packed_forward_run(const PackedCall &c, DType dt, const AttnMap &out, void *rest, float *stats, void *work,
                              void *extra, hipStream_t s)
{
    Forward f;
    f.c = c;
    f.out = out;
    f.rest = packed_dense(c, rest);
    f.stats = stats;
    f.blocks = int(packed_blocks(c.qs));
    f.splits = forward_splits(c, dt, extra != nullptr);
    f.part = static_cast<float *>(extra);
    f.part_stats = f.part + (f.splits > 1 ? size_t(f.splits) * c.heads * c.q_tokens() * 4 * padded_dq(c.dq) : 0);
    if (work != nullptr) {
        AttnPack pack;
        pack.maps = 0;
        unsigned char *at = static_cast<unsigned char *>(work);
        packed_copy_add(pack, f.c.q, c.images, c.qs.tokens, c.heads, c.dq, dt, at);
        packed_copy_add(pack, f.c.k, c.images, c.ks.tokens, c.kv_heads, c.dq, dt, at);
        packed_copy_add(pack, f.c.v, c.images, c.ks.tokens, c.kv_heads, c.dq, dt, at);
        if (hipError_t e = attention_pack_run(pack, c.images, c.dq, dt, s))
            return e;
    }
    f.near = near_heads(f.c.q, c.heads, c.dq, dt == DType::BF16 ? 2 : 4);
    return dt == DType::BF16 ? launch_dq<__bf16>(f, s) : launch_dq<float>(f, s);
}

}  // namespace quan
