// The gradients of causal attention of packed sequences on gfx950.
//
// With P the probabilities, recomputed from the rows' saved maxima and sums,
//   dP = dO V^T,  delta_i = dO_i . O_i,  dS = P (dP - delta),
//   dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO.
// Two launches, so that every sum has one owner and a fixed order: the first takes
// blocks of queries and walks over the keys that they see (dQ, delta), the second
// blocks of keys and walks over the queries that see them, head by head of those
// that share them (dK, dV).
//
// 7200 tokens in nine sequences, 8 heads of 64 reals: 41 to 43 us and 50 to 54; one of
// 6400, 4 heads of 128 on 2: 118 to 123 and 130 to 139, and 21 to sum the parts of shared
// walks, with matrix units 20 and 24 % busy.  Their waves, one to two a SIMD, wait 36 to
// 44 % of their time, for LDS and for each other at a tile's barrier; a walk of one tile
// takes 8 us, and the longest walks of the nine sequences three times the mean.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <utility>

#include "packed_tile.h"

namespace quan {
namespace {

struct Backward {
    PackedCall c;
    AttnMap out, rest, dout, dq, dk, dv;  // (rest.data may be NULL)
    const float *stats;
    float *delta;  // [heads][q_tokens]
    int q_blocks, k_blocks, q_splits, k_splits, q_near, k_near;
    float *part_q, *part_k, *part_v;  // [split][head][token][D] where walks are shared
};

// Heads of more than 64 bf16 reals have two waves for 32 tokens, each with one of the
// two parts of every tile, so that what a wave holds fits in half of a SIMD's
// registers; what they make of their parts they exchange through LDS.
template <typename T, int DQP> constexpr int kPair = sizeof(T) == 2 && DQP > 16 ? 2 : 1;
// Operands of a chain of products that are read together.  (Four of 64 reals against
// one at a time, 7200 tokens in nine sequences: the keys' gradient 62 us and 66; of 128
// there are no registers.)
template <typename T, int DP> constexpr int kBatch = sizeof(T) == 4 || DP == 32 ? 2 : DP == 64 ? 4 : 1;

template <typename T, int DQP, int PAIR = kPair<T, DQP>>
__global__ void __launch_bounds__(64 * kWaves * PAIR, DQP <= 16 || PAIR == 2 ? 2 : 1) packed_dq_kernel(Backward f)
{
    constexpr int DP = 4 * DQP, WAVES = kWaves * PAIR;
    typedef Stage<T, DP, 64 * WAVES> Tile;
    typedef typename Elem<T>::frag frag;
    constexpr int KT = Tile::kTokens, SUBS = KT / 32 / PAIR, MINE = DP / 32 / PAIR;  // parts, and sums' tiles, of a wave
    extern __shared__ __attribute__((aligned(16))) unsigned char lds_raw[];
    __shared__ int flags[2 * WAVES];
    __shared__ frag swap[PAIR == 2 ? WAVES * 2 * 64 : 1];
    T *k_lds = reinterpret_cast<T *>(lds_raw), *v_lds = k_lds + 2 * Tile::kElems;

    const PackedCall &c = f.c;
    const auto [head, id] = unit_of(blockIdx.x, c.heads, f.q_near);
    const int kv_head = head / (c.heads / c.kv_heads), split = id / f.q_blocks;
    if (split >= f.q_splits)
        return;
    const Place b = place_of<kBlock, KT, false>(c, id - split * f.q_blocks, f.q_splits);
    const Tokens &qt = b.q, &kt = b.k;
    const Walk &walk = b.walk;
    if (b.at >= qt.len || split >= walk.count)
        return;
    const int lane = threadIdx.x & 63, wave = (threadIdx.x >> 6) % kWaves, half = lane >> 5;
    const int second = (threadIdx.x >> 6) / kWaves;  // of a pair: the part that it takes, and the half of the sums
    const int half_at = KT / 2 * half;  // the lane's half of a tile
    const int query = b.at + 32 * wave + (lane & 31);
    const bool q_here = query < qt.len;
    const int shift = c.causal ? kt.len - qt.len + 1 : 0;
    const int all = c.causal ? min(kt.len, min(b.at + kBlock, qt.len) - 1 + shift) : kt.len;
    const int begin = split * walk.per * KT, end = min(all, begin + walk.per * KT);
    const int wave_end = b.at + 32 * wave >= qt.len ? 0 : c.causal ? min(end, b.at + 32 * wave + 31 + shift) : end;
    const int seen = min(c.causal ? query + shift : kt.len, end);

    const WholeMap<T, DQP> qm(c.q, qt.img, head), km(c.k, kt.img, kv_head), vm(c.v, kt.img, kv_head);
    Tile k_tile, v_tile;
    if (begin < end) {
        k_tile.fetch(km, kt.at + begin, kt.at + end);
        v_tile.fetch(vm, kt.at + begin, kt.at + end);
    }
    const int64_t row = head * c.q_tokens() + int64_t(qt.img) * c.qs.tokens + qt.at + query;
    frag q[DP / 16], go[DP / 16];
    float delta = 0.0f;
    {
        // (without a rest the map itself is read in its place, and not used)
        const bool rest = sizeof(T) == 2 && f.rest.data != nullptr;
        const WholeMap<T, DQP> gm(f.dout, qt.img, head), om(f.out, qt.img, head), rm(rest ? f.rest : f.out, qt.img, head);
        frag o[DP / 16], o_rest[DP / 16];
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) {
            const int d = 16 * i + 8 * half;
            q[i] = qm.load(qt.at + query, d, q_here);
            go[i] = gm.load(qt.at + query, d, q_here);
            o[i] = om.load(qt.at + query, d, q_here);
            if constexpr (sizeof(T) == 2)
                o_rest[i] = rm.load(qt.at + query, d, q_here);
        }
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) {
            f32x8 x = to_f32(o[i]);
            if constexpr (sizeof(T) == 2) {
                const f32x8 full = with_rest(o[i], o_rest[i]);
                x = rest ? full : x;
            }
            const f32x8 w = to_f32(go[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                delta = fmaf(w[e], x[e], delta);
        }
        delta = half_sum(delta);
        if (q_here && half == 0 && second == 0 && split == 0)
            f.delta[row] = delta;
    }
    // P = 2^(s - top) inv; rows without a key, and none, have P = 0
    const float sum = q_here ? f.stats[2 * row + 1] : 0.0f;
    const bool empty = sum == 0.0f;
    float top = q_here ? f.stats[2 * row] : 0.0f;
    top = empty ? INFINITY : top;
    const float inv = empty ? 0.0f : 1.0f / sum;
    const float minus = empty ? 0.0f : -delta * inv;
    const float scale = c.scale * kLog2e;
    // (waited for here, or each tile of the walk would wait for the loads before it)
    asm volatile("" : "+v"(top));

    f32x16 dq[MINE];
#pragma unroll
    for (int i = 0; i < MINE; ++i)
        dq[i] = 0.0f;
    // tiles from here on are not seen by all of the block's queries
    const int edge = c.causal ? max(0, b.at + shift) / KT * KT : all;
    bool left = false;
    int buf = 0;
    for (int j0 = begin; j0 < end; j0 += KT, buf ^= 1) {
        T *kb = k_lds + buf * Tile::kElems, *vb = v_lds + buf * Tile::kElems;
        if (j0 >= edge)
            flag_wave(flags + buf * WAVES, staged_not_finite(k_tile));
        k_tile.put(kb);
        v_tile.put(vb);
        __syncthreads();
        if (j0 + KT < end) {
            k_tile.fetch(km, kt.at + j0 + KT, kt.at + end);
            v_tile.fetch(vm, kt.at + j0 + KT, kt.at + end);
        }
        if (j0 >= edge && flagged<WAVES>(flags + buf * WAVES)) {
            left = true;
            continue;
        }
        const bool idle = j0 >= wave_end;  // (none of the wave's queries sees the tile, nor its partner's)
        const bool whole = j0 + KT <= min(end, c.causal ? b.at + 32 * wave + shift : end);
#pragma unroll
        for (int n = 0; n < SUBS; ++n) {
            const int sub = PAIR == 2 ? second : n;
            frag ds[2];
            if (!idle) {
                f32x16 s = 0.0f, dp = 0.0f;
#pragma unroll
                for (int i0 = 0; i0 < DP / 16; i0 += kBatch<T, DP>) {
                    frag kr[kBatch<T, DP>], vr[kBatch<T, DP>];
#pragma unroll
                    for (int i = 0; i < kBatch<T, DP>; ++i) {
                        kr[i] = row_frag<T, DP>(kb, sub, i0 + i);
                        vr[i] = row_frag<T, DP>(vb, sub, i0 + i);
                    }
#pragma unroll
                    for (int i = 0; i < kBatch<T, DP>; ++i) {
                        s = mma(kr[i], q[i0 + i], s);
                        dp = mma(vr[i], go[i0 + i], dp);
                    }
                }
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    s[r] = exp2_fast(fmaf(s[r], scale, -top)) * fmaf(dp[r], inv, minus);
                if (!whole)
                    clear_behind(s, seen - j0 - half_at - 16 * sub, 0, 0.0f);
#pragma unroll
                for (int st = 0; st < 2; ++st)
                    ds[st] = acc_frag<T>(s, st);
            }
            if constexpr (PAIR == 2) {
                frag *at = swap + lane;
                const int self = threadIdx.x >> 6, partner = (self + kWaves) % WAVES;
                if (!idle)
#pragma unroll
                    for (int st = 0; st < 2; ++st)
                        at[(2 * self + st) * 64] = ds[st];
                __syncthreads();
                if (idle)
                    continue;
#pragma unroll
                for (int st = 0; st < 2; ++st)
#pragma unroll
                    for (int i = 0; i < MINE; ++i)
                        dq[i] = mma(col_frag<DP>(kb, sub, st, second * MINE + i), ds[st], dq[i]);
#pragma unroll
                for (int st = 0; st < 2; ++st) {
                    const frag other = at[(2 * partner + st) * 64];
#pragma unroll
                    for (int i = 0; i < MINE; ++i)
                        dq[i] = mma(col_frag<DP>(kb, sub ^ 1, st, second * MINE + i), other, dq[i]);
                }
            } else if (!idle) {
                frag kc[2][MINE];
#pragma unroll
                for (int st = 0; st < 2; ++st)
#pragma unroll
                    for (int i = 0; i < MINE; ++i)
                        kc[st][i] = col_frag<DP>(kb, sub, st, i);
#pragma unroll
                for (int st = 0; st < 2; ++st)
#pragma unroll
                    for (int i = 0; i < MINE; ++i)
                        dq[i] = mma(kc[st][i], ds[st], dq[i]);
            }
        }
    }
    if (left)
        for (int j0 = max(begin, edge); j0 < end; j0 += KT) {
            if (!rows_not_finite(km, kt.at + j0, kt.at + min(j0 + KT, end)))
                continue;
            for (int j = j0; j < min(j0 + KT, end); ++j) {
                const float p = exp2_fast(fmaf(row_dot(km, kt.at + j, q), scale, -top));
                row_add(dq, km, kt.at + j, p * fmaf(row_dot(vm, kt.at + j, go), inv, minus), j < seen, second * MINE);
            }
        }
    if (walk.count > 1) {
        store_part<MINE>(f.part_q + (split * (c.heads * c.q_tokens()) + row) * DP + 32 * second * MINE, dq, q_here);
        return;
    }
    const HeadMap<T, DQP> om(f.dq, qt.img, head, c.dq);
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
        dq[i] *= c.scale;
        om.store(qt.at + query, second * MINE + i, half, dq[i], q_here);
    }
}

// A value of each row of a tile, as accumulators have them.
__device__ __forceinline__ f32x16 row_values(const float *values, int first, int sub)
{
    f32x16 v;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const f32x4 t = *reinterpret_cast<const f32x4 *>(values + first + 16 * sub + 4 * g);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            v[4 * g + e] = t[e];
    }
    return v;
}
// `value` in the accumulators of part `sub` whose tokens are before `from` of the
// lane's half of the tile.
__device__ __forceinline__ void clear_before(f32x16 &s, int from, int sub, float value)
{
    asm volatile("" : "+v"(from));
#pragma unroll
    for (int r = 0; r < 16; ++r)
        s[r] = 16 * sub + r < from ? value : s[r];
}

// The launch of the keys' side: lanes hold keys, registers queries.  Of a pair of
// waves one gathers dV, the other dK, each from its own and its partner's part.
template <typename T, int DQP, int PAIR = kPair<T, DQP>>
__global__ void __launch_bounds__(64 * kWaves * PAIR, DQP <= 16 || PAIR == 2 ? 2 : 1) packed_dkv_kernel(Backward f)
{
    constexpr int DP = 4 * DQP, WAVES = kWaves * PAIR;
    typedef Stage<T, DP, 64 * WAVES> Tile;
    typedef typename Elem<T>::frag frag;
    constexpr int QT = Tile::kTokens, SUBS = QT / 32 / PAIR;  // parts of a tile that a wave takes
    extern __shared__ __attribute__((aligned(16))) unsigned char lds_raw[];
    __shared__ int flags[2 * WAVES];
    __shared__ frag swap[PAIR == 2 ? WAVES * 2 * 64 : 1];
    float *rows = reinterpret_cast<float *>(lds_raw);  // [2][top, inv, -delta][QT]
    T *q_lds = reinterpret_cast<T *>(rows + 6 * QT), *g_lds = q_lds + 2 * Tile::kElems;

    const PackedCall &c = f.c;
    const auto [kv_head, id] = unit_of(blockIdx.x, c.kv_heads, f.k_near);
    const int group = c.heads / c.kv_heads, split = id / f.k_blocks;
    if (split >= f.k_splits)
        return;
    const Place b = place_of<kBlock, QT, true>(c, id - split * f.k_blocks, f.k_splits);
    const Tokens &qt = b.q, &kt = b.k;
    const Walk &walk = b.walk;
    if (b.at >= kt.len || split >= walk.count)
        return;
    // the walk: tiles of queries, head by head
    const Span tiles = query_tiles<QT>(c.causal, qt.len, kt.len, b.at);
    const int first = split * walk.per, last = min(group * tiles.count, first + walk.per);
    const int lane = threadIdx.x & 63, all_wave = threadIdx.x >> 6, wave = all_wave % kWaves, half = lane >> 5;
    const int second = all_wave / kWaves;  // of a pair: the part that it takes; the first gathers dV, the second dK
    const int half_at = QT / 2 * half;  // the lane's half of a tile
    const int wave_at = b.at + 32 * wave, key = wave_at + (lane & 31);
    const bool k_here = key < kt.len;
    // the first query that sees a key: key - back
    const int back = c.causal ? kt.len - qt.len : 0;

    const WholeMap<T, DQP> km(c.k, kt.img, kv_head), vm(c.v, kt.img, kv_head);
    frag k[DP / 16], v[DP / 16];
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) {
        k[i] = km.load(kt.at + key, 16 * i + 8 * half, k_here);
        v[i] = vm.load(kt.at + key, 16 * i + 8 * half, k_here);
    }
    f32x16 sums[3 - PAIR][DP / 32];  // dV, dK or the wave's one of them
#pragma unroll
    for (int which = 0; which < 3 - PAIR; ++which)
#pragma unroll
        for (int i = 0; i < DP / 32; ++i)
            sums[which][i] = 0.0f;
    const float scale = c.scale * kLog2e;
    Tile q_tile, g_tile;
    float row_top = 0.0f, row_sum = 0.0f, row_delta = 0.0f;  // of thread t < QT's query of a tile
    auto fetch = [&](int head, int i0) {
        q_tile.fetch(WholeMap<T, DQP>(c.q, qt.img, head), qt.at + i0, qt.at + qt.len);
        g_tile.fetch(WholeMap<T, DQP>(f.dout, qt.img, head), qt.at + i0, qt.at + qt.len);
        if (threadIdx.x < QT) {
            const int i = i0 + threadIdx.x;
            const int64_t row = head * c.q_tokens() + int64_t(qt.img) * c.qs.tokens + qt.at + min(i, qt.len - 1);
            row_top = f.stats[2 * row];
            row_sum = i < qt.len ? f.stats[2 * row + 1] : 0.0f;
            row_delta = f.delta[row];
        }
    };
    int head = kv_head * group, tile = tiles.from;
    if (first < last) {
        head += first / tiles.count;
        tile += first % tiles.count;
        fetch(head, tile * QT);
    }
    bool left = false;
    int buf = 0;
    for (int item = first; item < last; ++item, buf ^= 1) {
        const int i0 = tile * QT;
        T *qb = q_lds + buf * Tile::kElems, *gb = g_lds + buf * Tile::kElems;
        float *rw = rows + buf * 3 * QT;
        const bool edge = c.causal && i0 < b.at + kBlock - 1 - back;  // (a key is not seen by all of the tile)
        if (edge)
            flag_wave(flags + buf * WAVES, staged_not_finite(q_tile) || staged_not_finite(g_tile));
        q_tile.put(qb);
        g_tile.put(gb);
        if (threadIdx.x < QT) {
            const bool empty = row_sum == 0.0f;
            rw[threadIdx.x] = empty ? INFINITY : row_top;
            rw[QT + threadIdx.x] = empty ? 0.0f : 1.0f / row_sum;
            rw[2 * QT + threadIdx.x] = empty ? 0.0f : -row_delta;
        }
        __syncthreads();
        if (++tile == tiles.from + tiles.count) {
            tile = tiles.from;
            ++head;
        }
        if (item + 1 < last)
            fetch(head, tile * QT);
        if (edge && flagged<WAVES>(flags + buf * WAVES)) {
            left = true;
            continue;
        }
        // (a wave whose keys are not there, or that no query of the tile sees; its
        // partner has the same)
        const bool idle = wave_at >= kt.len || (c.causal && i0 + QT <= wave_at - back);
#pragma unroll
        for (int n = 0; n < SUBS; ++n) {
            const int sub = PAIR == 2 ? second : n;
            frag p[2], ds[2];
            if (!idle) {
                f32x16 s = 0.0f, dp = row_values(rw + 2 * QT, half_at, sub);  // dP - delta starts from -delta
#pragma unroll
                for (int j0 = 0; j0 < DP / 16; j0 += kBatch<T, DP>) {
                    frag qr[kBatch<T, DP>], gr[kBatch<T, DP>];
#pragma unroll
                    for (int i = 0; i < kBatch<T, DP>; ++i) {
                        qr[i] = row_frag<T, DP>(qb, sub, j0 + i);
                        gr[i] = row_frag<T, DP>(gb, sub, j0 + i);
                    }
#pragma unroll
                    for (int i = 0; i < kBatch<T, DP>; ++i) {
                        s = mma(qr[i], k[j0 + i], s);
                        dp = mma(gr[i], v[j0 + i], dp);
                    }
                }
                const f32x16 top = row_values(rw, half_at, sub), inv = row_values(rw + QT, half_at, sub);
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    s[r] = exp2_fast(fmaf(s[r], scale, -top[r])) * inv[r];
                    dp[r] *= s[r];
                }
                if (c.causal && i0 < wave_at + 31 - back) {
                    clear_before(s, key - back - i0 - half_at - 16 * sub, 0, 0.0f);
                    clear_before(dp, key - back - i0 - half_at - 16 * sub, 0, 0.0f);
                }
#pragma unroll
                for (int st = 0; st < 2; ++st) {
                    p[st] = acc_frag<T>(s, st);
                    ds[st] = acc_frag<T>(dp, st);
                }
            }
            if constexpr (PAIR == 2) {
                frag *at = swap + lane;
                if (!idle)
#pragma unroll
                    for (int st = 0; st < 2; ++st)
                        at[(2 * all_wave + st) * 64] = second == 0 ? ds[st] : p[st];
                __syncthreads();
                if (idle)
                    continue;
                const T *from = second == 0 ? gb : qb;
                const int partner = (all_wave + kWaves) % WAVES;
#pragma unroll
                for (int st = 0; st < 2; ++st) {
                    const frag mine = second == 0 ? p[st] : ds[st];
#pragma unroll
                    for (int i = 0; i < DP / 32; ++i)
                        sums[0][i] = mma(col_frag<DP>(from, sub, st, i), mine, sums[0][i]);
                }
#pragma unroll
                for (int st = 0; st < 2; ++st) {
                    const frag other = at[(2 * partner + st) * 64];
#pragma unroll
                    for (int i = 0; i < DP / 32; ++i)
                        sums[0][i] = mma(col_frag<DP>(from, sub ^ 1, st, i), other, sums[0][i]);
                }
            } else if (!idle) {
#pragma unroll
                for (int st = 0; st < 2; ++st) {
                    frag gc[DP / 32], qc[DP / 32];
#pragma unroll
                    for (int i = 0; i < DP / 32; ++i) {
                        gc[i] = col_frag<DP>(gb, sub, st, i);
                        qc[i] = col_frag<DP>(qb, sub, st, i);
                    }
#pragma unroll
                    for (int i = 0; i < DP / 32; ++i) {
                        sums[0][i] = mma(gc[i], p[st], sums[0][i]);
                        sums[2 - PAIR][i] = mma(qc[i], ds[st], sums[2 - PAIR][i]);
                    }
                }
            }
        }
    }
    if (left)
        for (int item = first; item < last; ++item) {
            const int h = kv_head * group + item / tiles.count, i0 = (tiles.from + item % tiles.count) * QT;
            const WholeMap<T, DQP> qm(c.q, qt.img, h), gm(f.dout, qt.img, h);
            const int end = min(i0 + QT, qt.len);
            if (i0 >= b.at + kBlock - 1 - back || (!rows_not_finite(qm, qt.at + i0, qt.at + end) &&
                                                   !rows_not_finite(gm, qt.at + i0, qt.at + end)))
                continue;
            for (int i = i0; i < end; ++i) {
                const int64_t row = h * c.q_tokens() + int64_t(qt.img) * c.qs.tokens + qt.at + i;
                const float sum = f.stats[2 * row + 1], inv = sum == 0.0f ? 0.0f : 1.0f / sum;
                const float top = sum == 0.0f ? INFINITY : f.stats[2 * row], delta = sum == 0.0f ? 0.0f : f.delta[row];
                const float p = exp2_fast(fmaf(row_dot(qm, qt.at + i, k), scale, -top)) * inv;
                const bool sees = i >= key - back;
                if (second == 0)
                    row_add(sums[0], gm, qt.at + i, p, sees);
                if (second == 1 || PAIR == 1)
                    row_add(sums[2 - PAIR], qm, qt.at + i, p * (row_dot(gm, qt.at + i, v) - delta), sees);
            }
        }
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        if (PAIR == 2 && which != second)
            continue;
        f32x16(&x)[DP / 32] = sums[PAIR == 2 ? 0 : which];
        if (walk.count > 1) {
            const int64_t row = kv_head * c.k_tokens() + int64_t(kt.img) * c.ks.tokens + kt.at + key;
            store_part<DP / 32>((which == 0 ? f.part_v : f.part_k) + (split * (c.kv_heads * c.k_tokens()) + row) * DP, x, k_here);
            continue;
        }
        const HeadMap<T, DQP> om(which == 0 ? f.dv : f.dk, kt.img, kv_head, c.dq);
#pragma unroll
        for (int i = 0; i < DP / 32; ++i) {
            if (which == 1)
                x[i] *= c.scale;
            om.store(kt.at + key, i, half, x[i], k_here);
        }
    }
}

// The results of work-groups that shared a block, added up in order: D / 4 lanes for
// a token, 4 reals each.  First the blocks of queries, then those of keys.
template <typename T, int DQP> __global__ void __launch_bounds__(kThreads) packed_sum_kernel(Backward f, int of_queries)
{
    constexpr int DP = 4 * DQP, TILE = Elem<T>::kTile, kLanes = DP / 4, kGroups = join_groups(DP);
    __shared__ int counts[kWaves];
    const PackedCall &c = f.c;
    const bool keys = int(blockIdx.x) >= of_queries;
    const int heads = keys ? c.kv_heads : c.heads;
    const auto [head, id] = unit_of(blockIdx.x - (keys ? of_queries : 0), heads, keys ? f.k_near : f.q_near);
    if (id >= (keys ? f.k_blocks : f.q_blocks) * kGroups)
        return;
    const Sequences &mine = keys ? c.ks : c.qs;
    const Block b = locate(mine, id / kGroups, counts);
    const Tokens qt = tokens_of(c.qs, c.qs.first, b.seq), kt = tokens_of(c.ks, c.ks.first, b.seq), t = keys ? kt : qt;
    const int token = b.at + id % kGroups * (kThreads / kLanes) + threadIdx.x / kLanes, d = 4 * (threadIdx.x % kLanes);
    const int q_tiles = query_tiles<TILE>(c.causal, qt.len, kt.len, b.at).count;
    const int k_tiles = key_tiles<TILE>(c.causal, qt.len, kt.len, b.at + kBlock);
    const Walk walk = keys ? walk_of<TILE, true>(c, qt.len, kt.len, q_tiles, f.k_splits, all_walks<kBlock, TILE, true>(c))
                           : walk_of<TILE, false>(c, qt.len, kt.len, k_tiles, f.q_splits, all_walks<kBlock, TILE, false>(c));
    if (walk.count == 1 || token >= t.len)
        return;
    const int64_t all = heads * (keys ? c.k_tokens() : c.q_tokens());
    const int64_t row = head * (keys ? c.k_tokens() : c.q_tokens()) + int64_t(t.img) * mine.tokens + t.at + token;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        if (which == 1 && !keys)
            break;
        const float *p = (keys ? which == 0 ? f.part_k : f.part_v : f.part_q) + row * DP + d;
        f32x4 s = 0.0f;
#pragma unroll 4
        for (int i = 0; i < walk.count; ++i)
            s += *reinterpret_cast<const f32x4 *>(p + i * all * DP);
        if (which == 0)
            s *= c.scale;
        const HeadMap<T, DQP> m(keys ? which == 0 ? f.dk : f.dv : f.dq, t.img, head, c.dq);
        store_quad(m.at(t.at + token, d), s, m.valid(d, 4), m.vec);
    }
}

template <typename T, int DQP> hipError_t launch(const Backward &f, hipStream_t s)
{
    constexpr int kTile = Elem<T>::kTile;
    const size_t lds = size_t(4) * kTile * Lds<T, 4 * DQP>::kRow * sizeof(T);
    const auto q_grid = [&](int64_t each) { return unsigned(unit_blocks(each * f.q_blocks, f.c.heads, f.q_near)); };
    const auto k_grid = [&](int64_t each) { return unsigned(unit_blocks(each * f.k_blocks, f.c.kv_heads, f.k_near)); };
    packed_dq_kernel<T, DQP><<<q_grid(f.q_splits), 64 * kWaves * kPair<T, DQP>, lds, s>>>(f);
    if (hipError_t e = hipGetLastError())
        return e;
    packed_dkv_kernel<T, DQP>
        <<<k_grid(f.k_splits), 64 * kWaves * kPair<T, DQP>, lds + 6 * kTile * sizeof(float), s>>>(f);
    if (hipError_t e = hipGetLastError())
        return e;
    const unsigned of_queries = f.q_splits > 1 ? q_grid(join_groups(4 * DQP)) : 0;
    const unsigned of_keys = f.k_splits > 1 ? k_grid(join_groups(4 * DQP)) : 0;
    if (of_queries + of_keys > 0)
        packed_sum_kernel<T, DQP><<<of_queries + of_keys, kThreads, 0, s>>>(f, int(of_queries));
    return hipGetLastError();
}
template <typename T> hipError_t launch_dq(const Backward &f, hipStream_t s)
{
    switch (padded_dq(f.c.dq)) {
    case 8:
        return launch<T, 8>(f, s);
    case 16:
        return launch<T, 16>(f, s);
    default:
        return launch<T, 32>(f, s);
    }
}

bool copies(const PackedCall &c, const PackedGradients &g)
{
    return !(c.q.vec && c.k.vec && c.v.vec && g.out.vec && g.dout.vec) || padded_dq(c.dq) != c.dq;
}
size_t round_up(size_t bytes)
{
    return (bytes + 255) & ~size_t(255);
}
size_t delta_bytes(const PackedCall &c)
{
    return round_up(size_t(c.heads) * c.q_tokens() * sizeof(float));
}

// Work-groups that share a walk of at most `tiles` where there are few walks.
int splits_of(int64_t groups, int64_t tiles)
{
    if (groups >= kSlots)
        return 1;
    return int(std::max<int64_t>(1, std::min<int64_t>((2 * kSlots + groups - 1) / groups, tiles / 4)));
}
struct Plan {
    int q_splits, k_splits;
    size_t part_q, part_k;
};
Plan plan(const PackedCall &c, DType dt)
{
    const int tile = dt == DType::BF16 ? 64 : 32, dp = 4 * padded_dq(c.dq);
    Plan p{};
    p.q_splits = splits_of(packed_blocks(c.qs) * c.heads, (c.ks.tokens + tile - 1) / tile);
    p.k_splits = splits_of(packed_blocks(c.ks) * c.kv_heads, int64_t(c.heads / c.kv_heads) * ((c.qs.tokens + tile - 1) / tile));
    if (p.q_splits > 1)
        p.part_q = round_up(size_t(p.q_splits) * c.heads * c.q_tokens() * dp * sizeof(float));
    if (p.k_splits > 1)
        p.part_k = round_up(size_t(p.k_splits) * c.kv_heads * c.k_tokens() * dp * sizeof(float));
    return p;
}

}  // namespace

size_t packed_backward_work_bytes(const PackedCall &c, DType dt, const PackedGradients &g)
{
    const Plan p = plan(c, dt);
    size_t bytes = delta_bytes(c) + p.part_q + 2 * p.part_k;
    if (copies(c, g))
        bytes += (g.rest != nullptr ? 4 : 3) * packed_copy_bytes(c.q_tokens(), c.heads, c.dq, dt) +
                 2 * packed_copy_bytes(c.k_tokens(), c.kv_heads, c.dq, dt);
    return bytes;
}

hipError_t packed_backward_run(const PackedCall &c, DType dt, const PackedGradients &g, void *work, hipStream_t s)
{
    Backward f;
    f.c = c;
    f.out = g.out;
    f.rest = packed_dense(c, g.rest);
    f.dout = g.dout;
    f.dq = g.dq;
    f.dk = g.dk;
    f.dv = g.dv;
    f.stats = g.stats;
    f.q_blocks = int(packed_blocks(c.qs));
    f.k_blocks = int(packed_blocks(c.ks));
    unsigned char *at = static_cast<unsigned char *>(work);
    f.delta = reinterpret_cast<float *>(at);
    at += delta_bytes(c);
    const Plan p = plan(c, dt);
    f.q_splits = p.q_splits;
    f.k_splits = p.k_splits;
    for (auto [part, bytes] : {std::pair{&f.part_q, p.part_q}, {&f.part_k, p.part_k}, {&f.part_v, p.part_k}}) {
        *part = reinterpret_cast<float *>(at);
        at += bytes;
    }
    if (copies(c, g)) {
        AttnPack pack;
        pack.maps = 0;
        for (AttnMap *m : {&f.c.q, &f.out, &f.dout, &f.rest})
            if (m->data != nullptr)
                packed_copy_add(pack, *m, c.images, c.qs.tokens, c.heads, c.dq, dt, at);
        for (AttnMap *m : {&f.c.k, &f.c.v})
            packed_copy_add(pack, *m, c.images, c.ks.tokens, c.kv_heads, c.dq, dt, at);
        if (hipError_t e = attention_pack_run(pack, c.images, c.dq, dt, s))
            return e;
    }
    f.q_near = near_heads(f.c.q, c.heads, c.dq, dt == DType::BF16 ? 2 : 4);
    f.k_near = near_heads(f.c.k, c.kv_heads, c.dq, dt == DType::BF16 ? 2 : 4);
    return dt == DType::BF16 ? launch_dq<__bf16>(f, s) : launch_dq<float>(f, s);
}

}  // namespace quan
