// Attention between the pixels of quaternion maps on gfx950, forward.
//
// A work-group of four waves takes 128 queries of one head and image and walks
// over the keys in tiles of LDS with the running maximum and sum of a softmax; a
// wave holds its 32 queries' rows, and the transposed scores S^T = K Q^T leave a
// query's scores in two lanes (see attention_tile.h), so that maxima and sums
// are taken in registers and the probabilities are the next product's operand.
// What bounds it is what a wave issues between two products, 16 exponentials, sums
// and biases of a lane's scores: 16 images of 40 x 40, 8 heads of 64 reals, in
// training 276 us, 300 TFLOP/s of its two products (it makes four, see PARTS), with
// the SIMDs at vector instructions 65 % of the time, the matrix units 29 %, LDS 24 %.
// Where there are few work-groups it is that: 2 of 80 x 80, 4 heads of 128, 255 us,
// 660 TFLOP/s, 400 of them, 1.3 waves a SIMD that wait 38 % of their time (vector
// instructions 35 %, matrix units 25 %, LDS 28 %).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "attention_tile.h"

namespace quan {
namespace {

constexpr int kThreads = 256, kQueries = 128;  // of a work-group: a wave per 32 queries

// What a forward launch computes, and where its partial results go.
struct Forward {
    AttnCall a;
    Offsets o;
    AttnMap out;
    void *rest;
    float *stats;
    int blocks, splits, tiles_per_split;  // of queries per head; of the keys; tiles of a split
    float *part, *part_stats;             // [split][row][D], [split][row][2] (splits > 1)
};

// PARTS (3 in a training step in bf16, else 1): bf16 numbers that a probability
// meets v in, each what the ones before leave of it.  At inference one will do: it
// is off by 2^-8 of a term at most, as out is of the sum once it is rounded (all in
// all 2.3e-3 of out's norm, 1.7e-3 from out's own rounding).  The gradient of the bias,
// which is fp32, goes by the rows' sums of dout out: with probabilities of 8 bits
// 3e-4 of its norm was wrong, of 16 bits 1e-6 to 7e-6, of 24 bits what fp32
// leaves, 1e-7 to 4e-7.  The third part is 45 us of the 270 at 1600 queries and
// keys, 16 images, 8 heads of 64 reals.
template <typename T, int DQP, int MODE, int PARTS>
__global__ void __launch_bounds__(kThreads, 2) attention_forward_kernel(Forward f)
{
    constexpr int DP = 4 * DQP;
    typedef Stage<T, DP, kThreads> Tile;
    typedef typename Elem<T>::frag frag;
    constexpr int KT = Tile::kTokens, SUBS = KT / 32;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds_raw[];
    float *bias = reinterpret_cast<float *>(lds_raw);  // (at 0: its reads then have their offsets in the instruction)
    int *place = reinterpret_cast<int *>(bias + f.o.cap);
    T *k_lds = reinterpret_cast<T *>(place + 2 * KT), *v_lds = k_lds + 2 * Tile::kElems;

    const AttnGeom &g = f.a.g;
    const int lq = g.lq(), lk = g.lk();
    const int total = g.n * g.heads * f.splits * f.blocks;
    int id = xcd_order(total);
    if (id >= total)
        return;
    const int block = id % f.blocks;
    id /= f.blocks;
    const int split = id % f.splits;
    id /= f.splits;
    const int head = id % g.heads, img = id / g.heads;
    const int kv_head = head / (g.heads / g.kv_heads);

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
    const int half_at = KT / 2 * half;  // the lane's half of a tile
    const int q0 = block * kQueries;
    const int query = q0 + 32 * wave + (lane & 31);
    const bool q_here = query < lq;
    const int len = f.a.kv_len != nullptr ? min(max(f.a.kv_len[img], 0), lk) : lk;
    const int first = split * f.tiles_per_split * KT;
    const int end = min(len, first + f.tiles_per_split * KT);

    const WholeMap<T, DQP> qm(f.a.q, img, head), km(f.a.k, img, kv_head), vm(f.a.v, img, kv_head);
    Tile kt, vt;
    if (first < end) {
        kt.fetch(km, first, end);
        vt.fetch(vm, first, end);
    }
    frag q[DP / 16];
#pragma unroll
    for (int i = 0; i < DP / 16; ++i)
        q[i] = qm.load(query, 16 * i + 8 * half, q_here);

    f32x16 o[DP / 32];
#pragma unroll
    for (int i = 0; i < DP / 32; ++i)
        o[i] = 0.0f;
    float top = -INFINITY, sum = 0.0f;
    const float c = g.scale * kLog2e;

    // offsets of this work-group's queries
    int pos_y = 0, pos_x = 0, lane_at = 0, low_q = 0, high_q = 0, segment = -1;
    const float *table = nullptr;
    if (MODE != 0) {
        if (f.a.pos != nullptr) {
            pos_y = query_pos(f.a.pos[2 * img]);
            pos_x = query_pos(f.a.pos[2 * img + 1]);
        }
        table = f.a.bias.table + int64_t(head) * f.a.bias.ny * f.a.bias.nx;
        low_q = f.o.origin - place_q(f.o, min(q0 + kQueries, lq) - 1);
        high_q = f.o.origin - place_q(f.o, q0);
        lane_at = f.o.origin - place_q(f.o, min(query, lq - 1));
    }
    const int high = MODE != 0 ? high_q + place_k(f.o, max(end, 1) - 1) + 4 : 0;  // past the last offset

    int buf = 0;
    for (int j0 = first; j0 < end; j0 += KT, buf ^= 1) {
        T *kb = k_lds + buf * Tile::kElems, *vb = v_lds + buf * Tile::kElems;
        int *pl = place + buf * KT;
        kt.put(kb);
        vt.put(vb);
        if (MODE != 0) {
            if (threadIdx.x < KT)
                pl[threadIdx.x] = place_k(f.o, min(j0 + int(threadIdx.x), lk - 1));
            const int lo = low_q + place_k(f.o, j0), hi = high_q + place_k(f.o, min(j0 + KT, lk) - 1) + 3;
            if (segment < 0 || hi >= segment + f.o.cap) {
                if (segment >= 0)
                    __syncthreads();  // the last segment has been read
                segment = lo;
                stage_bias(bias, f.o, f.a.bias, table, segment, min(f.o.cap, high - segment), pos_y, pos_x);
            }
        }
        __syncthreads();
        if (j0 + KT < end) {
            kt.fetch(km, j0 + KT, end);
            vt.fetch(vm, j0 + KT, end);
        }
        if (q0 + 32 * wave >= lq)
            continue;  // (none of the wave's queries is there)
        f32x16 s[SUBS];
#pragma unroll
        for (int sub = 0; sub < SUBS; ++sub) {
            s[sub] = 0.0f;
#pragma unroll
            for (int i = 0; i < DP / 16; ++i)
                s[sub] = mma(row_frag<T, DP>(kb, sub, i), q[i], s[sub]);
        }
#pragma unroll
        for (int sub = 0; sub < SUBS; ++sub)
            add_bias<MODE, 1>(s[sub], c, bias, pl, lane_at - segment, half_at, sub);
        if (j0 + KT > end) {
#pragma unroll
            for (int sub = 0; sub < SUBS; ++sub)
                clear_behind(s[sub], end - j0 - half_at, sub, -INFINITY);
        }
        float t = s[0][0];
#pragma unroll
        for (int sub = 0; sub < SUBS; ++sub)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                t = fmaxf(t, s[sub][r]);
        t = half_max(t);
        if (__any(t > top)) {
            const float now = fmaxf(top, t);
            const float back = exp2_fast(top - (now == -INFINITY ? 0.0f : now));
            top = now;
            sum *= back;
#pragma unroll
            for (int i = 0; i < DP / 32; ++i)
                o[i] *= back;
        }
        const float m = top == -INFINITY ? 0.0f : top;
#pragma unroll
        for (int sub = 0; sub < SUBS; ++sub)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[sub][r] = exp2_fast(s[sub][r] - m);
                sum += s[sub][r];
            }
#pragma unroll
        for (int sub = 0; sub < SUBS; ++sub)
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                frag p[PARTS];
#pragma unroll
                for (int part = 0; part < PARTS; ++part) {
                    if (part > 0)
                        take_from(s[sub], st, p[part - 1]);
                    p[part] = acc_frag<T>(s[sub], st);
                }
#pragma unroll
                for (int i = 0; i < DP / 32; ++i) {
                    const frag column = col_frag<DP>(vb, sub, st, i);
#pragma unroll
                    for (int part = 0; part < PARTS; ++part)
                        o[i] = mma(column, p[part], o[i]);
                }
            }
    }
    sum = half_sum(sum);

    const int64_t row = (int64_t(img) * g.heads + head) * lq + query;
    if (f.splits > 1) {
        const int64_t rows = int64_t(g.n) * g.heads * lq;
        if (q_here) {
            float *dst = f.part + (split * rows + row) * DP;
#pragma unroll
            for (int i = 0; i < DP / 32; ++i)
#pragma unroll
                for (int gq = 0; gq < 4; ++gq) {
                    const f32x4 v = {o[i][4 * gq], o[i][4 * gq + 1], o[i][4 * gq + 2], o[i][4 * gq + 3]};
                    *reinterpret_cast<f32x4 *>(dst + 32 * i + 8 * gq + 4 * half) = v;
                }
            if (half == 0) {
                f.part_stats[(split * rows + row) * 2] = top;
                f.part_stats[(split * rows + row) * 2 + 1] = sum;
            }
        }
        return;
    }
    const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
    const HeadMap<T, DQP> om(f.out, img, head, g.dq);
#pragma unroll
    for (int i = 0; i < DP / 32; ++i) {
        o[i] *= inv;
        om.store(query, i, half, o[i], q_here);
    }
    if constexpr (sizeof(T) == 2) {
        if (f.rest != nullptr) {
            const int64_t c_all = int64_t(g.heads) * g.dq;
            const AttnMap dense{f.rest, lq * 4 * c_all, 4 * c_all, c_all, g.dq % 8 == 0, g.dq};
            const HeadMap<T, DQP> rm(dense, img, head, g.dq);
#pragma unroll
            for (int i = 0; i < DP / 32; ++i)
#pragma unroll
                for (int gq = 0; gq < 4; ++gq) {
                    const int d = 32 * i + 8 * gq + 4 * half;
                    const f32x4 v = {o[i][4 * gq], o[i][4 * gq + 1], o[i][4 * gq + 2], o[i][4 * gq + 3]};
                    if (q_here)
                        store_rest(rm.at(query, d), v, rm.valid(d, 4), rm.vec);
                }
        }
    }
    if (f.stats != nullptr && half == 0 && q_here) {
        f.stats[2 * row] = top == -INFINITY ? 0.0f : top;
        f.stats[2 * row + 1] = sum;
    }
}

// One real of a row's output from its sum over the keys.
template <typename T, int DQP>
__device__ __forceinline__ void finish_real(const Forward &f, int64_t row, int real, float value, float top, float sum)
{
    const AttnGeom &g = f.a.g;
    const int lq = g.lq();
    const int query = int(row % lq), head = int(row / lq % g.heads);
    const int64_t img = row / lq / g.heads;
    value *= sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
    const HeadMap<T, DQP> om(f.out, img, head, g.dq);
    if (om.valid(real, 1) > 0) {
        const T rounded = T(value);
        *om.at(query, real) = rounded;
        if constexpr (sizeof(T) == 2) {
            if (f.rest != nullptr) {
                const int64_t c_all = int64_t(g.heads) * g.dq;
                static_cast<short *>(f.rest)[((img * lq + query) * 4 + real / DQP) * c_all + int64_t(head) * g.dq + real % DQP] =
                    rest_of(value, rounded);
            }
        }
    }
    if (f.stats != nullptr && real == 0) {
        f.stats[2 * row] = top;
        f.stats[2 * row + 1] = sum;
    }
}

// The splits' partial results joined: a work-group per row, its lanes in sets
// of D / 4 (4 reals each) that take the splits in turn and meet in LDS.
template <typename T, int DQP>
__global__ void __launch_bounds__(256) attention_join_kernel(Forward f)
{
    constexpr int DP = 4 * DQP, kLanes = DP / 4, kSets = 256 / kLanes;
    __shared__ float acc_lds[kSets * DP];
    __shared__ float stat_lds[2 * kSets];
    const AttnGeom &g = f.a.g;
    const int lq = g.lq();
    const int64_t rows = int64_t(g.n) * g.heads * lq, row = blockIdx.x;
    const int set = threadIdx.x / kLanes, d = 4 * (threadIdx.x % kLanes);
    float top = -INFINITY, sum = 0.0f;
    f32x4 o = 0.0f;
#pragma unroll 4
    for (int s = set; s < f.splits; s += kSets) {
        const float t = f.part_stats[(s * rows + row) * 2], l = f.part_stats[(s * rows + row) * 2 + 1];
        const f32x4 v = *reinterpret_cast<const f32x4 *>(f.part + (s * rows + row) * DP + d);
        const float now = fmaxf(top, t), m = now == -INFINITY ? 0.0f : now;
        const float back = exp2_fast(top - m), w = exp2_fast(t - m);
        top = now;
        sum = sum * back + l * w;
        o = o * back + v * w;
    }
    *reinterpret_cast<f32x4 *>(acc_lds + set * DP + d) = o;
    if (d == 0) {
        stat_lds[2 * set] = top;
        stat_lds[2 * set + 1] = sum;
    }
    __syncthreads();
    if (threadIdx.x >= DP)
        return;
    const int real = threadIdx.x;
    top = -INFINITY;
    for (int s = 0; s < kSets; ++s)
        top = fmaxf(top, stat_lds[2 * s]);
    const float m = top == -INFINITY ? 0.0f : top;
    float value = 0.0f;
    sum = 0.0f;
    for (int s = 0; s < kSets; ++s) {
        const float w = exp2_fast(stat_lds[2 * s] - m);
        sum = fmaf(w, stat_lds[2 * s + 1], sum);
        value = fmaf(w, acc_lds[s * DP + real], value);
    }
    finish_real<T, DQP>(f, row, real, value, m, sum);
}

// ------------------------------------------------------- one query per image

// A chunk of 8 reals per lane: G = D / 8 neighbouring lanes hold a key of one
// head for GRP of the query heads that share it, and a work-group's lanes hold
// as many heads of a token as there are, so that they read whole rows of the
// map.  Each such set of lanes walks over every `slots`-th key with a softmax
// of its own; they are joined in LDS, and those of several splits of an image's
// keys (equal shares of what the image has) by attention_join_kernel.  Biases of
// a chunk of keys are looked up into LDS at a time.  Probabilities stay in fp32.
// Bound by the way of keys and values from memory, read once: a cache of 4 x 65536
// keys (half of them there), 8 heads of 64 reals on 2 of keys: 27 us, 2.5 TB/s, 1.9
// waves a SIMD that wait 53 % of their time, and 4 us of joining; 64 maps of 20 x 20,
// 4 heads of 64: 12 and 3 us, 0.9 waves, 73 %.
struct Token {
    int heads_per_block, slots, kv_blocks, group_blocks, chunk;
};
constexpr int kTokenBias = 8192;  // biases in LDS: keys of a chunk x query heads of the work-group
constexpr int kTokenUnroll = 4;   // keys that a set of lanes reads at a time

// Sum over the 4, 8 or 16 lanes of a row.
template <int G> __device__ __forceinline__ float lanes_sum(float x)
{
#define QUAN_DPP_ADD(ctrl) \
    x += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), ctrl, 0xf, 0xf, false))
    QUAN_DPP_ADD(0xB1);  // lane ^ 1
    QUAN_DPP_ADD(0x4E);  // lane ^ 2
    if (G >= 8)
        QUAN_DPP_ADD(0x141);  // 7 - lane of 8: the other four's sum
    if (G >= 16)
        QUAN_DPP_ADD(0x140);  // 15 - lane of 16
#undef QUAN_DPP_ADD
    return x;
}

template <typename T, int DQP, int GRP, bool BIAS>
__global__ void __launch_bounds__(kThreads) attention_token_kernel(Forward f, Token tk)
{
    constexpr int DP = 4 * DQP, G = DP / 8, kPairs = kThreads / G, U = kTokenUnroll;
    typedef typename Elem<T>::frag frag;
    // (a chunk's biases are done with when the results are joined)
    constexpr int kLds = kPairs * GRP * DP > kTokenBias ? kPairs * GRP * DP : kTokenBias;
    __shared__ __attribute__((aligned(16))) float acc_lds[kLds];
    __shared__ float stat_lds[kPairs * GRP * 2];
    float *bias_lds = acc_lds;
    const AttnGeom &g = f.a.g;
    const int lk = g.lk(), group = g.heads / g.kv_heads;
    int id = blockIdx.x;
    const int split = id % f.splits;
    id /= f.splits;
    const int gb = id % tk.group_blocks;
    id /= tk.group_blocks;
    const int kvb = id % tk.kv_blocks, img = id / tk.kv_blocks;
    const int pair = threadIdx.x / G, d = 8 * (threadIdx.x % G);
    const int slot = pair / tk.heads_per_block, kv_head = kvb * tk.heads_per_block + pair % tk.heads_per_block;
    const bool active = slot < tk.slots && kv_head < g.kv_heads;
    const int len = f.a.kv_len != nullptr ? min(max(f.a.kv_len[img], 0), lk) : lk;
    const int round = U * tk.slots, share = ((len + f.splits - 1) / f.splits + round - 1) / round * round;
    const int first = int(min(int64_t(split) * share, int64_t(len))), end = min(len, first + share);
    const int head0 = kv_head * group + gb * GRP;  // of GRP query heads
    const int heads_here = min(GRP, group - gb * GRP);

    const HeadMap<T, DQP> km(f.a.k, img, active ? kv_head : 0, g.dq), vm(f.a.v, img, active ? kv_head : 0, g.dq);
    f32x8 q[GRP], o[GRP];
    float top[GRP], sum[GRP];
    const float c = g.scale * kLog2e;
#pragma unroll
    for (int i = 0; i < GRP; ++i) {
        const bool here = active && i < heads_here;
        const HeadMap<T, DQP> qm(f.a.q, img, here ? head0 + i : 0, g.dq);
        q[i] = to_f32(qm.load(0, d, here)) * c;
        o[i] = 0.0f;
        top[i] = -INFINITY;
        sum[i] = 0.0f;
    }
    const int valid = active ? km.valid(d, 8) : 0;
    int pos_y = 0, pos_x = 0;
    if (BIAS && f.a.pos != nullptr) {
        pos_y = query_pos(f.a.pos[2 * img]);
        pos_x = query_pos(f.a.pos[2 * img + 1]);
    }
    const int nb = f.a.bias.ny * f.a.bias.nx;
    const int chunk = BIAS ? tk.chunk : max(end - first, 1);
    for (int c0 = first; c0 < end; c0 += chunk) {
        const int c1 = min(c0 + chunk, end);
        if (BIAS) {
            __syncthreads();  // the last chunk's biases have been read
            for (int j = c0 + int(threadIdx.x); j < c1; j += kThreads) {
                const float *row = f.a.bias.table + bucket_of(f.o, f.a.bias, place_k(f.o, j), pos_y, pos_x);
                for (int h = 0; h < tk.heads_per_block; ++h)
#pragma unroll
                    for (int i = 0; i < GRP; ++i) {
                        const int head = (kvb * tk.heads_per_block + h) * group + gb * GRP + i;
                        if (i < heads_here && head < g.heads)
                            bias_lds[(h * GRP + i) * tk.chunk + j - c0] = in_log2(row[int64_t(head) * nb]);
                    }
            }
            __syncthreads();
        }
        if (!active)
            continue;
        for (int j = c0 + slot; j < c1; j += round) {
            frag k[U], v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int t = j + u * tk.slots;
                const int n = t < c1 ? valid : 0;
                k[u] = load_chunk<T>(n > 0 ? km.at(t, d) : km.p, n, km.vec);
                v[u] = load_chunk<T>(n > 0 ? vm.at(t, d) : vm.p, n, vm.vec);
            }
            float s[U][GRP];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const f32x8 kf = to_f32(k[u]);
#pragma unroll
                for (int i = 0; i < GRP; ++i) {
                    float x = 0.0f;
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        x = fmaf(kf[e], q[i][e], x);
                    s[u][i] = lanes_sum<G>(x);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int t = j + u * tk.slots;
#pragma unroll
                for (int i = 0; i < GRP; ++i) {
                    if (BIAS)
                        s[u][i] += bias_lds[(pair % tk.heads_per_block * GRP + i) * tk.chunk + min(t, c1 - 1) - c0];
                    if (t >= c1)
                        s[u][i] = -INFINITY;
                }
            }
#pragma unroll
            for (int i = 0; i < GRP; ++i) {
                float now = top[i];
#pragma unroll
                for (int u = 0; u < U; ++u)
                    now = fmaxf(now, s[u][i]);
                const float m = now == -INFINITY ? 0.0f : now;
                const float back = exp2_fast(top[i] - m);
                top[i] = now;
                sum[i] *= back;
                o[i] *= back;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    s[u][i] = exp2_fast(s[u][i] - m);
                    sum[i] += s[u][i];
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const f32x8 vf = to_f32(v[u]);
#pragma unroll
                for (int i = 0; i < GRP; ++i)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        o[i][e] = fmaf(s[u][i], vf[e], o[i][e]);
            }
        }
    }
    // the slots' results joined, a thread per real of a head
    __syncthreads();
#pragma unroll
    for (int i = 0; i < GRP; ++i) {
        const int at = pair * GRP + i;
        *reinterpret_cast<f32x8 *>(acc_lds + at * DP + d) = o[i];
        if (d == 0) {
            stat_lds[2 * at] = top[i];
            stat_lds[2 * at + 1] = sum[i];
        }
    }
    __syncthreads();
    const int64_t rows = int64_t(g.n) * g.heads;
    for (int e = threadIdx.x; e < tk.heads_per_block * GRP * DP; e += kThreads) {
        const int real = e % DP, i = e / DP % GRP, h = e / DP / GRP;
        const int kvh = kvb * tk.heads_per_block + h, head = kvh * group + gb * GRP + i;
        if (kvh >= g.kv_heads || i >= heads_here)
            continue;
        float m = -INFINITY;
        for (int w = 0; w < tk.slots; ++w)
            m = fmaxf(m, stat_lds[2 * ((w * tk.heads_per_block + h) * GRP + i)]);
        const float base = m == -INFINITY ? 0.0f : m;
        float total = 0.0f, value = 0.0f;
        for (int w = 0; w < tk.slots; ++w) {
            const int at = (w * tk.heads_per_block + h) * GRP + i;
            const float x = exp2_fast(stat_lds[2 * at] - base);
            total = fmaf(x, stat_lds[2 * at + 1], total);
            value = fmaf(x, acc_lds[at * DP + real], value);
        }
        const int64_t row = int64_t(img) * g.heads + head;
        if (f.splits > 1) {
            f.part[(split * rows + row) * DP + real] = value;
            if (real == 0) {
                f.part_stats[(split * rows + row) * 2] = m;
                f.part_stats[(split * rows + row) * 2 + 1] = total;
            }
            continue;
        }
        finish_real<T, DQP>(f, row, real, value, base, total);
    }
}

// ---------------------------------------------------------------------- host

struct Plan {
    int blocks, splits, tiles_per_split, cap;
    size_t lds;
    Token token;  // one query
    int grp;
};

// may_split: there is memory for partial results.
Plan forward_plan(const AttnCall &a, DType dt, bool may_split = true)
{
    const AttnGeom &g = a.g;
    const int es = dt == DType::BF16 ? 2 : 4, tile = dt == DType::BF16 ? 64 : 32, dp = 4 * padded_dq(g.dq);
    Plan p{};
    const int lq = g.lq();
    if (lq == 1) {
        // one query: heads of a token side by side
        const int group = g.heads / g.kv_heads;
        p.grp = group == 1 ? 1 : group == 2 ? 2 : 4;
        const int pairs = kThreads / (dp / 8);
        p.token.heads_per_block = std::min(g.kv_heads, pairs);
        p.token.slots = pairs / p.token.heads_per_block;
        p.token.kv_blocks = (g.kv_heads + p.token.heads_per_block - 1) / p.token.heads_per_block;
        p.token.group_blocks = (group + p.grp - 1) / p.grp;
        p.blocks = 1;
        // (biases of a work-group's heads for a chunk of keys fill the LDS array)
        p.token.chunk = kTokenBias / (p.token.heads_per_block * p.grp);
        // up to four rounds of keys in one work-group (40 x 483 keys: 15 us,
        // 22 with two launches); beyond that, where the chip has room, two at
        // least to each of several (64 x 400 keys: 12.6 + 3.6 us, 29.6 in one;
        // 4 x 65536: 27 + 4, 3100 in one)
        const int64_t groups = int64_t(g.n) * p.token.kv_blocks * p.token.group_blocks;
        const int rounds = (g.lk() + kTokenUnroll * p.token.slots - 1) / (kTokenUnroll * p.token.slots);
        const int64_t room = 1024 / groups;
        p.splits = may_split && rounds > 4 ? int(std::max<int64_t>(1, std::min<int64_t>(room, (rounds + 1) / 2))) : 1;
        return p;
    }
    p.blocks = (lq + kQueries - 1) / kQueries;
    const int64_t groups = int64_t(g.n) * g.heads * p.blocks;
    const int tiles = (g.lk() + tile - 1) / tile;
    // fewer work-groups than compute units: the keys are dealt out too, two tiles
    // at least to each (one image of 40 x 40, 4 heads of 64: 20 us and 7 of joining,
    // 58 in one piece; 2 of 20 x 20: 12.5 and 4.5, 22 in one)
    p.splits = 1;
    if (groups < 256 && may_split)
        p.splits = int(std::max<int64_t>(1, std::min<int64_t>(512 / groups, tiles / 2)));
    p.tiles_per_split = (tiles + p.splits - 1) / p.splits;
    p.splits = (tiles + p.tiles_per_split - 1) / p.tiles_per_split;
    const size_t tiles_bytes = size_t(4) * tile * (dp + (es == 2 ? 0 : 4)) * es + size_t(2) * tile * 4;
    p.cap = 0;
    if (a.bias.table != nullptr) {
        const Offsets o = make_offsets(g);
        // the widest range of offsets that a tile of queries and one of keys have
        const int window = place_span(std::min(kQueries, lq), g.wq, g.hq, o.skip_q) +
                           place_span(tile, g.wk, g.hk, o.skip_k) + 8;
        p.cap = segment_cap(window, tiles_bytes, 4);
        if (p.cap < o.total && p.cap < 2048)
            p.cap = 2048;
    }
    p.lds = tiles_bytes + size_t(p.cap) * 4;
    return p;
}

template <typename T, int DQP, int MODE>
hipError_t forward_launch(const Forward &f, const Plan &p, hipStream_t s)
{
    const AttnGeom &g = f.a.g;
    const unsigned grid = xcd_grid(int64_t(g.n) * g.heads * p.splits * p.blocks);
    constexpr int kParts = sizeof(T) == 2 ? 3 : 1;
    if (f.rest != nullptr)
        attention_forward_kernel<T, DQP, MODE, kParts><<<grid, kThreads, p.lds, s>>>(f);
    else
        attention_forward_kernel<T, DQP, MODE, 1><<<grid, kThreads, p.lds, s>>>(f);
    if (hipError_t e = hipGetLastError())
        return e;
    if (p.splits > 1) {
        attention_join_kernel<T, DQP><<<unsigned(int64_t(g.n) * g.heads * g.lq()), 256, 0, s>>>(f);
    }
    return hipGetLastError();
}
template <typename T, int DQP, int GRP> hipError_t token_launch(const Forward &f, const Plan &p, hipStream_t s)
{
    const AttnGeom &g = f.a.g;
    const unsigned grid = unsigned(int64_t(g.n) * p.token.kv_blocks * p.token.group_blocks * p.splits);
    if (f.a.bias.table != nullptr)
        attention_token_kernel<T, DQP, GRP, true><<<grid, kThreads, 0, s>>>(f, p.token);
    else
        attention_token_kernel<T, DQP, GRP, false><<<grid, kThreads, 0, s>>>(f, p.token);
    if (hipError_t e = hipGetLastError())
        return e;
    if (p.splits > 1) {
        attention_join_kernel<T, DQP><<<unsigned(int64_t(g.n) * g.heads), 256, 0, s>>>(f);
    }
    return hipGetLastError();
}
template <typename T, int DQP> hipError_t forward_mode(const Forward &f, const Plan &p, hipStream_t s)
{
    if (f.a.g.lq() == 1)
        return p.grp == 1 ? token_launch<T, DQP, 1>(f, p, s)
                          : p.grp == 2 ? token_launch<T, DQP, 2>(f, p, s) : token_launch<T, DQP, 4>(f, p, s);
    if (f.a.bias.table == nullptr)
        return forward_launch<T, DQP, 0>(f, p, s);
    // (four keys of a row have biases side by side: 275 us for 16 x 40 x 40, 283
    // key by key; 302 and 322 for 2 x 80 x 80 with 128 reals a head)
    if (f.a.g.hk == 1 || f.a.g.wk % 4 == 0)
        return forward_launch<T, DQP, 1>(f, p, s);
    return forward_launch<T, DQP, 2>(f, p, s);
}
template <typename T> hipError_t forward_dq(const Forward &f, const Plan &p, hipStream_t s)
{
    switch (padded_dq(f.a.g.dq)) {
    case 8:
        return forward_mode<T, 8>(f, p, s);
    case 16:
        return forward_mode<T, 16>(f, p, s);
    default:
        return forward_mode<T, 32>(f, p, s);
    }
}

// The maps that are copied: a map per z, its images along y (several to a
// work-group where they are small: `threads` take one, a power of two), and along x
// 8 reals of a head's row per thread, the heads of a token side by side as they lie
// in the map.  (16 images of 40 x 40, 8 heads of 12 channels: 42 us, 76 head by
// head.)  Of keys and values only what the images have is read: 64 tokens in a
// cache of 4 million, heads of 10 channels, 35 us for the call, 1336 when all of
// it was.  (An image's rows of all heads are less than 2^31: their copy would be
// larger than the memory.)
template <typename T, int DQP>
__global__ void __launch_bounds__(256) attention_pack_kernel(AttnPack p, int n, int dq, int threads)
{
    constexpr int DP = 4 * DQP, kChunks = DP / 8;
    const int d = 8 * int(threadIdx.x % kChunks), per = 256 / threads;
    const int first = int((blockIdx.x * threads + (threadIdx.x & (threads - 1))) / kChunks);
    const int step = int(gridDim.x * threads / kChunks);
#pragma unroll
    for (int m = 0; m < AttnPack::kMaps; ++m) {
        if (m != int(blockIdx.z))
            continue;
        const int heads = p.heads[m];
        for (int img = int(blockIdx.y) * per + int(threadIdx.x) / threads; img < n; img += int(gridDim.y) * per) {
            T *dst = static_cast<T *>(p.dst[m]) + int64_t(img) * heads * p.tokens[m] * DP + d;
            const int tokens = p.kv_len[m] != nullptr ? min(max(p.kv_len[m][img], 0), p.tokens[m]) : p.tokens[m];
            const int64_t rows = int64_t(tokens) * heads;
            for (int64_t row = first; row < rows; row += step) {
                const int token = fast_div(int(row), p.by_heads[m]), head = int(row) - token * heads;
                const HeadMap<T, DQP> src(p.src[m], img, head, dq);
                *reinterpret_cast<typename Elem<T>::frag *>(dst + (int64_t(head) * p.tokens[m] + token) * DP) =
                    src.load(token, d, true);
            }
        }
    }
}

size_t packed_bytes(int n, int heads, int tokens, int dq, DType dt)
{
    return size_t(n) * heads * tokens * 4 * padded_dq(dq) * (dt == DType::BF16 ? 2 : 4);
}

bool whole_maps(const AttnCall &a)
{
    return a.q.vec && a.k.vec && a.v.vec && padded_dq(a.g.dq) == a.g.dq;
}

}  // namespace

hipError_t attention_pack_run(const AttnPack &p, int n, int dq, DType dt, hipStream_t s)
{
    const int dqp = padded_dq(dq);
    int64_t chunks = 1;
    for (int m = 0; m < p.maps; ++m)
        chunks = std::max(chunks, int64_t(p.heads[m]) * p.tokens[m] * (dqp / 2));
    int threads = dqp / 2;
    while (threads < 256 && threads < chunks)
        threads *= 2;
    // (work-groups for several rounds of the chip, each with as many turns as it takes)
    const dim3 grid(unsigned(std::min((chunks + 255) / 256, std::max<int64_t>(1, 24576 / (int64_t(n) * p.maps)))),
                    unsigned(std::min<int64_t>((int64_t(n) * threads + 255) / 256, 65535)), unsigned(p.maps));
    if (dt == DType::BF16) {
        if (dqp == 8)
            attention_pack_kernel<__bf16, 8><<<grid, 256, 0, s>>>(p, n, dq, threads);
        else if (dqp == 16)
            attention_pack_kernel<__bf16, 16><<<grid, 256, 0, s>>>(p, n, dq, threads);
        else
            attention_pack_kernel<__bf16, 32><<<grid, 256, 0, s>>>(p, n, dq, threads);
    } else {
        if (dqp == 8)
            attention_pack_kernel<float, 8><<<grid, 256, 0, s>>>(p, n, dq, threads);
        else if (dqp == 16)
            attention_pack_kernel<float, 16><<<grid, 256, 0, s>>>(p, n, dq, threads);
        else
            attention_pack_kernel<float, 32><<<grid, 256, 0, s>>>(p, n, dq, threads);
    }
    return hipGetLastError();
}

size_t attention_forward_work_bytes(const AttnCall &a, DType dt)
{
    const AttnGeom &g = a.g;
    if (g.lq() == 1 || whole_maps(a))
        return 0;
    return packed_bytes(g.n, g.heads, g.lq(), g.dq, dt) + 2 * packed_bytes(g.n, g.kv_heads, g.lk(), g.dq, dt);
}

size_t attention_forward_extra_bytes(const AttnCall &a, DType dt)
{
    const Plan p = forward_plan(a, dt);
    if (p.splits == 1)
        return 0;
    const size_t rows = size_t(a.g.n) * a.g.heads * a.g.lq();
    return size_t(p.splits) * rows * (4 * padded_dq(a.g.dq) + 2) * sizeof(float);
}

bool attention_forward_fits(const AttnCall &a, DType dt)
{
    return forward_plan(a, dt).lds <= kLdsLimit;
}

hipError_t attention_forward_run(const AttnCall &a, DType dt, const AttnMap &out, void *rest, float *stats, void *work,
                                 void *extra, hipStream_t s)
{
    const Plan p = forward_plan(a, dt, extra != nullptr);
    const AttnGeom &g = a.g;
    Forward f;
    f.a = a;
    if (work != nullptr) {
        AttnPack pack;
        unsigned char *at = static_cast<unsigned char *>(work);
        pack.maps = 0;
        for (AttnMap *m : {&f.a.q, &f.a.k, &f.a.v}) {
            const bool q = m == &f.a.q;
            const int i = pack.maps++;
            pack.src[i] = *m;
            pack.kv_len[i] = q ? nullptr : a.kv_len;
            pack.heads[i] = q ? g.heads : g.kv_heads;
            pack.by_heads[i] = FastDiv(pack.heads[i]);
            pack.tokens[i] = q ? g.lq() : g.lk();
            pack.dst[i] = at;
            const int64_t d = 4 * padded_dq(g.dq);
            *m = {at, int64_t(pack.heads[i]) * pack.tokens[i] * d, d, d / 4, true, pack.tokens[i] * d};
            at += packed_bytes(g.n, pack.heads[i], pack.tokens[i], g.dq, dt);
        }
        if (hipError_t e = attention_pack_run(pack, g.n, g.dq, dt, s))
            return e;
    }
    f.o = make_offsets(g);
    f.o.cap = p.cap;
    f.out = out;
    f.rest = rest;
    f.stats = stats;
    f.blocks = p.blocks;
    f.splits = p.splits;
    f.tiles_per_split = p.tiles_per_split;
    f.part = static_cast<float *>(extra);
    f.part_stats = f.part + (p.splits > 1 ? size_t(p.splits) * g.n * g.heads * g.lq() * 4 * padded_dq(g.dq) : 0);
    return dt == DType::BF16 ? forward_dq<__bf16>(f, p, s) : forward_dq<float>(f, p, s);
}

}  // namespace quan
