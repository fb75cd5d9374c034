// The gradients of attention between the pixels of quaternion maps on gfx950.
//
// With P the probabilities, recomputed from the rows' saved maxima and sums,
//   dP = dO V^T,  delta_i = dO_i . O_i,  dS = P (dP - delta),
//   dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO,
//   dtable[head][b] = sum of dS over the pairs of pixels in bucket b.
// Two launches, so that every sum has one owner and a fixed order: the first
// takes blocks of queries and walks over the keys (dQ, delta, and the sums of
// dS by offset), the second blocks of keys and walks over the queries of the
// heads that share them (dK, dV).  Where there are few blocks, several
// work-groups share a block's walk, and a third launch adds up their results.
// One or two more bring the sums by offset to buckets, in fp64; where the sums of
// all blocks of queries would take too much memory, the first launch and theirs
// come in turns.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "attention_tile.h"

namespace quan {
namespace {

struct Backward {
    AttnCall a;
    Offsets o;
    AttnMap out, rest, dout, dq, dk, dv;  // (rest.data may be NULL)
    const float *stats;
    float *delta;    // [n][heads][lq]
    // sums of dS by offset, [rows][q_splits][range]: a work-group's entries are those
    // between its queries and its share of the keys, from the lowest on; NULL: none
    // asked for
    float *offsets;
    int blocks, range;
    // the launch's blocks of queries, counted by image, head and block
    int first_row, rows;
    // work-groups that share a block of queries, of keys; the tiles of each
    int q_splits, k_splits, q_tiles, k_tiles;
    int q_span;  // tokens of q_tiles
    float *part_q, *part_k, *part_v;  // [split][row][D] where shared
};

constexpr int kWaves = 4, kThreads = 64 * kWaves, kQueries = 32 * kWaves;

// Sums of dS by offset in 64-bit fixed point: integer additions in LDS take 7
// clocks a wave where those of floats take 194 (measured), and their order
// changes nothing, so that the waves share one array.  Its units 2^-k follow
// from a bound of the terms known before they are: |dS| <= |dP - delta| <= (sum of
// |dO|'s elements) max |v| + |delta|, with the largest such sum and |delta| of the
// work-group's rows and the tile's largest element of v (no squares: they leave
// fp32 long before dO does).  k = kSumBits - e for a bound below 2^e: an
// offset's terms (one per query, 128) stay below 2^50, and a term's last place
// is 2^-42 of the bound.  A tile with a larger bound takes the array to coarser
// units.  What NaN or infinity is in the work-group's rows or in v, and a bound
// beyond fp32, gives NaN.
//
// Adding 1.5 * 2^52 to a term brings it, rounded, to the low bits of a double;
// those bits are added as they are, the constant with them: it is a multiple of
// 2^51, so that the sum is what its low 51 bits say.
constexpr int kSumBits = 42, kNoUnits = 127, kBadUnits = 128;
constexpr double kRound = 6755399441055744.0;
__device__ __forceinline__ void add_fixed(long long *entry, float v, double scale)
{
    const double t = fma(double(v), scale, kRound);
    __hip_atomic_fetch_add(reinterpret_cast<unsigned long long *>(entry), __builtin_bit_cast(unsigned long long, t),
                           __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
}
__device__ __forceinline__ long long fixed_sum(long long entry)
{
    return (long long)((unsigned long long)entry << 13) >> 13;
}
// The larger of two values >= 0; as unsigned numbers such floats keep their
// order, and NaN is above infinity.
__device__ __forceinline__ float bits_max(float a, float b)
{
    return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b)));
}
// Largest |value| of a wave, in all its lanes.
__device__ __forceinline__ float wave_top(float x)
{
    unsigned v = __float_as_uint(x) & 0x7fffffffu;
#define QUAN_DPP_MAX(ctrl) v = max(v, unsigned(__builtin_amdgcn_update_dpp(0, int(v), ctrl, 0xf, 0xf, false)))
    QUAN_DPP_MAX(0xB1);   // lane ^ 1
    QUAN_DPP_MAX(0x4E);   // lane ^ 2
    QUAN_DPP_MAX(0x141);  // 7 - lane of 8
    QUAN_DPP_MAX(0x140);  // 15 - lane of 16
#undef QUAN_DPP_MAX
    v = max(v, unsigned(__shfl_xor(int(v), 16, 64)));
    v = max(v, unsigned(__shfl_xor(int(v), 32, 64)));
    return __uint_as_float(v);
}
// |largest| of this thread's chunks of a tile, as wave_top takes it.
template <typename F, int N> __device__ __forceinline__ float chunk_top(const F (&r)[N])
{
    unsigned v = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const f32x8 t = to_f32(r[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v = max(v, __float_as_uint(t[e]) & 0x7fffffffu);
    }
    return __uint_as_float(v);
}

// A D x 32 tile of accumulators, transposed, to a row of fp32.
template <int DP>
__device__ __forceinline__ void store_part(float *dst, const f32x16 (&v)[DP / 32], int half, bool here)
{
    if (!here)
        return;
#pragma unroll
    for (int i = 0; i < DP / 32; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const f32x4 t = {v[i][4 * g], v[i][4 * g + 1], v[i][4 * g + 2], v[i][4 * g + 3]};
            *reinterpret_cast<f32x4 *>(dst + 32 * i + 8 * g + 4 * half) = t;
        }
}

// The launch of the queries' side.  Sums of dS by offset are gathered over the
// segment whose biases are staged; as the walk leaves it they go to the
// work-group's own row of `offsets`.  16 images of 40 x 40, 8 heads of 64 reals:
// 343 us, 370 TFLOP/s of its three products, 190 us without a bias: an addition and
// a quarter of a bias in LDS per pair are the rest.  2.2 waves a SIMD wait 49 % of
// their time (vector instructions 43 %, LDS 38 %, matrix units 17 %).  32 of 14 x
// 14, 16 heads: 66 us (a tile of 64 keys in four has 4; 1.7 waves, 60 %).  Three
// waves a SIMD spill 7 registers a lane, 16 where places are looked up one by one;
// two, which spill none, take 380 us for the first (56 for the second).  dS meets k
// rounded to bf16, off by 2^-8 of a term at most, as dq is once it is rounded.
template <typename T, int DQP, int MODE>
__global__ void __launch_bounds__(kThreads, DQP <= 16 ? 3 : 1) attention_dq_kernel(Backward f)
{
    constexpr int DP = 4 * DQP;
    typedef Stage<T, DP, kThreads> Tile;
    typedef typename Elem<T>::frag frag;
    constexpr int KT = Tile::kTokens, SUBS = KT / 32;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds_raw[];
    float *bias = reinterpret_cast<float *>(lds_raw);  // (at 0: its reads then have their offsets in the instruction)
    long long *sums = reinterpret_cast<long long *>(bias + f.o.cap);
    int *place = reinterpret_cast<int *>(sums + (f.offsets != nullptr ? f.o.cap : 0));
    T *k_lds = reinterpret_cast<T *>(place + 2 * KT), *v_lds = k_lds + 2 * Tile::kElems;
    __shared__ float tops[2 * kWaves];  // of a tile's v, by buffer and wave

    const AttnGeom &g = f.a.g;
    const int lq = g.lq(), lk = g.lk();
    const int total = f.rows * f.q_splits;
    int id = xcd_order(total);
    if (id >= total)
        return;
    id += f.first_row;  // (0 with several splits)
    const int block = id % f.blocks;
    id /= f.blocks;
    const int split = id % f.q_splits;
    id /= f.q_splits;
    const int head = id % g.heads, img = id / g.heads;
    const int kv_head = head / (g.heads / g.kv_heads);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
    const int half_at = KT / 2 * half;  // the lane's half of a tile
    const int q0 = block * kQueries, query = q0 + 32 * wave + (lane & 31);
    const bool q_here = query < lq;
    const int len = f.a.kv_len != nullptr ? min(max(f.a.kv_len[img], 0), lk) : lk;
    const int begin = split * f.q_span, end = min(len, begin + f.q_span);
    const int64_t row = (int64_t(img) * g.heads + head) * lq + query;

    const WholeMap<T, DQP> qm(f.a.q, img, head), km(f.a.k, img, kv_head), vm(f.a.v, img, kv_head);
    Tile kt, vt;
    if (begin < end) {
        kt.fetch(km, begin, end);
        vt.fetch(vm, begin, end);
    }
    frag q[DP / 16], go[DP / 16];
    float delta = 0.0f;
    {
        const WholeMap<T, DQP> gm(f.dout, img, head), om(f.out, img, head), rm(f.rest, img, head);
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) {
            const int d = 16 * i + 8 * half;
            q[i] = qm.load(query, d, q_here);
            go[i] = gm.load(query, d, q_here);
            const frag rounded = om.load(query, d, q_here);
            const f32x8 o = f.rest.data != nullptr ? with_rest(rounded, rm.load(query, d, q_here)) : to_f32(rounded);
            const f32x8 w = to_f32(go[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                delta = fmaf(w[e], o[e], delta);
        }
        delta = half_sum(delta);
        if (q_here && half == 0 && split == 0)
            f.delta[row] = delta;
    }
    // P = 2^(s - top) inv; rows without a key, and none, have P = 0
    const float sum = q_here ? f.stats[2 * row + 1] : 0.0f;
    const bool empty = sum == 0.0f;
    const float top = empty ? INFINITY : f.stats[2 * row];
    const float inv = empty ? 0.0f : 1.0f / sum;
    const float shift = empty ? 0.0f : -delta * inv;
    const float c = g.scale * kLog2e;

    int pos_y = 0, pos_x = 0, lane_at = 0, low_q = 0, high_q = 0, segment = -1, done = 0;
    const float *table = nullptr;
    float *offsets = nullptr;
    if (MODE != 0) {
        if (f.a.pos != nullptr) {
            pos_y = query_pos(f.a.pos[2 * img]);
            pos_x = query_pos(f.a.pos[2 * img + 1]);
        }
        table = f.a.bias.table + int64_t(head) * f.a.bias.ny * f.a.bias.nx;
        low_q = f.o.origin - place_q(f.o, min(q0 + kQueries, lq) - 1);
        high_q = f.o.origin - place_q(f.o, q0);
        lane_at = f.o.origin - place_q(f.o, min(query, lq - 1));
        done = low_q + place_k(f.o, begin);
        if (f.offsets != nullptr)
            offsets = f.offsets + (int64_t((img * g.heads + head) * f.blocks + block - f.first_row) * f.q_splits + split) * f.range - done;
    }
    // past the last offset to this work-group's keys
    const int past = MODE != 0 ? high_q + place_k(f.o, min(begin + f.q_span, lk) - 1) + 1 : 0;
    auto start_segment = [&](int lo) {
        segment = lo;
        const int count = min(f.o.cap, past + 3 - segment);  // (a quad may pass the last offset)
        stage_bias(bias, f.o, f.a.bias, table, segment, count, pos_y, pos_x);
        if (offsets != nullptr)
            for (int e = threadIdx.x; e < count; e += kThreads)
                sums[e] = 0;
    };
    if (MODE != 0 && begin < end)
        start_segment(low_q + place_k(f.o, begin));
    // the bound's parts from the work-group's rows: the sum of |dO| and |delta|; a
    // row whose sum of probabilities is no number has NaN
    float top_go = 0.0f, top_delta = 0.0f;
    if (MODE != 0 && offsets != nullptr) {
        float n1 = 0.0f;
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) {
            const f32x8 w = to_f32(go[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                n1 += fabsf(w[e]);
        }
        top_go = wave_top(sum <= -kLowest ? half_sum(n1) : NAN);
        top_delta = wave_top(delta);
        if (lane == 0) {
            tops[wave] = top_go;
            tops[kWaves + wave] = top_delta;
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            top_go = bits_max(top_go, tops[w]);
            top_delta = bits_max(top_delta, tops[kWaves + w]);
        }
        __syncthreads();
    }
    int units = kNoUnits;  // k of the array's units 2^-k
    double unit = 0.0;     // 2^k
    // Zeros to entries [from, to), and the segment's sums, added to the entries
    // that an earlier one has written: a thread has the same entries modulo
    // kThreads each time.
    auto own = [&](int from) {
        const int a = from - from % kThreads + int(threadIdx.x);
        return a < from ? a + kThreads : a;
    };
    auto clear = [&](int from, int to) {
        for (int a = own(from); a < to; a += kThreads)
            offsets[a] = 0.0f;
    };
    auto flush = [&]() {
        const int last = min(segment + f.o.cap, past);
        const double back = __longlong_as_double((long long)(1023 - units) << 52);  // 2^-units
        for (int a = own(segment); a < last; a += kThreads) {
            const float v = units == kBadUnits ? NAN : units == kNoUnits ? 0.0f : float(double(fixed_sum(sums[a - segment])) * back);
            offsets[a] = a < done ? offsets[a] + v : v;
        }
        done = max(done, last);
    };

    f32x16 dq[DP / 32];
#pragma unroll
    for (int i = 0; i < DP / 32; ++i)
        dq[i] = 0.0f;
    int buf = 0;
    for (int j0 = begin; j0 < end; j0 += KT, buf ^= 1) {
        T *kb = k_lds + buf * Tile::kElems, *vb = v_lds + buf * Tile::kElems;
        int *pl = place + buf * KT;
        kt.put(kb);
        vt.put(vb);
        if (MODE != 0 && offsets != nullptr) {
            const float most = wave_top(chunk_top(vt.r));
            if (lane == 0)
                tops[buf * kWaves + wave] = most;
        }
        if (MODE != 0) {
            if (threadIdx.x < KT)
                pl[threadIdx.x] = place_k(f.o, min(j0 + int(threadIdx.x), lk - 1));
            const int lo = low_q + place_k(f.o, j0), hi = high_q + place_k(f.o, min(j0 + KT, lk) - 1) + 3;
            if (hi >= segment + f.o.cap) {
                __syncthreads();  // the last segment has been read and added to
                if (offsets != nullptr) {
                    flush();
                    if (lo > done) {  // (a row of keys ended: offsets that the block has to none)
                        clear(done, lo);
                        done = lo;
                    }
                }
                __syncthreads();
                start_segment(lo);
            }
        }
        __syncthreads();
        if (j0 + KT < end) {
            kt.fetch(km, j0 + KT, end);
            vt.fetch(vm, j0 + KT, end);
        }
        if (MODE != 0 && offsets != nullptr) {
            float most = 0.0f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w)
                most = bits_max(most, tops[buf * kWaves + w]);
            most = fmaf(most, top_go, top_delta);
            if (!(most <= -kLowest)) {
                units = kBadUnits;
                unit = 0.0;
            } else if (units != kBadUnits) {
                const int e = int(__float_as_uint(most) >> 23) - 126;  // most < 2^e
                const int now = min(kSumBits - e, kNoUnits - 1);
                if (now < units) {
                    if (units != kNoUnits) {  // (what other waves add meanwhile waits for the barriers)
                        __syncthreads();
                        for (int i = threadIdx.x; i < f.o.cap; i += kThreads)
                            sums[i] = fixed_sum(sums[i]) >> min(units - now, 63);
                        __syncthreads();
                    }
                    units = now;
                    unit = __longlong_as_double((long long)(1023 + now) << 52);
                }
            }
        }
        if (q0 + 32 * wave >= lq)
            continue;  // (none of the wave's queries is there)
        const int at = lane_at - segment;
#pragma unroll
        for (int sub = 0; sub < SUBS; ++sub) {
            if (16 * sub >= end - j0)
                break;
            f32x16 s = 0.0f, dp = 0.0f;
#pragma unroll
            for (int i = 0; i < DP / 16; ++i) {
                s = mma(row_frag<T, DP>(kb, sub, i), q[i], s);
                dp = mma(row_frag<T, DP>(vb, sub, i), go[i], dp);
            }
            add_bias<MODE, 1>(s, c, bias, pl, at, half_at, sub);
#pragma unroll
            for (int r = 0; r < 16; ++r)
                s[r] = exp2_fast(s[r] - top) * fmaf(dp[r], inv, shift);
            if (j0 + KT > end)
                clear_behind(s, end - j0 - half_at, sub, 0.0f);
            // (lanes without a query would all add to the last one's offsets, and
            // such additions take their turns: 5 of a small launch's 17 us)
            if (MODE != 0 && offsets != nullptr && q_here) {
#pragma unroll
                for (int gq = 0; gq < 4; ++gq) {
                    const i32x4 p4 = places<MODE>(pl, half_at, sub, gq);
#pragma unroll
                    for (int t = 0; t < 4; ++t)
                        add_fixed(sums + at + p4[t], s[4 * gq + t], unit);
                }
            }
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                const frag p = acc_frag<T>(s, st);
#pragma unroll
                for (int i = 0; i < DP / 32; ++i)
                    dq[i] = mma(col_frag<DP>(kb, sub, st, i), p, dq[i]);
            }
        }
    }
    if (f.q_splits > 1) {
        const int64_t rows = int64_t(g.n) * g.heads * lq;
        store_part<DP>(f.part_q + (split * rows + row) * DP, dq, half, q_here);
    } else {
        const HeadMap<T, DQP> om(f.dq, img, head, g.dq);
#pragma unroll
        for (int i = 0; i < DP / 32; ++i) {
            dq[i] *= g.scale;
            om.store(query, i, half, dq[i], q_here);
        }
    }
    if (MODE != 0 && offsets != nullptr) {
        if (segment >= 0) {
            __syncthreads();
            flush();
        }
        clear(done, past);  // entries of keys that the image has not
    }
}

// The launch of the keys' side: lanes hold keys, registers queries.  Bound by what
// two waves a SIMD, all that its accumulators leave room for, wait for: 16 images of
// 40 x 40, 8 heads of 64 reals, 330 us, 510 TFLOP/s of its four products (45 % of
// 1.6 waves' time; vector instructions and LDS 34 %, matrix units 23 %); 32 of 14 x
// 14, 16 heads, 47 us.  P meets dout and dS meets q rounded to bf16, off by 2^-8 of a
// term at most, as dv and dk are once they are rounded.
constexpr int kNoSegment = -(1 << 30);
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
template <typename T, int DQP, int MODE>
__global__ void __launch_bounds__(kThreads, DQP <= 16 ? 2 : 1) attention_dkv_kernel(Backward f)
{
    constexpr int DP = 4 * DQP;
    typedef Stage<T, DP, kThreads> Tile;
    typedef typename Elem<T>::frag frag;
    constexpr int QT = Tile::kTokens, SUBS = QT / 32;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds_raw[];
    float *bias = reinterpret_cast<float *>(lds_raw);  // (at 0: its reads then have their offsets in the instruction)
    float *rows = bias + f.o.cap;                      // [2][top, inv, -delta][QT]
    int *place = reinterpret_cast<int *>(rows + 6 * QT);
    T *q_lds = reinterpret_cast<T *>(place + 2 * QT), *g_lds = q_lds + 2 * Tile::kElems;

    const AttnGeom &g = f.a.g;
    const int lq = g.lq(), lk = g.lk(), group = g.heads / g.kv_heads;
    const int blocks = (lk + kQueries - 1) / kQueries;
    const int total = g.n * g.kv_heads * blocks * f.k_splits;
    int id = xcd_order(total);
    if (id >= total)
        return;
    const int block = id % blocks;
    id /= blocks;
    const int split = id % f.k_splits;
    id /= f.k_splits;
    const int kv_head = id % g.kv_heads, img = id / g.kv_heads;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
    const int half_at = QT / 2 * half;  // the lane's half of a tile
    const int k0 = block * kQueries, key = k0 + 32 * wave + (lane & 31);
    const int end = f.a.kv_len != nullptr ? min(max(f.a.kv_len[img], 0), lk) : lk;
    const bool k_here = key < end;

    const WholeMap<T, DQP> km(f.a.k, img, kv_head), vm(f.a.v, img, kv_head);
    frag k[DP / 16], v[DP / 16];
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) {
        k[i] = km.load(key, 16 * i + 8 * half, k_here);
        v[i] = vm.load(key, 16 * i + 8 * half, k_here);
    }
    f32x16 dk[DP / 32], dv[DP / 32];
#pragma unroll
    for (int i = 0; i < DP / 32; ++i) {
        dk[i] = 0.0f;
        dv[i] = 0.0f;
    }
    const float c = g.scale * kLog2e;
    int pos_y = 0, pos_x = 0, lane_at = 0, low_k = 0, high_k = 0;
    if (MODE != 0) {
        if (f.a.pos != nullptr) {
            pos_y = query_pos(f.a.pos[2 * img]);
            pos_x = query_pos(f.a.pos[2 * img + 1]);
        }
        low_k = f.o.origin + place_k(f.o, k0);
        high_k = f.o.origin + place_k(f.o, min(k0 + kQueries, lk) - 1);
        lane_at = f.o.origin + place_k(f.o, min(key, lk - 1));
    }
    // The walk: tile by tile from the last, so that offsets ascend, head by head.
    const int tiles = (lq + QT - 1) / QT, first = split * f.k_tiles;
    const int last = k0 < end ? min(group * tiles, first + f.k_tiles) : first;
    Tile qt, gt;
    float row_top = 0.0f, row_sum = 0.0f, row_delta = 0.0f;  // of thread t < QT's query of a tile
    auto fetch = [&](int item) {
        const int head = kv_head * group + item / tiles, i0 = (tiles - 1 - item % tiles) * QT;
        qt.fetch(WholeMap<T, DQP>(f.a.q, img, head), i0, lq);
        gt.fetch(WholeMap<T, DQP>(f.dout, img, head), i0, lq);
        if (threadIdx.x < QT) {
            const int i = i0 + threadIdx.x;
            const int64_t row = (int64_t(img) * g.heads + head) * lq + min(i, lq - 1);
            row_top = f.stats[2 * row];
            row_sum = i < lq ? f.stats[2 * row + 1] : 0.0f;
            row_delta = f.delta[row];
        }
    };
    if (first < last)
        fetch(first);
    int segment = kNoSegment, buf = 0;
    for (int item = first; item < last; ++item, buf ^= 1) {
        const int head = kv_head * group + item / tiles, i0 = (tiles - 1 - item % tiles) * QT;
        const float *table = MODE != 0 ? f.a.bias.table + int64_t(head) * f.a.bias.ny * f.a.bias.nx : nullptr;
        T *qb = q_lds + buf * Tile::kElems, *gb = g_lds + buf * Tile::kElems;
        int *pl = place + buf * QT;
        float *rw = rows + buf * 3 * QT;
        qt.put(qb);
        gt.put(gb);
        if (threadIdx.x < QT) {
            const bool empty = row_sum == 0.0f;
            rw[threadIdx.x] = empty ? INFINITY : row_top;
            rw[QT + threadIdx.x] = empty ? 0.0f : 1.0f / row_sum;
            rw[2 * QT + threadIdx.x] = empty ? 0.0f : -row_delta;
            if (MODE != 0)
                pl[threadIdx.x] = place_q(f.o, min(i0 + int(threadIdx.x), lq - 1));
        }
        if (MODE != 0) {
            const int lo = low_k - place_q(f.o, min(i0 + QT, lq) - 1) - 3, hi = high_k - place_q(f.o, i0);
            if (segment == kNoSegment || hi >= segment + f.o.cap || item % tiles == 0) {
                if (segment != kNoSegment)
                    __syncthreads();
                segment = lo;  // (down to -3)
                stage_bias(bias, f.o, f.a.bias, table, segment, min(f.o.cap, high_k + 1 - segment), pos_y, pos_x);
            }
        }
        __syncthreads();
        if (item + 1 < last)
            fetch(item + 1);
        if (k0 + 32 * wave >= end)
            continue;  // (none of the wave's keys is there)
        f32x16 s[SUBS], dp[SUBS];
#pragma unroll
        for (int sub = 0; sub < SUBS; ++sub) {
            s[sub] = 0.0f;
            dp[sub] = row_values(rw + 2 * QT, half_at, sub);  // dP - delta starts from -delta
        }
#pragma unroll
        for (int i = 0; i < DP / 16; ++i)
#pragma unroll
            for (int sub = 0; sub < SUBS; ++sub) {
                s[sub] = mma(row_frag<T, DP>(qb, sub, i), k[i], s[sub]);
                dp[sub] = mma(row_frag<T, DP>(gb, sub, i), v[i], dp[sub]);
            }
#pragma unroll
        for (int sub = 0; sub < SUBS; ++sub) {
            add_bias<MODE, -1>(s[sub], c, bias, pl, lane_at - segment, half_at, sub);
            const f32x16 top = row_values(rw, half_at, sub), inv = row_values(rw + QT, half_at, sub);
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[sub][r] = exp2_fast(s[sub][r] - top[r]) * inv[r];
                dp[sub][r] *= s[sub][r];
            }
        }
#pragma unroll
        for (int sub = 0; sub < SUBS; ++sub)
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                const frag p = acc_frag<T>(s[sub], st), ds = acc_frag<T>(dp[sub], st);
#pragma unroll
                for (int i = 0; i < DP / 32; ++i) {
                    dv[i] = mma(col_frag<DP>(gb, sub, st, i), p, dv[i]);
                    dk[i] = mma(col_frag<DP>(qb, sub, st, i), ds, dk[i]);
                }
            }
    }
    // keys behind the image's last have no gradient
    if (!k_here)
#pragma unroll
        for (int i = 0; i < DP / 32; ++i) {
            dk[i] = 0.0f;
            dv[i] = 0.0f;
        }
    if (f.k_splits > 1) {
        const int64_t at = (split * int64_t(g.n) * g.kv_heads * lk + (int64_t(img) * g.kv_heads + kv_head) * lk + key) * DP;
        store_part<DP>(f.part_k + at, dk, half, key < lk);
        store_part<DP>(f.part_v + at, dv, half, key < lk);
        return;
    }
    const HeadMap<T, DQP> okm(f.dk, img, kv_head, g.dq), ovm(f.dv, img, kv_head, g.dq);
#pragma unroll
    for (int i = 0; i < DP / 32; ++i) {
        dk[i] *= g.scale;
        okm.store(key, i, half, dk[i], key < lk);
        ovm.store(key, i, half, dv[i], key < lk);
    }
}

// The results of work-groups that shared a block, added up in order: a thread
// per quad of reals.
template <typename T, int DQP> __global__ void __launch_bounds__(256) gradient_join_kernel(Backward f)
{
    constexpr int DP = 4 * DQP;
    const AttnGeom &g = f.a.g;
    int64_t id = int64_t(blockIdx.x) * 256 + threadIdx.x;
#pragma unroll
    for (int which = 0; which < 3; ++which) {
        const int splits = which == 0 ? f.q_splits : f.k_splits, heads = which == 0 ? g.heads : g.kv_heads;
        const int tokens = which == 0 ? g.lq() : g.lk();
        const int64_t rows = int64_t(g.n) * heads * tokens, quads = splits > 1 ? rows * (DP / 4) : 0;
        if (id < quads) {
            const float *p = (which == 0 ? f.part_q : which == 1 ? f.part_k : f.part_v) + id * 4;
            f32x4 s = 0.0f;
#pragma unroll 4
            for (int i = 0; i < splits; ++i)
                s += *reinterpret_cast<const f32x4 *>(p + i * rows * DP);
            if (which < 2)
                s *= g.scale;
            const int64_t row = id / (DP / 4);
            const int d = 4 * int(id % (DP / 4)), token = int(row % tokens), head = int(row / tokens % heads);
            const HeadMap<T, DQP> m(which == 0 ? f.dq : which == 1 ? f.dk : f.dv, row / tokens / heads, head, g.dq);
            store_quad(m.at(token, d), s, m.valid(d, 4), m.vec);
            return;
        }
        id -= quads;
    }
}

// The last key whose place is at most `place` >= 0, and the first whose place is
// at least that.
__device__ __forceinline__ int last_key(const Offsets &o, int place, int lk)
{
    const int w = o.pitch - o.skip_k, row = fast_div(place, o.by_pitch);
    return min(row * w + min(place - row * o.pitch, w - 1), lk - 1);
}
__device__ __forceinline__ int first_key(const Offsets &o, int place)
{
    const int w = o.pitch - o.skip_k, row = fast_div(max(place, 0), o.by_pitch);
    return row * w + min(max(place, 0) - row * o.pitch, w);
}

// Sum over images slice, slice + slices, .., blocks b0, b0 + step, .. and their
// work-groups of what offset `a` has in them, in a fixed order.  (Of those whose
// blocks the launch before has taken.)
__device__ __forceinline__ double offset_sum(const Backward &f, int head, int a, int slice, int slices, int b0, int step,
                                             int last_k)
{
    const AttnGeom &g = f.a.g;
    const int lq = g.lq();
    const int64_t image = int64_t(g.heads) * f.blocks * f.q_splits * f.range;
    double s = 0.0;
    for (int b = b0; b < f.blocks; b += step) {
        const int low = f.o.origin - place_q(f.o, min((b + 1) * kQueries, lq) - 1);
        const int high = f.o.origin - place_q(f.o, b * kQueries);
        if (a < low || a > high + last_k)
            continue;
        const int row = head * f.blocks + b, per_image = g.heads * f.blocks;  // of image 0
        const float *p = f.offsets + int64_t(row - f.first_row) * f.q_splits * f.range + (a - low);
        if (f.q_splits > 1) {  // (few images then; those that have the offset to one of their keys)
            const int sp0 = first_key(f.o, a - high) / f.q_span, sp1 = last_key(f.o, a - low, g.lk()) / f.q_span;
            for (int img = slice; img < g.n; img += slices)
#pragma unroll 8
                for (int sp = sp0; sp <= sp1; ++sp)
                    s += double(p[img * image + int64_t(sp) * f.range - place_k(f.o, sp * f.q_span)]);
        } else {
            int img = slice, end = g.n;
            if (f.rows < g.n * per_image) {  // images that have the block in the launch
                const int first = max((f.first_row - row + per_image - 1) / per_image, 0);
                end = min(max((f.first_row + f.rows - row + per_image - 1) / per_image, 0), end);
                img += (max(first - slice, 0) + slices - 1) / slices * slices;
            }
#pragma unroll 8
            for (; img < end; img += slices)
                s += double(p[img * image]);
        }
    }
    return s;
}

// Sums by offset of each slice of the images, in fp64: out [slices][heads][total],
// added to what is there where `more`.
// A lane per offset, the blocks and, where they are few, the images shared out
// among the waves: what bounds it are the chains of loads (one image of 1600
// queries, 4 heads: 9 us; 22 where a wave takes all of its offsets' blocks).
constexpr int kSumWaves = 4;
__global__ void __launch_bounds__(64 * kSumWaves) offset_sums_kernel(Backward f, int slices, bool more, double *__restrict__ out)
{
    __shared__ double parts[kSumWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int a = blockIdx.x * 64 + lane, head = blockIdx.y;
    const int last_k = place_k(f.o, f.a.g.lk() - 1);
    const int step = f.blocks >= 4 ? 4 : f.blocks >= 2 ? 2 : 1;
    static_assert(kSumWaves % 4 == 0, "waves share blocks and images evenly");
    for (int slice = blockIdx.z; slice < slices; slice += gridDim.z) {
        parts[wave][lane] = a < f.o.total ? offset_sum(f, head, a, slice + slices * (wave / step), slices * (kSumWaves / step),
                                                       wave % step, step, last_k)
                                          : 0.0;
        __syncthreads();
        if (wave == 0 && a < f.o.total) {
            double s = 0.0;
            for (int w = 0; w < kSumWaves; ++w)
                s += parts[w][lane];
            double *to = out + (int64_t(slice) * f.a.g.heads + head) * f.o.total + a;
            *to = more ? *to + s : s;
        }
        __syncthreads();
    }
}

// dtable from the sums by offset: a work-group per row of buckets (head, by),
// which takes columns dx of offsets in turn.  Its waves share the rows dy of that
// bucket out among them, a lane per column; then each wave adds up the columns of
// its buckets bx.  The slices have their offsets' buckets in common, but where
// queries have places of their own (pos): there a slice is an image, and they are
// taken one by one.  DIRECT: from the work-groups' sums themselves (few of them),
// one slice.
constexpr int kTableThreads = 512, kTableWaves = kTableThreads / 64, kTableCols = 128;
template <bool DIRECT>
__global__ void __launch_bounds__(kTableThreads)
table_gradient_kernel(Backward f, int rows, int slices, const double *__restrict__ sums, float *__restrict__ dtable)
{
    constexpr int kCols = kTableCols / 64;
    __shared__ double parts[kTableWaves][kTableCols];
    __shared__ short taken[kTableThreads];  // rows of that bucket among kTableThreads, in order
    __shared__ int counts[kTableWaves];
    __shared__ double tot[kAttnMaxBuckets];
    const AttnBias &b = f.a.bias;
    const Offsets &o = f.o;
    const int *pos = f.a.pos;
    const int heads = f.a.g.heads, iy = blockIdx.x % b.ny, head = blockIdx.x / b.ny;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, last_k = place_k(o, f.a.g.lk() - 1);
    for (int x = threadIdx.x; x < b.nx; x += kTableThreads)
        tot[x] = 0.0;
    const int groups = pos != nullptr ? slices : 1, per = slices / groups;
    for (int group = 0; group < groups; ++group) {
        const int pos_y = pos != nullptr ? query_pos(pos[2 * group]) : 0;
        const int pos_x = pos != nullptr ? query_pos(pos[2 * group + 1]) : 0;
        for (int x0 = 0; x0 < o.pitch; x0 += kTableCols) {
            double s[kCols] = {};
            for (int y0 = 0; y0 < rows; y0 += kTableThreads) {
                const int y = y0 + threadIdx.x, dy = min(max(y - o.hq1 - pos_y, -b.ry), b.ry);
                const bool here = y < rows && (b.by != nullptr ? min(max(b.by[dy + b.ry], 0), b.ny - 1) : 0) == iy;
                const unsigned long long mine = __ballot(here);
                __syncthreads();  // the last rows and columns have been read
                if (lane == 0)
                    counts[wave] = __popcll(mine);
                __syncthreads();
                int before = 0, all = 0;
                for (int w = 0; w < kTableWaves; ++w) {
                    before += w < wave ? counts[w] : 0;
                    all += counts[w];
                }
                if (here)
                    taken[before + __popcll(mine & ((1ull << lane) - 1))] = short(threadIdx.x);
                __syncthreads();
                // (row, slice) pairs in turn
#pragma unroll 4
                for (int i = wave; i < all * per; i += kTableWaves) {
                    const int r = i / per, sl = group * per + (i - r * per);
#pragma unroll
                    for (int c = 0; c < kCols; ++c) {
                        const int x = x0 + 64 * c + lane, a = (y0 + taken[r]) * o.pitch + x;
                        if (x < o.pitch)
                            s[c] += DIRECT ? offset_sum(f, head, a, sl, slices, 0, 1, last_k)
                                           : sums[(int64_t(sl) * heads + head) * o.total + a];
                    }
                }
            }
            int bucket[kCols];
#pragma unroll
            for (int c = 0; c < kCols; ++c) {
                parts[wave][64 * c + lane] = s[c];
                const int dx = min(max(x0 + 64 * c + lane - o.wq1 - pos_x, -b.rx), b.rx);
                bucket[c] = b.bx != nullptr ? min(max(b.bx[dx + b.rx], 0), b.nx - 1) : 0;
            }
            __syncthreads();
#pragma unroll
            for (int c = 0; c < kCols; ++c) {
                s[c] = 0.0;
                for (int w = 0; w < kTableWaves; ++w)
                    s[c] += parts[w][64 * c + lane];
            }
            for (int ix = wave; ix < b.nx; ix += kTableWaves) {
                double t = 0.0;
                bool any = false;
#pragma unroll
                for (int c = 0; c < kCols; ++c) {
                    any = any || bucket[c] == ix;
                    t += bucket[c] == ix ? s[c] : 0.0;
                }
                if (!__any(any))
                    continue;
                for (int m = 1; m < 64; m <<= 1)
                    t += __shfl_xor(t, m, 64);
                if (lane == 0)
                    tot[ix] += t;
            }
        }
    }
    __syncthreads();
    for (int x = threadIdx.x; x < b.nx; x += kTableThreads)
        dtable[(int64_t(head) * b.ny + iy) * b.nx + x] = float(tot[x]);
}

// ---------------------------------------------------------------------- host

struct Plan {
    int blocks, range, slices, q_cap, k_cap;
    int rows;  // blocks of queries whose sums by offset are held at a time
    int q_splits, k_splits, q_tiles, k_tiles;
    bool copies, direct;
    size_t q_lds, k_lds;
    // workspace: copies of q, dout, out and rest, of k and v; delta; sums by
    // work-group and by slice; partial gradients
    size_t q_copy, k_copy, delta_bytes, offset_bytes, sum_bytes, part_q, part_k;
};

size_t round_up(size_t bytes)
{
    return (bytes + 255) & ~size_t(255);
}

// Work-groups that share a walk of `tiles` where there are only `groups` walks
// for 256 compute units: two rounds of the chip, two tiles at least to each (one
// image of 40 x 40, 4 heads of 64 reals: 28 and 21 us and 9 of joining, 89 and 65
// with a work-group to a walk; 32, 24 and 7 with four tiles at least, and 2 of 20 x
// 20 then 30 and 23 where they take 21, 15 and 5).
constexpr int kLeastTiles = 2;
int share(int64_t groups, int tiles)
{
    return groups >= 256 ? 1 : int(std::max<int64_t>(1, std::min<int64_t>(512 / groups, tiles / kLeastTiles)));
}

// That, in whole tiles.
struct Walk {
    int splits, tiles;  // tiles of each
    Walk(int64_t groups, int walk)
    {
        tiles = (walk + share(groups, walk) - 1) / share(groups, walk);
        splits = (walk + tiles - 1) / tiles;
    }
};

// What sums by offset may take: they grow with the square of a map's pixels, so
// that beyond this the queries' launch and the sums over its blocks come in turns
// (backward pass of 64 and 96 heads of 160 x 160, 32 reals each, 2.6 and 3.9 GB of
// sums: 70.0 and 102.4 ms, 69.2 and 102.7 with all of them held).
constexpr size_t kOffsetBytes = size_t(2) << 30;

// Entries of a work-group's sums by offset.
int offset_range(const AttnGeom &g, const Offsets &o, int keys)
{
    return place_span(std::min(kQueries, g.lq()), g.wq, g.hq, o.skip_q) +
           place_span(std::min(keys, g.lk()), g.wk, g.hk, o.skip_k);
}

Plan backward_plan(const AttnCall &a, DType dt, const AttnGradients &gr)
{
    const AttnGeom &g = a.g;
    const int es = dt == DType::BF16 ? 2 : 4, tile = dt == DType::BF16 ? 64 : 32, dp = 4 * padded_dq(g.dq);
    const int lq = g.lq(), lk = g.lk();
    const bool table = gr.dtable != nullptr && a.bias.table != nullptr;
    Plan p{};
    p.copies = padded_dq(g.dq) != g.dq || !(a.q.vec && a.k.vec && a.v.vec && gr.out.vec && gr.dout.vec);
    if (p.copies) {
        p.q_copy = round_up(size_t(g.n) * g.heads * lq * dp * es);
        p.k_copy = round_up(size_t(g.n) * g.kv_heads * lk * dp * es);
    }
    p.blocks = (lq + kQueries - 1) / kQueries;
    const int key_blocks = (lk + kQueries - 1) / kQueries;
    const int q_walk = (lk + tile - 1) / tile, k_walk = (lq + tile - 1) / tile * (g.heads / g.kv_heads);
    const int64_t q_groups = int64_t(g.n) * g.heads * p.blocks, k_groups = int64_t(g.n) * g.kv_heads * key_blocks;
    const Walk qw(q_groups, q_walk), kw(k_groups, k_walk);
    p.q_splits = qw.splits;
    p.q_tiles = qw.tiles;
    p.k_splits = kw.splits;
    p.k_tiles = kw.tiles;
    // (room for what smaller batches share: at most 512 work-groups)
    const bool q_shared = q_walk >= 2 * kLeastTiles, k_shared = k_walk >= 2 * kLeastTiles;
    if (q_shared)
        p.part_q = round_up(size_t(512) * kQueries * dp * sizeof(float));
    if (k_shared)
        p.part_k = round_up(size_t(512) * kQueries * dp * sizeof(float));
    p.q_lds = size_t(4) * tile * (dp + (es == 2 ? 0 : 4)) * es + size_t(2) * tile * 4;
    p.k_lds = p.q_lds + size_t(6) * tile * 4;
    const int q_entry = table ? 12 : 4;  // bytes: a bias, and a sum
    p.slices = 1;
    p.rows = int(q_groups);
    p.delta_bytes = round_up(size_t(g.n) * g.heads * lq * sizeof(float));
    if (a.bias.table != nullptr) {
        const Offsets o = make_offsets(g);
        // a segment holds the widest tile's offsets
        const int block_q = place_span(std::min(kQueries, lq), g.wq, g.hq, o.skip_q);
        const int block_k = place_span(std::min(kQueries, lk), g.wk, g.hk, o.skip_k);
        p.q_cap = segment_cap(block_q + place_span(tile, g.wk, g.hk, o.skip_k) + 8, p.q_lds, q_entry);
        p.k_cap = segment_cap(block_k + place_span(tile, g.wq, g.hq, o.skip_q) + 8, p.k_lds, 4);
        if (table) {
            p.range = offset_range(g, o, p.q_tiles * tile);
            // (shared walks are few, and their sums no more than the maps)
            if (p.q_splits == 1)
                p.rows = int(std::min<int64_t>(q_groups, std::max<int64_t>(1, kOffsetBytes / (size_t(p.range) * sizeof(float)))));
            p.offset_bytes = round_up(size_t(p.rows) * p.q_splits * p.range * sizeof(float));
            // few sums are taken to their buckets directly: `entries` that an offset
            // has, 16 at most, and 8192 of them in all (backward pass of 16 images
            // of 8 x 8, 16 heads: 22.7 us, 24.8 in two launches; 8 of 14 x 9, 2 heads:
            // 28.1, 30.5; one of 30 x 30 and 2 of 32 x 32, 32 heads: no difference;
            // 4 of 20 x 20, 64 heads: 119.5, 112.8; one of 1 x 2000, 64 heads: 1089,
            // 473); images whose queries have places of their own have slices of
            // their own
            const int64_t entries = int64_t(g.n) * p.blocks * p.q_splits;
            p.direct = entries <= 16 && entries * o.total <= 8192 && p.rows == q_groups;
            const int most = a.pos != nullptr
                                 ? g.n
                                 : std::min(g.n, std::max(1, int(2048 / std::max<int64_t>(1, (o.total + 63) / 64 * int64_t(g.heads)))));
            p.slices = p.direct && a.pos == nullptr ? 1 : most;
            // (a smaller batch's may go through slices where this one's do not)
            p.sum_bytes = round_up(size_t(most) * g.heads * o.total * sizeof(double));
        }
    }
    p.q_lds += size_t(p.q_cap) * q_entry;
    p.k_lds += size_t(p.k_cap) * 4;
    return p;
}

template <typename T, int DQP, int QMODE, int KMODE> hipError_t launch(Backward f, const Plan &p, double *sums, hipStream_t s)
{
    const AttnGeom &g = f.a.g;
    f.o.cap = p.q_cap;
    const int rows = g.n * g.heads * p.blocks;
    for (f.first_row = 0; f.first_row < rows; f.first_row += p.rows) {
        f.rows = std::min(p.rows, rows - f.first_row);
        attention_dq_kernel<T, DQP, QMODE><<<xcd_grid(int64_t(f.rows) * p.q_splits), kThreads, p.q_lds, s>>>(f);
        if (hipError_t e = hipGetLastError())
            return e;
        if (f.offsets == nullptr || p.direct)
            continue;
        offset_sums_kernel<<<dim3((f.o.total + 63) / 64, g.heads, std::min(p.slices, 65535)), 64 * kSumWaves, 0, s>>>(
            f, p.slices, f.first_row > 0, sums);
        if (hipError_t e = hipGetLastError())
            return e;
    }
    f.o.cap = p.k_cap;
    const int64_t blocks = (g.lk() + kQueries - 1) / kQueries;
    attention_dkv_kernel<T, DQP, KMODE>
        <<<xcd_grid(g.n * g.kv_heads * blocks * p.k_splits), kThreads, p.k_lds, s>>>(f);
    if (hipError_t e = hipGetLastError())
        return e;
    const int64_t quads = DQP * int64_t(g.n) * ((p.q_splits > 1 ? int64_t(g.heads) * g.lq() : 0) +
                                                (p.k_splits > 1 ? 2 * int64_t(g.kv_heads) * g.lk() : 0));
    if (quads > 0)
        gradient_join_kernel<T, DQP><<<unsigned((quads + 255) / 256), 256, 0, s>>>(f);
    return hipGetLastError();
}
template <typename T, int DQP> hipError_t launch_mode(const Backward &f, const Plan &p, double *sums, hipStream_t s)
{
    const AttnGeom &g = f.a.g;
    if (f.a.bias.table == nullptr)
        return launch<T, DQP, 0, 0>(f, p, sums, s);
    const bool k4 = g.hk == 1 || g.wk % 4 == 0, q4 = g.hq == 1 || g.wq % 4 == 0;
    // (four pixels of a row have biases and sums side by side: 341 and 328 us for
    // 16 x 40 x 40, 426 and 343 pixel by pixel)
    if (k4 && q4)
        return launch<T, DQP, 1, 1>(f, p, sums, s);
    return launch<T, DQP, 2, 2>(f, p, sums, s);
}
template <typename T> hipError_t launch_dq(const Backward &f, const Plan &p, double *sums, hipStream_t s)
{
    switch (padded_dq(f.a.g.dq)) {
    case 8:
        return launch_mode<T, 8>(f, p, sums, s);
    case 16:
        return launch_mode<T, 16>(f, p, sums, s);
    default:
        return launch_mode<T, 32>(f, p, sums, s);
    }
}

}  // namespace

bool attention_backward_fits(const AttnCall &a, DType dt, const AttnGradients &gr)
{
    const Plan p = backward_plan(a, dt, gr);
    return std::max(p.q_lds, p.k_lds) <= kLdsLimit;
}

size_t attention_backward_work_bytes(const AttnCall &a, DType dt, const AttnGradients &gr)
{
    const Plan p = backward_plan(a, dt, gr);
    size_t offset_bytes = p.offset_bytes;
    if (offset_bytes > 0 && p.part_q > 0) {
        // (smaller batches are shared by more work-groups, whose entries overlap)
        const Offsets o = make_offsets(a.g);
        const int tile = dt == DType::BF16 ? 64 : 32, walk = (a.g.lk() + tile - 1) / tile;
        const int64_t image = int64_t(a.g.heads) * p.blocks;
        for (int64_t groups = image; groups < std::min<int64_t>(256, image * a.g.n); groups += image) {
            const Walk w(groups, walk);
            offset_bytes = std::max(offset_bytes, round_up(size_t(groups) * w.splits * offset_range(a.g, o, w.tiles * tile) *
                                                           sizeof(float)));
        }
    }
    return 4 * p.q_copy + 2 * p.k_copy + p.delta_bytes + offset_bytes + p.sum_bytes + p.part_q + 2 * p.part_k;
}

hipError_t attention_backward_run(const AttnCall &a, DType dt, const AttnGradients &gr, void *work, hipStream_t s)
{
    const Plan p = backward_plan(a, dt, gr);
    const AttnGeom &g = a.g;
    unsigned char *at = static_cast<unsigned char *>(work);
    auto take = [&](size_t bytes) {
        void *r = at;
        at += bytes;
        return r;
    };
    Backward f;
    f.a = a;
    f.o = make_offsets(g);
    f.out = gr.out;
    f.dout = gr.dout;
    f.dq = gr.dq;
    f.dk = gr.dk;
    f.dv = gr.dv;
    const int64_t c_all = int64_t(g.heads) * g.dq;
    f.rest = {gr.rest, g.lq() * 4 * c_all, 4 * c_all, c_all, true, g.dq};
    f.stats = gr.stats;
    if (p.copies) {
        AttnPack pack;
        pack.maps = 0;
        const int64_t d = 4 * padded_dq(g.dq);
        for (AttnMap *m : {&f.a.q, &f.dout, &f.out, &f.rest, &f.a.k, &f.a.v}) {
            if (m->data == nullptr)
                continue;
            const bool keys = m == &f.a.k || m == &f.a.v;
            const int i = pack.maps++;
            pack.src[i] = *m;
            // (rest is dense and aligned, but its rows may not be whole chunks)
            pack.src[i].vec = m->vec && g.dq % 8 == 0;
            pack.kv_len[i] = keys ? a.kv_len : nullptr;
            pack.heads[i] = keys ? g.kv_heads : g.heads;
            pack.by_heads[i] = FastDiv(pack.heads[i]);
            pack.tokens[i] = keys ? g.lk() : g.lq();
            pack.dst[i] = take(keys ? p.k_copy : p.q_copy);
            *m = {pack.dst[i], int64_t(pack.heads[i]) * pack.tokens[i] * d, d, d / 4, true, pack.tokens[i] * d};
        }
        if (hipError_t e = attention_pack_run(pack, g.n, g.dq, dt, s))
            return e;
    }
    const bool table = gr.dtable != nullptr && a.bias.table != nullptr;
    f.delta = static_cast<float *>(take(p.delta_bytes));
    f.offsets = table ? static_cast<float *>(take(p.offset_bytes)) : nullptr;
    double *sums = static_cast<double *>(take(p.sum_bytes));
    f.part_q = static_cast<float *>(take(p.part_q));
    f.part_k = static_cast<float *>(take(p.part_k));
    f.part_v = static_cast<float *>(take(p.part_k));
    f.blocks = p.blocks;
    f.range = p.range;
    f.q_splits = p.q_splits;
    f.k_splits = p.k_splits;
    f.q_tiles = p.q_tiles;
    f.k_tiles = p.k_tiles;
    f.q_span = p.q_tiles * (dt == DType::BF16 ? 64 : 32);
    if (hipError_t e = dt == DType::BF16 ? launch_dq<__bf16>(f, p, sums, s) : launch_dq<float>(f, p, sums, s))
        return e;
    if (!table)
        return hipSuccess;
    const int rows = g.hk + g.hq - 1, groups = g.heads * a.bias.ny;
    f.first_row = 0;
    f.rows = p.rows;
    if (p.direct)
        table_gradient_kernel<true><<<groups, kTableThreads, 0, s>>>(f, rows, p.slices, nullptr, gr.dtable);
    else
        table_gradient_kernel<false><<<groups, kTableThreads, 0, s>>>(f, rows, p.slices, sums, gr.dtable);
    return hipGetLastError();
}

}  // namespace quan
