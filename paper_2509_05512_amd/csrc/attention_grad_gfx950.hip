// The gradients of attention between the pixels of quaternion maps on gfx950.
//
// With P the probabilities, recomputed from the rows' saved maxima and sums,
//   dP = dO V^T,  delta_i = dO_i . O_i,  dS = P (dP - delta),
//   dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO,
//   dtable[head][b] = sum of dS over the pairs of pixels in bucket b.
// Two launches, so that every sum has one owner and a fixed order: the first
// takes blocks of queries and walks over the keys (dQ, delta, and the sums of
// dS by offset), the second blocks of keys and walks over the queries (dK, dV).
// Two more small ones bring the sums by offset to buckets, in fp64.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "attention_tile.h"

namespace quan {
namespace {

struct Backward {
    AttnCall a;
    Offsets o;
    AttnMap out, dout, dq, dk, dv;
    const void *rest;
    const float *stats;
    float *delta;    // [n][heads][lq]
    float *offsets;  // [n * heads * blocks][range] sums of dS by offset, NULL: none asked for
    int blocks, range;
};

constexpr int kWaves = 4, kThreads = 64 * kWaves, kQueries = 32 * kWaves;

// Sums of dS by offset in 64-bit fixed point: integer additions in LDS take 7
// clocks a wave where those of floats take 194 (measured), and their order
// changes nothing, so that the waves share one array.  Its units 2^-k follow
// from a bound of the terms known before they are: |dS| <= |dP - delta| <=
// |dO| |v| + |delta|, with the work-group's largest |dO| and |delta| and the
// tile's largest element of v.  k = 50 - e for a bound below 2^e: a term is
// below 2^51, an offset's terms (one per query, 128) stay below 2^58, and a
// term's last place is 2^-50 of the bound.  A tile with a larger bound takes the
// array to coarser units.  What NaN or infinity is in the work-group's rows or
// in v gives NaN.
constexpr int kSumBits = 50, kNoUnits = 127, kBadUnits = 128;
constexpr double kRound = 6755399441055744.0;  // 1.5 * 2^52: to add it rounds to an integer in the low bits
__device__ __forceinline__ void add_fixed(long long *entry, float v, double scale)
{
    const double t = fma(double(v), scale, kRound);
    const long long term = __builtin_bit_cast(long long, t) - __builtin_bit_cast(long long, kRound);
    __hip_atomic_fetch_add(reinterpret_cast<unsigned long long *>(entry), (unsigned long long)term, __ATOMIC_RELAXED,
                           __HIP_MEMORY_SCOPE_WORKGROUP);
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

// The launch of the queries' side.  Sums of dS by offset are gathered over the
// segment whose biases are staged; as the walk leaves it they go, over the
// waves, to the work-group's own row of `offsets`.
template <typename T, int DQP, int MODE>
__global__ void __launch_bounds__(kThreads, DQP <= 16 ? 3 : 1) attention_dq_kernel(Backward f)
{
    constexpr int DP = 4 * DQP;
    typedef Stage<T, DP, kThreads> Tile;
    typedef typename Elem<T>::frag frag;
    constexpr int KT = Tile::kTokens, SUBS = KT / 32;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds_raw[];
    T *k_lds = reinterpret_cast<T *>(lds_raw), *v_lds = k_lds + 2 * Tile::kElems;
    int *place = reinterpret_cast<int *>(v_lds + 2 * Tile::kElems);
    float *bias = reinterpret_cast<float *>(place + 2 * KT);
    long long *sums = reinterpret_cast<long long *>(bias + f.o.cap);
    __shared__ float tops[2 * kWaves];  // of a tile's v, by buffer and wave

    const AttnGeom &g = f.a.g;
    const int lq = g.lq(), lk = g.lk();
    const int total = g.n * g.heads * f.blocks;
    const int id = xcd_order(total);
    if (id >= total)
        return;
    const int block = id % f.blocks, head = id / f.blocks % g.heads, img = id / f.blocks / g.heads;
    const int kv_head = head / (g.heads / g.kv_heads);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
    const int q0 = block * kQueries, query = q0 + 32 * wave + (lane & 31);
    const bool q_here = query < lq;
    const int end = f.a.kv_len != nullptr ? min(max(f.a.kv_len[img], 0), lk) : lk;
    const int64_t row = (int64_t(img) * g.heads + head) * lq + query;

    const HeadMap<const T, DQP> qm(f.a.q, img, head, g.dq), km(f.a.k, img, kv_head, g.dq), vm(f.a.v, img, kv_head, g.dq);
    frag q[DP / 16], go[DP / 16];
    float delta = 0.0f;
    {
        const HeadMap<const T, DQP> gm(f.dout, img, head, g.dq), om(f.out, img, head, g.dq);
        const int64_t c_all = int64_t(g.heads) * g.dq;
        const AttnMap dense{f.rest, lq * 4 * c_all, 4 * c_all, c_all, f.out.vec && g.dq % 8 == 0};
        const HeadMap<const T, DQP> rm(dense, img, head, g.dq);
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) {
            const int d = 16 * i + 8 * half;
            q[i] = qm.load(query, d, q_here);
            go[i] = gm.load(query, d, q_here);
            f32x8 o = to_f32(om.load(query, d, q_here));
            if (f.rest != nullptr)
                o += to_f32(rm.load(query, d, q_here));
            const f32x8 w = to_f32(go[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                delta = fmaf(w[e], o[e], delta);
        }
        delta = half_sum(delta);
        if (q_here && half == 0)
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
            pos_y = f.a.pos[2 * img];
            pos_x = f.a.pos[2 * img + 1];
        }
        table = f.a.bias.table + int64_t(head) * f.a.bias.ny * f.a.bias.nx;
        low_q = f.o.origin - place_q(f.o, min(q0 + kQueries, lq) - 1);
        high_q = f.o.origin - place_q(f.o, q0);
        lane_at = f.o.origin - place_q(f.o, min(query, lq - 1));
        if (f.offsets != nullptr)
            offsets = f.offsets + ((int64_t(img) * g.heads + head) * f.blocks + block) * f.range - low_q;
        done = low_q;
    }
    const int past = MODE != 0 ? high_q + place_k(f.o, lk - 1) + 1 : 0;  // past the last offset
    // the bound's parts from the work-group's rows: |dO| and |delta|; a row whose
    // sum is no number has NaN
    float top_go = 0.0f, top_delta = 0.0f;
    if (MODE != 0 && offsets != nullptr) {
        float n2 = 0.0f;
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) {
            const f32x8 w = to_f32(go[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                n2 = fmaf(w[e], w[e], n2);
        }
        top_go = wave_top(sum <= -kLowest ? sqrtf(half_sum(n2)) : NAN);
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
        top_go *= sqrtf(float(DP));
        __syncthreads();
    }
    int units = kNoUnits;  // k of the array's units 2^-k
    double unit = 0.0;     // 2^k
    // The segment's sums, added to the entries that an earlier one has written; a thread has the same entries modulo kThreads of every
    // segment.
    auto flush = [&]() {
        const int last = min(segment + f.o.cap, past);
        int a = segment - segment % kThreads + int(threadIdx.x);
        if (a < segment)
            a += kThreads;
        for (; a < last; a += kThreads) {
            const int e = a - segment;
            const float v = units == kBadUnits ? NAN : units == kNoUnits ? 0.0f : float(ldexp(double(sums[e]), -units));
            offsets[a] = a < done ? offsets[a] + v : v;
        }
        done = max(done, last);
    };

    f32x16 dq[DP / 32];
#pragma unroll
    for (int i = 0; i < DP / 32; ++i)
        dq[i] = 0.0f;
    Tile kt, vt;
    if (0 < end) {
        kt.fetch(km, 0, end);
        vt.fetch(vm, 0, end);
    }
    int buf = 0;
    for (int j0 = 0; j0 < end; j0 += KT, buf ^= 1) {
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
            if (segment < 0 || hi >= segment + f.o.cap) {
                if (segment >= 0) {
                    __syncthreads();  // the last segment has been read and added to
                    if (offsets != nullptr)
                        flush();
                    __syncthreads();
                }
                segment = lo;
                stage_bias(bias, f.o, f.a.bias, table, segment, f.o.cap, pos_y, pos_x);
                if (offsets != nullptr)
                    for (int e = threadIdx.x; e < f.o.cap; e += kThreads)
                        sums[e] = 0;
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
                            sums[i] >>= min(units - now, 63);
                        __syncthreads();
                    }
                    units = now;
                    unit = ldexp(1.0, now);
                }
            }
        }
        const int at = lane_at - segment;
#pragma unroll
        for (int sub = 0; sub < SUBS; ++sub) {
            f32x16 s[1], dp = 0.0f;
            s[0] = 0.0f;
#pragma unroll
            for (int i = 0; i < DP / 16; ++i) {
                s[0] = mma(row_frag<T, DP>(kb, sub, i), q[i], s[0]);
                dp = mma(row_frag<T, DP>(vb, sub, i), go[i], dp);
            }
            add_bias<MODE, 1>(s[0], c, bias, pl, at, sub, half);
#pragma unroll
            for (int r = 0; r < 16; ++r)
                s[0][r] = exp2_fast(s[0][r] - top) * fmaf(dp[r], inv, shift);
            if (j0 + KT > end)
                clear_behind(s, j0 + 32 * sub, end, half, 0.0f);
            if (MODE != 0 && offsets != nullptr) {
#pragma unroll
                for (int gq = 0; gq < 4; ++gq) {
                    const i32x4 p4 = places<MODE>(pl, sub, gq, half);
#pragma unroll
                    for (int t = 0; t < 4; ++t)
                        add_fixed(sums + at + p4[t], s[0][4 * gq + t], unit);
                }
            }
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                const frag p = acc_frag<T>(s[0], st);
#pragma unroll
                for (int i = 0; i < DP / 32; ++i)
                    dq[i] = mma(col_frag<DP>(kb, sub, st, i), p, dq[i]);
            }
        }
    }
    const HeadMap<T, DQP> om(f.dq, img, head, g.dq);
#pragma unroll
    for (int i = 0; i < DP / 32; ++i) {
        dq[i] *= g.scale;
        om.store(query, i, half, dq[i], q_here);
    }
    if (MODE != 0 && offsets != nullptr) {
        if (segment >= 0) {
            __syncthreads();
            flush();
        }
        // entries of offsets to keys that the image lacks
        int a = done - done % kThreads + int(threadIdx.x);
        if (a < done)
            a += kThreads;
        for (; a < past; a += kThreads)
            offsets[a] = 0.0f;
    }
}

// The launch of the keys' side: lanes hold keys, registers queries.
constexpr int kNoSegment = -(1 << 30);
template <typename T, int DQP, int MODE>
__global__ void __launch_bounds__(kThreads, DQP <= 16 ? 2 : 1) attention_dkv_kernel(Backward f)
{
    constexpr int DP = 4 * DQP;
    typedef Stage<T, DP, kThreads> Tile;
    typedef typename Elem<T>::frag frag;
    constexpr int QT = Tile::kTokens, SUBS = QT / 32;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds_raw[];
    T *q_lds = reinterpret_cast<T *>(lds_raw), *g_lds = q_lds + 2 * Tile::kElems;
    float *rows = reinterpret_cast<float *>(g_lds + 2 * Tile::kElems);  // [2][top, inv, shift][QT]
    int *place = reinterpret_cast<int *>(rows + 6 * QT);
    float *bias = reinterpret_cast<float *>(place + 2 * QT);

    const AttnGeom &g = f.a.g;
    const int lq = g.lq(), lk = g.lk(), group = g.heads / g.kv_heads;
    const int blocks = (lk + kQueries - 1) / kQueries;
    const int total = g.n * g.kv_heads * blocks;
    const int id = xcd_order(total);
    if (id >= total)
        return;
    const int block = id % blocks, kv_head = id / blocks % g.kv_heads, img = id / blocks / g.kv_heads;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
    const int k0 = block * kQueries, key = k0 + 32 * wave + (lane & 31);
    const int end = f.a.kv_len != nullptr ? min(max(f.a.kv_len[img], 0), lk) : lk;
    const bool k_here = key < end;

    const HeadMap<const T, DQP> km(f.a.k, img, kv_head, g.dq), vm(f.a.v, img, kv_head, g.dq);
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
            pos_y = f.a.pos[2 * img];
            pos_x = f.a.pos[2 * img + 1];
        }
        low_k = f.o.origin + place_k(f.o, k0);
        high_k = f.o.origin + place_k(f.o, min(k0 + kQueries, lk) - 1);
        lane_at = f.o.origin + place_k(f.o, min(key, lk - 1));
    }
    const int tiles = k0 < end ? (lq + QT - 1) / QT : 0;
    for (int head = kv_head * group; head < (kv_head + 1) * group && tiles > 0; ++head) {
        const HeadMap<const T, DQP> qm(f.a.q, img, head, g.dq), gm(f.dout, img, head, g.dq);
        const float *table = MODE != 0 ? f.a.bias.table + int64_t(head) * f.a.bias.ny * f.a.bias.nx : nullptr;
        const int64_t row0 = (int64_t(img) * g.heads + head) * lq;
        int segment = kNoSegment, buf = 0;
        Tile qt, gt;
        __syncthreads();  // the last head's tiles and segment have been read
        qt.fetch(qm, (tiles - 1) * QT, lq);
        gt.fetch(gm, (tiles - 1) * QT, lq);
        // from the last tile, so that offsets ascend
        for (int tile = tiles - 1; tile >= 0; --tile, buf ^= 1) {
            const int i0 = tile * QT;
            T *qb = q_lds + buf * Tile::kElems, *gb = g_lds + buf * Tile::kElems;
            int *pl = place + buf * QT;
            float *rw = rows + buf * 3 * QT;
            qt.put(qb);
            gt.put(gb);
            if (threadIdx.x < QT) {
                const int i = i0 + threadIdx.x;
                const float sum = i < lq ? f.stats[2 * (row0 + i) + 1] : 0.0f;
                const bool empty = sum == 0.0f;
                const float inv = empty ? 0.0f : 1.0f / sum;
                rw[threadIdx.x] = empty ? INFINITY : f.stats[2 * (row0 + i)];
                rw[QT + threadIdx.x] = inv;
                rw[2 * QT + threadIdx.x] = empty ? 0.0f : -f.delta[row0 + i];
                if (MODE != 0)
                    pl[threadIdx.x] = place_q(f.o, min(i, lq - 1));
            }
            if (MODE != 0) {
                const int lo = low_k - place_q(f.o, min(i0 + QT, lq) - 1) - 3, hi = high_k - place_q(f.o, i0);
                if (segment == kNoSegment || hi >= segment + f.o.cap) {
                    if (segment != kNoSegment)
                        __syncthreads();
                    segment = lo;  // (down to -3)
                    stage_bias(bias, f.o, f.a.bias, table, segment, f.o.cap, pos_y, pos_x);
                }
            }
            __syncthreads();
            if (tile > 0) {
                qt.fetch(qm, i0 - QT, lq);
                gt.fetch(gm, i0 - QT, lq);
            }
            f32x16 s[SUBS], dp[SUBS];
#pragma unroll
            for (int sub = 0; sub < SUBS; ++sub) {
                s[sub] = 0.0f;
                dp[sub] = 0.0f;
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
                add_bias<MODE, -1>(s[sub], c, bias, pl, lane_at - segment, sub, half);
#pragma unroll
                for (int gq = 0; gq < 4; ++gq) {
                    const int first = 32 * sub + 8 * gq + 4 * half;
                    const f32x4 top = *reinterpret_cast<const f32x4 *>(rw + first);
                    const f32x4 inv = *reinterpret_cast<const f32x4 *>(rw + QT + first);
                    const f32x4 shift = *reinterpret_cast<const f32x4 *>(rw + 2 * QT + first);
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        const int r = 4 * gq + t;
                        const float p = exp2_fast(s[sub][r] - top[t]) * inv[t];
                        s[sub][r] = p;
                        dp[sub][r] = p * (dp[sub][r] + shift[t]);
                    }
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
    }
    // keys behind the image's last have no gradient
    const HeadMap<T, DQP> okm(f.dk, img, kv_head, g.dq), ovm(f.dv, img, kv_head, g.dq);
#pragma unroll
    for (int i = 0; i < DP / 32; ++i) {
        dk[i] *= g.scale;
        if (!k_here) {
            dk[i] = 0.0f;
            dv[i] = 0.0f;
        }
        okm.store(key, i, half, dk[i], key < lk);
        ovm.store(key, i, half, dv[i], key < lk);
    }
}

// Sums by offset over the work-groups of a head, in fp64 and a fixed order:
// slice s takes every slices-th image.  out [slices][heads][total].
__global__ void __launch_bounds__(256) offset_sums_kernel(Backward f, int slices, double *__restrict__ out)
{
    const AttnGeom &g = f.a.g;
    const int a = blockIdx.x * 256 + threadIdx.x, head = blockIdx.y;
    if (a >= f.o.total)
        return;
    const int lq = g.lq(), last_k = place_k(f.o, g.lk() - 1);
    for (int slice = blockIdx.z; slice < slices; slice += gridDim.z) {
        double s = 0.0;
        for (int b = 0; b < f.blocks; ++b) {
            const int low = f.o.origin - place_q(f.o, min((b + 1) * kQueries, lq) - 1);
            const int past = f.o.origin - place_q(f.o, b * kQueries) + last_k + 1;
            if (a < low || a >= past)
                continue;
            const float *p = f.offsets + (int64_t(head) * f.blocks + b) * f.range + (a - low);
            for (int img = slice; img < g.n; img += slices)
                s += double(p[int64_t(img) * g.heads * f.blocks * f.range]);
        }
        out[(int64_t(slice) * g.heads + head) * f.o.total + a] = s;
    }
}

// dtable from the sums by offset: a work-group per row of buckets (head, by).
// Its threads add up the rows dy of offsets in that bucket, column by column,
// then its waves the columns dx of each bucket bx.  The slices have their
// offsets' buckets in common, but where queries have places of their own (pos):
// there a slice is an image, and they are taken one by one.
constexpr int kTableThreads = 512, kTableCols = 2048;
__global__ void __launch_bounds__(kTableThreads)
table_gradient_kernel(AttnBias b, Offsets o, int heads, int rows, int slices, const int *__restrict__ pos,
                      const double *__restrict__ sums, float *__restrict__ dtable)
{
    __shared__ double cols[kTableCols];
    __shared__ short bucket[kTableCols];
    __shared__ double tot[kAttnMaxBuckets];
    const int iy = blockIdx.x % b.ny, head = blockIdx.x / b.ny;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int x = threadIdx.x; x < b.nx; x += kTableThreads)
        tot[x] = 0.0;
    const int groups = pos != nullptr ? slices : 1, per = slices / groups;
    for (int group = 0; group < groups; ++group) {
        const int pos_y = pos != nullptr ? pos[2 * group] : 0, pos_x = pos != nullptr ? pos[2 * group + 1] : 0;
        for (int x0 = 0; x0 < o.pitch; x0 += kTableCols) {
            const int width = min(kTableCols, o.pitch - x0);
            __syncthreads();  // cols has been read
            for (int x = threadIdx.x; x < width; x += kTableThreads) {
                double s = 0.0;
                for (int y = 0; y < rows; ++y) {
                    const int dy = min(max(y - o.hq1 - pos_y, -b.ry), b.ry);
                    if ((b.by != nullptr ? min(max(b.by[dy + b.ry], 0), b.ny - 1) : 0) != iy)
                        continue;
                    for (int sl = group * per; sl < (group + 1) * per; ++sl)
                        s += sums[(int64_t(sl) * heads + head) * o.total + int64_t(y) * o.pitch + x0 + x];
                }
                cols[x] = s;
                const int dx = min(max(x0 + x - o.wq1 - pos_x, -b.rx), b.rx);
                bucket[x] = short(b.bx != nullptr ? min(max(b.bx[dx + b.rx], 0), b.nx - 1) : 0);
            }
            __syncthreads();
            for (int ix = wave; ix < b.nx; ix += kTableThreads / 64) {
                double s = 0.0;
                for (int x = lane; x < width; x += 64)
                    if (bucket[x] == ix)
                        s += cols[x];
                for (int m = 1; m < 64; m <<= 1)
                    s += __shfl_xor(s, m, 64);
                if (lane == 0)
                    tot[ix] += s;
            }
        }
    }
    __syncthreads();
    for (int x = threadIdx.x; x < b.nx; x += kTableThreads)
        dtable[(int64_t(head) * b.ny + iy) * b.nx + x] = float(tot[x]);
}

// ---------------------------------------------------------------------- host

int padded_dq(int dq)
{
    return dq <= 8 ? 8 : dq <= 16 ? 16 : 32;
}

struct Plan {
    int blocks, range, slices, q_cap, k_cap;
    size_t q_lds, k_lds;
    size_t delta_bytes, offset_bytes, sum_bytes;
};

Plan backward_plan(const AttnCall &a, DType dt, bool table)
{
    const AttnGeom &g = a.g;
    const int es = dt == DType::BF16 ? 2 : 4, tile = dt == DType::BF16 ? 64 : 32, dp = 4 * padded_dq(g.dq);
    const int lq = g.lq(), lk = g.lk();
    Plan p{};
    p.blocks = (lq + kQueries - 1) / kQueries;
    p.slices = 1;
    p.delta_bytes = (size_t(g.n) * g.heads * lq * sizeof(float) + 255) & ~size_t(255);
    if (a.bias.table != nullptr) {
        const Offsets o = make_offsets(g);
        auto span = [](int count, int w, int h, int skip) { return count + std::min((count - 1) / w + 1, h - 1) * skip; };
        // a segment holds the widest tile's offsets
        auto cap = [&](int window) {
            int c = 1024;
            while (c < window)
                c *= 2;
            return c;
        };
        const int block_q = span(std::min(kQueries, lq), g.wq, g.hq, o.skip_q);
        const int block_k = span(std::min(kQueries, lk), g.wk, g.hk, o.skip_k);
        p.q_cap = cap(block_q + span(tile, g.wk, g.hk, o.skip_k) + 8);
        p.k_cap = cap(block_k + span(tile, g.wq, g.hq, o.skip_q) + 8);
        if (table) {
            p.range = block_q + host_place(lk - 1, g.wk, o.skip_k) + 1;
            p.offset_bytes = (size_t(g.n) * g.heads * p.blocks * p.range * sizeof(float) + 255) & ~size_t(255);
            // (images whose queries have places of their own have slices of their own)
            p.slices = a.pos != nullptr ? g.n : std::min(g.n, std::max(1, 1024 / std::max(1, (o.total + 255) / 256 * g.heads)));
            p.sum_bytes = size_t(p.slices) * g.heads * o.total * sizeof(double);
        }
    }
    const size_t tiles = size_t(4) * tile * (dp + (es == 2 ? 0 : 4)) * es + size_t(2) * tile * 4;
    p.q_lds = tiles + size_t(p.q_cap) * 4 * (table && a.bias.table != nullptr ? 3 : 1);
    p.k_lds = tiles + size_t(6) * tile * 4 + size_t(p.k_cap) * 4;
    return p;
}

template <typename T, int DQP, int QMODE, int KMODE> hipError_t launch(Backward f, const Plan &p, hipStream_t s)
{
    const AttnGeom &g = f.a.g;
    f.o.cap = p.q_cap;
    attention_dq_kernel<T, DQP, QMODE><<<xcd_grid(int64_t(g.n) * g.heads * p.blocks), kThreads, p.q_lds, s>>>(f);
    if (hipError_t e = hipGetLastError())
        return e;
    f.o.cap = p.k_cap;
    const int64_t blocks = (g.lk() + kQueries - 1) / kQueries;
    attention_dkv_kernel<T, DQP, KMODE><<<xcd_grid(g.n * g.kv_heads * blocks), kThreads, p.k_lds, s>>>(f);
    return hipGetLastError();
}
template <typename T, int DQP> hipError_t launch_mode(const Backward &f, const Plan &p, hipStream_t s)
{
    const AttnGeom &g = f.a.g;
    if (f.a.bias.table == nullptr)
        return launch<T, DQP, 0, 0>(f, p, s);
    const bool k4 = g.hk == 1 || g.wk % 4 == 0, q4 = g.hq == 1 || g.wq % 4 == 0;
    if (k4 && q4)
        return launch<T, DQP, 1, 1>(f, p, s);
    return launch<T, DQP, 2, 2>(f, p, s);
}
template <typename T> hipError_t launch_dq(const Backward &f, const Plan &p, hipStream_t s)
{
    switch (padded_dq(f.a.g.dq)) {
    case 8:
        return launch_mode<T, 8>(f, p, s);
    case 16:
        return launch_mode<T, 16>(f, p, s);
    default:
        return launch_mode<T, 32>(f, p, s);
    }
}

}  // namespace

size_t attention_backward_work_bytes(const AttnCall &a, DType dt, bool table)
{
    const Plan p = backward_plan(a, dt, table);
    return p.delta_bytes + p.offset_bytes + p.sum_bytes;
}

hipError_t attention_backward_run(const AttnCall &a, DType dt, const AttnMap &out, const void *rest,
                                  const float *stats, const AttnMap &dout, const AttnMap &dq, const AttnMap &dk,
                                  const AttnMap &dv, float *dtable, void *work, hipStream_t s)
{
    const bool table = dtable != nullptr && a.bias.table != nullptr;
    const Plan p = backward_plan(a, dt, table);
    unsigned char *w = static_cast<unsigned char *>(work);
    Backward f;
    f.a = a;
    f.o = make_offsets(a.g);
    f.out = out;
    f.dout = dout;
    f.dq = dq;
    f.dk = dk;
    f.dv = dv;
    f.rest = rest;
    f.stats = stats;
    f.delta = reinterpret_cast<float *>(w);
    f.offsets = table ? reinterpret_cast<float *>(w + p.delta_bytes) : nullptr;
    f.blocks = p.blocks;
    f.range = p.range;
    if (hipError_t e = dt == DType::BF16 ? launch_dq<__bf16>(f, p, s) : launch_dq<float>(f, p, s))
        return e;
    if (!table)
        return hipSuccess;
    double *sums = reinterpret_cast<double *>(w + p.delta_bytes + p.offset_bytes);
    offset_sums_kernel<<<dim3((f.o.total + 255) / 256, a.g.heads, std::min(p.slices, 65535)), 256, 0, s>>>(f, p.slices, sums);
    if (hipError_t e = hipGetLastError())
        return e;
    table_gradient_kernel<<<a.g.heads * a.bias.ny, kTableThreads, 0, s>>>(a.bias, f.o, a.g.heads, a.g.hk + a.g.hq - 1,
                                                                        p.slices, a.pos, sums, dtable);
    return hipGetLastError();
}

}  // namespace quan
