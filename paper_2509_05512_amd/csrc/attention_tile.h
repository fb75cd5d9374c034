// Device helpers shared by the attention kernels (gfx950): element types and
// their matrix products, chunks of a head's row, tiles in LDS and the position
// bias of a tile.
//
// A head's row is D = 4 DQP reals, component-major, DQP = 8, 16 or 32 the
// quaternion channels dq of a head rounded up (the added ones are zero).
//
// Products are 32 x 32 tiles over 16 reals of depth.  Lane l of a wave holds
// row (or column) l % 32 and 8 values of the depth; its accumulators are
// column l % 32 and the rows 8 (r / 4) + 4 (l / 32) + r % 4, r < 16.  Rows and
// depth may be any tokens that both operands agree on.  Row m of the products of
// part `sub` of a tile of kTile tokens stands for token
//   kTile / 2 * (m / 4 % 2) + 16 sub + 4 (m / 8) + m % 4,
// so that accumulator r of a lane is token 16 sub + r of its half-wave's half of
// the tile.  Then 8 accumulators, r = 8 s .. 8 s + 7, are at once the operand of
// 8 tokens of depth (the probabilities go from one product to the next without
// leaving their lanes), and the two half-waves' tokens are 32 apart in bf16: of
// the 32 neighbouring queries that they hold, none has the same offset to both.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>

#include "gfx950_dma.h"
#include "quan_block.h"

namespace quan {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLowest = -3.402823466e38f;

template <typename T> struct Elem;
template <> struct Elem<__bf16> {
    typedef bf16x8 frag;
    static constexpr int kTile = 64;  // tokens of a tile in LDS
};
template <> struct Elem<float> {
    typedef f32x8 frag;
    static constexpr int kTile = 32;
};

__device__ __forceinline__ f32x16 mma(const bf16x8 &a, const bf16x8 &b, const f32x16 &c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
// fp32: 8 products over two reals of depth, one of each half-wave.
__device__ __forceinline__ f32x16 mma(const f32x8 &a, const f32x8 &b, f32x16 c)
{
#pragma unroll
    for (int e = 0; e < 8; ++e)
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
    return c;
}

template <typename T> __device__ __forceinline__ typename Elem<T>::frag to_frag(const f32x8 &v);
template <> __device__ __forceinline__ bf16x8 to_frag<__bf16>(const f32x8 &v)
{
    return __builtin_convertvector(v, bf16x8);
}
template <> __device__ __forceinline__ f32x8 to_frag<float>(const f32x8 &v)
{
    return v;
}
__device__ __forceinline__ f32x8 to_f32(const bf16x8 &v)
{
    return __builtin_convertvector(v, f32x8);
}
__device__ __forceinline__ f32x8 to_f32(const f32x8 &v)
{
    return v;
}

// Accumulators 8 s .. 8 s + 7 as an operand.
template <typename T> __device__ __forceinline__ typename Elem<T>::frag acc_frag(const f32x16 &v, int s)
{
    f32x8 t;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        t[e] = v[8 * s + e];
    return to_frag<T>(t);
}

// Takes from accumulators 8 s .. 8 s + 7 what they were rounded to.
template <typename F> __device__ __forceinline__ void take_from(f32x16 &v, int s, const F &rounded)
{
    const f32x8 r = to_f32(rounded);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        v[8 * s + e] -= r[e];
}

// What the rounding of a result to bf16 leaves, in 16 bits: by how much the bits
// of the fp32 value are above those of the rounded one, at most half of its last
// place (a tie, the one distance that does not fit, is cut by 2^-24 of the value).
__device__ __forceinline__ short rest_of(float value, __bf16 rounded)
{
    const int above = int(__float_as_uint(value) - (unsigned(__builtin_bit_cast(unsigned short, rounded)) << 16));
    return short(max(min(above, 32767), -32768));
}
// The fp32 values again.
__device__ __forceinline__ f32x8 with_rest(const bf16x8 &rounded, const bf16x8 &rest)
{
    const auto high = __builtin_bit_cast(u16x8, rounded);
    const auto low = __builtin_bit_cast(s16x8, rest);
    f32x8 v;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        v[e] = __uint_as_float((unsigned(high[e]) << 16) + unsigned(int(low[e])));
    return v;
}
__device__ __forceinline__ f32x8 with_rest(const f32x8 &value, const f32x8 &)
{
    return value;
}

// Values of the two half-waves joined: the lane's own and lane ^ 32's.
__device__ __forceinline__ float half_max(float x)
{
    const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(w[0]), __uint_as_float(w[1]));
}
__device__ __forceinline__ float half_sum(float x)
{
    const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(w[0]) + __uint_as_float(w[1]);
}
__device__ __forceinline__ float exp2_fast(float x)
{
    return __builtin_amdgcn_exp2f(x);
}

// 8 reals of a row that has `valid` of them from p on, zeros behind; p can be
// read where valid is 0 too.  vec: p is 16-byte aligned and valid is 0 or 8.
template <typename T> __device__ __forceinline__ typename Elem<T>::frag load_chunk(const T *p, int valid, bool vec)
{
    typename Elem<T>::frag v = {};
    if (vec) {
        const typename Elem<T>::frag t = *reinterpret_cast<const typename Elem<T>::frag *>(p);
        v = valid > 0 ? t : v;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const T t = p[max(min(e, valid - 1), 0)];
            v[e] = e < valid ? t : v[e];
        }
    }
    return v;
}
template <typename T> __device__ __forceinline__ void store_chunk(T *p, const f32x8 &v, int valid, bool vec)
{
    const typename Elem<T>::frag f = to_frag<T>(v);
    if (vec) {
        if (valid > 0)
            *reinterpret_cast<typename Elem<T>::frag *>(p) = f;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < valid)
                p[e] = f[e];
    }
}
// 4 reals (a quad of accumulators): aligned to 4 elements where vec.
__device__ __forceinline__ void store_quad(__bf16 *p, const f32x4 &v, int valid, bool vec)
{
    const bf16x4 f = __builtin_convertvector(v, bf16x4);
    if (vec) {
        if (valid > 0)
            *reinterpret_cast<bf16x4 *>(p) = f;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < valid)
                p[e] = f[e];
    }
}
__device__ __forceinline__ void store_quad(float *p, const f32x4 &v, int valid, bool vec)
{
    if (vec) {
        if (valid > 0)
            *reinterpret_cast<f32x4 *>(p) = v;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < valid)
                p[e] = v[e];
    }
}

__device__ __forceinline__ void store_rest(__bf16 *to, const f32x4 &v, int valid, bool vec)
{
    s16x4 f;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        f[e] = rest_of(v[e], __bf16(v[e]));
    short *p = reinterpret_cast<short *>(to);
    if (vec) {
        if (valid > 0)
            *reinterpret_cast<s16x4 *>(p) = f;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < valid)
                p[e] = f[e];
    }
}

// A head of one image in a map: element d = component * DQP + channel of a
// token at at(token, d); channels dq and beyond do not exist.
template <typename T, int DQP> struct HeadMap {
    T *p;
    int64_t s_t, s_p;
    int dq;
    bool vec;
    __device__ __forceinline__ HeadMap(const AttnMap &m, int64_t img, int head, int dq_)
        : p(static_cast<T *>(const_cast<void *>(m.data)) + img * m.s_n + head * m.s_h), s_t(m.s_t), s_p(m.s_p),
          dq(dq_), vec(m.vec)
    {
    }
    __device__ __forceinline__ T *at(int64_t token, int d) const
    {
        return p + token * s_t + (d / DQP) * s_p + d % DQP;
    }
    __device__ __forceinline__ int valid(int d, int most) const { return max(0, min(most, dq - d % DQP)); }
    __device__ __forceinline__ typename Elem<T>::frag load(int64_t token, int d, bool here) const
    {
        const int n = here ? valid(d, 8) : 0;
        return load_chunk<T>(n > 0 ? at(token, d) : p, n, vec);
    }
    // Accumulators of a D x 32 tile, transposed: column = token.
    __device__ __forceinline__ void store(int64_t token, int tile, int half, const f32x16 &v, bool here) const
    {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int d = 32 * tile + 8 * g + 4 * half;
            const f32x4 q = {v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]};
            if (here)
                store_quad(at(token, d), q, valid(d, 4), vec);
        }
    }
};
// One whose rows are whole chunks, aligned (see AttnPack), to be read.
template <typename T, int DQP> struct WholeMap {
    typedef typename Elem<T>::frag frag;
    const T *p;
    int64_t s_t, s_p;
    __device__ __forceinline__ WholeMap(const AttnMap &m, int64_t img, int head)
        : p(static_cast<const T *>(m.data) + img * m.s_n + head * m.s_h), s_t(m.s_t), s_p(m.s_p)
    {
    }
    __device__ __forceinline__ const T *at(int64_t token, int d) const
    {
        return p + token * s_t + (d / DQP) * s_p + d % DQP;
    }
    __device__ __forceinline__ frag load(int64_t token, int d, bool here) const
    {
        const frag v = *reinterpret_cast<const frag *>(at(here ? token : 0, d));
        return here ? v : frag{};
    }
};

// ------------------------------------------------------------- tiles in LDS

// A tile is read by rows, 16 bytes of 16 rows (8 neighbouring ones of each half)
// at a time, and in bf16 by columns, 64 bytes of 4 neighbouring rows (tr reads).
// Its chunks of 16 bytes change places within a row by a number that the row
// gives, so that both fall into different banks: rows of 64 bytes (4 in a line
// of the 64 banks) by bits 2 and 5 of the row, of 128 bytes by bit 1 (to the
// other half of the row) and bits 2, 5, of 256 bytes by bits 0, 1 and 2, 5.  fp32
// tiles, read by columns real by real, have 16 bytes between their rows instead.
template <typename T, int DP> struct Lds;
template <int DP> struct Lds<__bf16, DP> {
    static constexpr int kRow = DP;
    static __device__ __forceinline__ int turn(int row)
    {
        const int q = (row >> 2 & 1) | (row >> 4 & 2);
        return DP == 32 ? q : DP == 64 ? (row << 1 & 4) | q : (row << 2 & 12) | q;
    }
    static __device__ __forceinline__ int at(int row, int chunk) { return row * DP + ((chunk ^ turn(row)) << 3); }
};
template <int DP> struct Lds<float, DP> {
    static constexpr int kRow = DP + 4;
    static __device__ __forceinline__ int at(int row, int chunk) { return row * kRow + (chunk << 3); }
};

// A tile of kTile tokens x D reals, staged by THREADS threads: fetch() loads
// this thread's chunks of the tile at `token`, put() writes them to LDS.
template <typename T, int DP, int THREADS> struct Stage {
    typedef typename Elem<T>::frag frag;
    static constexpr int kTokens = Elem<T>::kTile, kRow = Lds<T, DP>::kRow;
    static constexpr int kChunks = DP / 8, kStep = THREADS / kChunks;
    static constexpr int kCount = kTokens > kStep ? kTokens / kStep : 1;  // (more threads than chunks: some idle)
    static_assert(THREADS % kChunks == 0 && kCount * kStep >= kTokens, "whole rows per step");
    static constexpr int kElems = kTokens * kRow;
    frag r[kCount];
    template <int DQP> __device__ __forceinline__ void fetch(const WholeMap<T, DQP> &m, int token, int end)
    {
        const int row = threadIdx.x / kChunks, d = 8 * (threadIdx.x % kChunks);
        const T *p = m.at(token + row, d);  // (dereferenced below `end` only)
        if (kStep <= kTokens && token + kTokens <= end) {
#pragma unroll
            for (int i = 0; i < kCount; ++i)
                r[i] = *reinterpret_cast<const frag *>(p + int64_t(i * kStep) * m.s_t);
            return;
        }
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            const bool here = token + row + i * kStep < end && (kStep <= kTokens || row < kTokens);
            const frag v = *reinterpret_cast<const frag *>(here ? p + int64_t(i * kStep) * m.s_t : m.p);
            r[i] = here ? v : frag{};
        }
    }
    __device__ __forceinline__ void put(T *lds) const
    {
        const int row = threadIdx.x / kChunks, d = 8 * (threadIdx.x % kChunks);
        if (kStep > kTokens && row >= kTokens)
            return;
#pragma unroll
        for (int i = 0; i < kCount; ++i)
            *reinterpret_cast<frag *>(lds + Lds<T, DP>::at(row + i * kStep, d / 8)) = r[i];
    }
};
// Operand whose rows are the tokens of a tile's part `sub` and whose depth is
// reals 16 f + 8 (lane / 32) ..+7 of a row.
template <typename T, int DP> __device__ __forceinline__ typename Elem<T>::frag row_frag(const T *tile, int sub, int f)
{
    const int lane = threadIdx.x & 63, m = lane & 31;
    const int row = Elem<T>::kTile / 2 * (m >> 2 & 1) + 4 * (m >> 3) + (m & 3);
    // (16 rows on, a row's turn of chunks is the same)
    return *reinterpret_cast<const typename Elem<T>::frag *>(tile + Lds<T, DP>::at(row, 2 * f + (lane >> 5)) +
                                                             16 * sub * Lds<T, DP>::kRow);
}

// Operand whose rows are reals 32 mt + lane % 32 and whose depth is the tokens
// that acc_frag(., s) of part `sub` stands for: 16 sub + 8 s ..+7 of the lane's
// half of the tile.  In bf16 four tokens of one real come from one transposing
// read, in which 16 lanes give the addresses of 4 rows of 16 reals.
template <int DP> __device__ __forceinline__ bf16x8 col_frag(const __bf16 *tile, int sub, int s, int mt)
{
    typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;
    const int lane = threadIdx.x & 63, i = lane & 15;
    const int row = Elem<__bf16>::kTile / 2 * (lane >> 5) + (i >> 2), at = 4 * (i & 1);
    const int chunk = 4 * mt + (lane >> 3 & 2) + (i >> 1 & 1);
    const __bf16 *p = tile + (16 * sub + 8 * s) * DP + at;
    const bf16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4 *)(p + Lds<__bf16, DP>::at(row, chunk)));
    const bf16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4 *)(p + Lds<__bf16, DP>::at(row + 4, chunk)));
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}
template <int DP> __device__ __forceinline__ f32x8 col_frag(const float *tile, int sub, int s, int mt)
{
    constexpr int kRow = Lds<float, DP>::kRow;
    const int lane = threadIdx.x & 63;
    const float *p = tile + (Elem<float>::kTile / 2 * (lane >> 5) + 16 * sub + 8 * s) * kRow + 32 * mt + (lane & 31);
    f32x8 v;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        v[e] = p[e * kRow];
    return v;
}

// ------------------------------------------------------- the position bias

// Offsets in one number: A = place(key) - place(query) + origin with place(t)
// = (t / w) * pitch + t % w, pitch = wk + wq - 1 and origin = place of the last
// query, so that A / pitch and A % pitch are dy + hq - 1 and dx + wq - 1.  Of a
// tile of queries and keys A lies in a range not much longer than the tile's
// sides and the rows' ends between them; biases of a range (a segment) are
// looked up once into LDS, as table * log2 e.
struct Offsets {
    int pitch, origin, hq1, wq1;  // hq - 1, wq - 1
    int total;                    // A < total
    FastDiv by_pitch, by_wq, by_wk;
    int skip_q, skip_k;  // pitch - wq, pitch - wk
    int cap;             // entries of a segment
};
// Tokens side by side, from any one on: the range of their places.
inline int place_span(int count, int w, int h, int skip)
{
    return count + std::min((count - 1) / w + 1, h - 1) * skip;
}
// What a work-group may have of a compute unit's 160 KiB, static arrays aside.
constexpr size_t kLdsLimit = 160 * 1024 - 512;
// Entries of a segment that holds a tile's `window` of offsets at `bytes` each
// beside `fixed` bytes of LDS: a power of two, or where that does not fit the
// window alone (which may not fit either).
inline int segment_cap(int window, size_t fixed, int bytes)
{
    int c = 1024;
    while (c < window)
        c *= 2;
    return fixed + size_t(c) * bytes <= kLdsLimit ? c : (window + 3) / 4 * 4;
}
inline Offsets make_offsets(const AttnGeom &g)
{
    Offsets o;
    o.pitch = g.wk + g.wq - 1;
    o.hq1 = g.hq - 1;
    o.wq1 = g.wq - 1;
    o.origin = o.hq1 * o.pitch + o.wq1;
    o.total = (g.hk + g.hq - 1) * o.pitch;
    o.by_pitch = FastDiv(o.pitch);
    o.by_wq = FastDiv(g.wq);
    o.by_wk = FastDiv(g.wk);
    o.skip_q = o.pitch - g.wq;
    o.skip_k = o.pitch - g.wk;
    o.cap = 0;
    return o;
}
__device__ __forceinline__ int place_q(const Offsets &o, int t)
{
    return t + fast_div(t, o.by_wq) * o.skip_q;
}
__device__ __forceinline__ int place_k(const Offsets &o, int t)
{
    return t + fast_div(t, o.by_wk) * o.skip_k;
}

// A coordinate of a query's place.  Maps and radii are at most 2^24, so that
// offsets from 2^26 on are beyond any radius; closer to the ends of the type
// their differences would wrap.  (One for all lanes, and kept as that: in vector
// registers it cost the queries' gradient two more spilled ones, 341 us for 327.)
__device__ __forceinline__ int query_pos(int p)
{
    return __builtin_amdgcn_readfirstlane(min(max(p, -(1 << 26)), 1 << 26));
}
// Bucket (by * nx + bx) of offset A for an image whose queries start at (y, x).
__device__ __forceinline__ int bucket_of(const Offsets &o, const AttnBias &b, int a, int y, int x)
{
    const int qy = fast_div(a, o.by_pitch);
    int dy = qy - o.hq1 - y, dx = a - qy * o.pitch - o.wq1 - x;
    dy = min(max(dy, -b.ry), b.ry);
    dx = min(max(dx, -b.rx), b.rx);
    const int iy = b.by != nullptr ? min(max(b.by[dy + b.ry], 0), b.ny - 1) : 0;
    const int ix = b.bx != nullptr ? min(max(b.bx[dx + b.rx], 0), b.nx - 1) : 0;
    return iy * b.nx + ix;
}
// A bias in units of log 2; finite ones stay finite, so that rows whose every
// bias is the type's lowest value keep a softmax.
__device__ __forceinline__ float in_log2(float t)
{
    const float v = t * kLog2e;
    return fabsf(t) <= -kLowest ? fminf(fmaxf(v, kLowest), -kLowest) : v;
}
// Entries [first, first + count) of offsets into lds; those that no pair of
// pixels has (a quad's tokens may pass the last one) are zero.
__device__ __forceinline__ void stage_bias(float *lds, const Offsets &o, const AttnBias &b, const float *table,
                                           int first, int count, int y, int x)
{
    for (int e = threadIdx.x; e < count; e += blockDim.x) {
        const int a = first + e;
        lds[e] = a >= 0 && a < o.total ? in_log2(table[bucket_of(o, b, a, y, x)]) : 0.0f;
    }
}

// Places of the 4 tokens of a quad of accumulators.  MODE 1: they lie in one row
// of the map; 2: anywhere.
// (`first`: the lane's half of the tile's first token.)
template <int MODE> __device__ __forceinline__ i32x4 places(const int *place, int first, int sub, int quad)
{
    const int *p = place + first + 16 * sub + 4 * quad;
    if (MODE == 2)
        return *reinterpret_cast<const i32x4 *>(p);
    const int p0 = MODE == 1 ? p[0] : 0;
    return i32x4{p0, p0 + 1, p0 + 2, p0 + 3};
}
// Scores in units of log 2: c times the products plus the bias of the lane's
// offset `at` + SIGN * place (MODE 0: no bias).
template <int MODE, int SIGN>
__device__ __forceinline__ void add_bias(f32x16 &s, float c, const float *bias, const int *place, int at, int first,
                                         int sub)
{
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        if (MODE == 0) {
#pragma unroll
            for (int t = 0; t < 4; ++t)
                s[4 * g + t] *= c;
        } else if (MODE == 1) {
            const int p0 = place[first + 16 * sub + 4 * g];
            const float *b = bias + (SIGN > 0 ? at + p0 : at - p0 - 3);
#pragma unroll
            for (int t = 0; t < 4; ++t)
                s[4 * g + t] = fmaf(s[4 * g + t], c, b[SIGN > 0 ? t : 3 - t]);
        } else {
            const i32x4 p = places<MODE>(place, first, sub, g);
#pragma unroll
            for (int t = 0; t < 4; ++t)
                s[4 * g + t] = fmaf(s[4 * g + t], c, bias[at + SIGN * p[t]]);
        }
    }
}
// `value` in the accumulators of part `sub` whose tokens are at or behind `left`
// of the lane's half of the tile.  (The empty statement ties the comparisons to
// this branch: the compiler would else make selects of them for every tile.)
__device__ __forceinline__ void clear_behind(f32x16 &s, int left, int sub, float value)
{
    asm volatile("" : "+v"(left));
#pragma unroll
    for (int r = 0; r < 16; ++r)
        s[r] = 16 * sub + r >= left ? value : s[r];
}

// The work-group's place among `total` in an order in which neighbours run on
// the same XCD (work-groups go to the 8 XCDs in turn), so that those that read
// the same keys share an L2.
__device__ __forceinline__ int xcd_order(int total)
{
    const int per = (total + 7) / 8;
    return (blockIdx.x & 7) * per + (blockIdx.x >> 3);
}
inline unsigned xcd_grid(int64_t total)
{
    return unsigned((total + 7) / 8 * 8);
}

}  // namespace
}  // namespace quan
