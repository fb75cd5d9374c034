// The row operators of a residual block on gfx950: norms over a pixel's 4C
// reals, gate, residual scale and dropout in one pass over the maps, forward
// and backward, and dropout by itself.
//
// A row is held by `lpr` neighbouring lanes (a power of two, at most a wave) as
// chunks of 8 reals, chunk k of a lane being lane + k * lpr, so that a wave
// reads 64 consecutive chunks; rows of more than 128 chunks take a whole
// work-group.  Sums over a row are butterflies over its lanes: every operand
// is read once, and nothing is written but the results.  All arithmetic is
// fp32, rounded once at the store.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "gfx950_dma.h"
#include "quan_block.h"

namespace quan {
namespace {

constexpr int kThreads = 256;         // of a work-group whose rows are held by waves or parts of them
constexpr int kBlockThreads = 512;     // at most, of one that holds a row together
constexpr int kWaves = kThreads / 64;
constexpr int kBlockWaves = kBlockThreads / 64;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// 8 reals of a row as they lie in memory.
template <typename T> struct Raw;
template <> struct Raw<__bf16> {
    bf16x8 v;
    __device__ __forceinline__ f32x8 get() const { return __builtin_convertvector(v, f32x8); }
};
template <> struct Raw<float> {
    f32x8 v;
    __device__ __forceinline__ f32x8 get() const { return v; }
};
// Those from element `at` of a map, of which the first `valid` (0, 4 or 8: rows
// are whole quaternions per channel, 4C reals) exist; zeros behind.  `whole` rows
// are multiples of 8 reals, so that every chunk is 16-byte aligned; others are
// aligned to 4 reals.
template <typename T> __device__ __forceinline__ Raw<T> load_raw(const T *map, int64_t at, int valid, bool whole)
{
    typedef T half __attribute__((ext_vector_type(4)));
    Raw<T> r;
    if (whole) {
        const Raw<T> t = *reinterpret_cast<const Raw<T> *>(map + (valid > 0 ? at : 0));
        r.v = valid > 0 ? t.v : T(0.0f);
        return r;
    }
    const half lo = *reinterpret_cast<const half *>(map + (valid > 0 ? at : 0));
    const half hi = *reinterpret_cast<const half *>(map + (valid > 4 ? at + 4 : 0));
    r.v.lo = valid > 0 ? lo : half(T(0.0f));
    r.v.hi = valid > 4 ? hi : half(T(0.0f));
    return r;
}
template <typename T> __device__ __forceinline__ f32x8 load8(const T *map, int64_t at, int valid, bool whole)
{
    return load_raw(map, at, valid, whole).get();
}
template <typename T> __device__ __forceinline__ void store8(T *p, const f32x8 &v, int valid, bool whole)
{
    typedef T half __attribute__((ext_vector_type(4)));
    typedef T full __attribute__((ext_vector_type(8)));
    const full b = __builtin_convertvector(v, full);
    if (whole) {
        if (valid > 0)
            __builtin_nontemporal_store(b, reinterpret_cast<full *>(p));
        return;
    }
    if (valid > 0)
        __builtin_nontemporal_store(b.lo, reinterpret_cast<half *>(p));
    if (valid > 4)
        __builtin_nontemporal_store(b.hi, reinterpret_cast<half *>(p + 4));
}

// Parameters are aligned to their element only.
__device__ __forceinline__ f32x8 param8(const float *p, int col, int valid)
{
    f32x8 v = 1.0f;
    if (p != nullptr)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < valid)
                v[e] = p[col + e];
    return v;
}

// Dropout of a chunk: see Drop.
__device__ __forceinline__ void drop8(f32x8 &v, unsigned chunk, unsigned pixel, uint64_t seed, uint64_t offset,
                                      const Drop &d)
{
    unsigned c0 = chunk, c1 = pixel, c2 = unsigned(offset), c3 = unsigned(offset >> 32);
    unsigned k0 = unsigned(seed), k1 = unsigned(seed >> 32);
#pragma unroll
    for (int r = 0; r < 7; ++r) {
        const uint64_t a = uint64_t(0xD2511F53u) * c0, b = uint64_t(0xCD9E8D57u) * c2;
        c0 = unsigned(b >> 32) ^ c1 ^ k0;
        c1 = unsigned(b);
        c2 = unsigned(a >> 32) ^ c3 ^ k1;
        c3 = unsigned(a);
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    const unsigned w[4] = {c0, c1, c2, c3};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const unsigned bits = e & 1 ? w[e >> 1] >> 16 : w[e >> 1] & 0xffffu;
        v[e] = bits >= d.cut ? v[e] * d.factor : 0.0f;
    }
}
__device__ __forceinline__ float dot8(const f32x8 &a, const f32x8 &b)
{
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        s = fmaf(a[e], b[e], s);
    return s;
}

// Sums over the lanes of a row; BLOCK: over the work-group.
template <int CTRL> __device__ __forceinline__ float dpp_add(float x)
{
    return x + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), CTRL, 0xf, 0xf, false));
}
template <bool BLOCK, int N>
__device__ __forceinline__ void row_sums(float (&s)[N], int lpr, float *lds)
{
    // (lane ^ 1, ^ 2, then the mirrors of 8 and of 16 lanes, whose halves hold
    // equal sums by then, and the other half of 32 and of 64)
    if (lpr >= 2)
#pragma unroll
        for (int i = 0; i < N; ++i)
            s[i] = dpp_add<0xB1>(s[i]);
    if (lpr >= 4)
#pragma unroll
        for (int i = 0; i < N; ++i)
            s[i] = dpp_add<0x4E>(s[i]);
    if (lpr >= 8)
#pragma unroll
        for (int i = 0; i < N; ++i)
            s[i] = dpp_add<0x141>(s[i]);
    if (lpr >= 16)
#pragma unroll
        for (int i = 0; i < N; ++i)
            s[i] = dpp_add<0x140>(s[i]);
    if (lpr >= 32)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const auto w = __builtin_amdgcn_permlane16_swap(__float_as_uint(s[i]), __float_as_uint(s[i]), false, false);
            s[i] = __uint_as_float(w[0]) + __uint_as_float(w[1]);
        }
    if (lpr >= 64)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(s[i]), __float_as_uint(s[i]), false, false);
            s[i] = __uint_as_float(w[0]) + __uint_as_float(w[1]);
        }
    if (BLOCK) {
        __syncthreads();  // the last sums have been read
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i)
                lds[i * kBlockWaves + (threadIdx.x >> 6)] = s[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            s[i] = 0.0f;
            for (int w = 0; w < int(blockDim.x >> 6); ++w)
                s[i] += lds[i * kBlockWaves + w];
        }
    }
}

// 1 / sqrt(x) of a normal number x > 0; NaN stays NaN.
__device__ __forceinline__ float inv_sqrt(float x)
{
    return __builtin_amdgcn_rsqf(x);
}

// The three sums of a gradient's row, those of absent parts left out.
template <bool BLOCK, bool HAS_Y, bool HAS_H>
__device__ __forceinline__ void row_sums3(float (&s)[3], int lpr, float *lds)
{
    if (HAS_Y) {
        float t[1] = {s[0]};
        row_sums<BLOCK>(t, lpr, lds);
        s[0] = t[0];
    }
    if (HAS_H) {
        float t[2] = {s[1], s[2]};
        row_sums<BLOCK>(t, lpr, lds);
        s[1] = t[0];
        s[2] = t[1];
    }
}

// A lane's place: its chunk of the row, the work-group's row.
struct Lane {
    int chunk, row;
    __device__ __forceinline__ Lane(int lpr, bool block)
        : chunk(block ? threadIdx.x : threadIdx.x & (lpr - 1)), row(block ? 0 : threadIdx.x / lpr)
    {
    }
    __device__ __forceinline__ int valid(int reals) const { return max(0, min(8, reals - 8 * chunk)); }
};

// ------------------------------------------------------------------- forward

// Bound by HBM: two maps read and two written, 8 bytes per real in bf16 (64 x 56
// x 56, 64 channels: 411 MB in 93 us, 4.4 TB/s where a large copy has 5.3; 108 us
// where every pass has maps of its own, none of them left in the last cache).  The
// work-groups walk over the rows side by side, so that at any time few DRAM
// pages are in use, and what they write goes past the caches (116 us before).
template <typename T, bool BLOCK, bool HAS_Y, bool HAS_H>
__global__ void __launch_bounds__(BLOCK ? kBlockThreads : kThreads)
residual_forward_kernel(int64_t rows, FastDiv by_hw, int reals, int lpr, bool whole, ResidualForward a, Drop drop,
                        float eps)
{
    __shared__ float lds[kBlockWaves];
    const Lane l(lpr, BLOCK);
    const int per = BLOCK ? 1 : kThreads / lpr, col = 8 * l.chunk, valid = l.valid(reals);
    const float mean = 1.0f / float(reals);
    const bool normed = HAS_Y && a.gamma != nullptr;
    uint64_t seed = 0, offset = 0;
    if (HAS_Y && drop.cut) {
        seed = drop.rng[0];
        offset = drop.rng[1];
    }
    f32x8 f, next;
    if (HAS_Y)
        f = param8(a.gamma, col, valid) * param8(a.scale, col, valid);
    if (HAS_H)
        next = param8(a.next_gamma, col, valid);
    const T *x = static_cast<const T *>(a.x), *y = static_cast<const T *>(a.y), *gate = static_cast<const T *>(a.gate);
    T *out = static_cast<T *>(a.out), *h = static_cast<T *>(a.h);
    // the next row's maps are on their way while this one's are summed
    Raw<T> nx, ny;
    auto fetch = [&](int64_t row) {
        const int v = row < rows ? valid : 0;
        nx = load_raw(x, row * reals + col, v, whole);
        if (HAS_Y)
            ny = load_raw(y, row * reals + col, v, whole);
    };
    const int64_t step = int64_t(gridDim.x) * per;
    fetch(int64_t(blockIdx.x) * per + l.row);
    for (int64_t base = int64_t(blockIdx.x) * per; base < rows; base += step) {
        const int64_t row = base + l.row;
        const int v = row < rows ? valid : 0;
        const int64_t at = row * reals + col;
        f32x8 xv = nx.get(), yv;
        if (HAS_Y)
            yv = ny.get();
        fetch(row + step);
        if (HAS_Y) {
            float r = 1.0f;
            if (normed) {
                float s[1] = {dot8(yv, yv)};
                row_sums<BLOCK>(s, lpr, lds);
                r = inv_sqrt(fmaf(s[0], mean, eps));
            }
            f32x8 z = yv * r * f;
            if (drop.cut)
                drop8(z, unsigned(l.chunk), unsigned(row), seed, offset, drop);
            if (gate != nullptr) {
                const int64_t img = row < rows ? fast_div(int(row), by_hw) : 0;
                z *= load8(gate, img * reals + col, v, whole);
            }
            xv += z;
            store8(out + at, xv, v, whole);
        }
        if (HAS_H) {
            float s[1] = {dot8(xv, xv)};
            row_sums<BLOCK>(s, lpr, lds);
            store8(h + at, xv * inv_sqrt(fmaf(s[0], mean, eps)) * next, v, whole);
        }
    }
}

// ------------------------------------------------------------------ backward

// How a gradient's rows are dealt to work-groups: `bpi` work-groups share each
// image (of `n` with `hw` rows; all rows are one image where no gate asks for
// sums by image) and take its rows in turn, or a work-group takes `ipb` images.
// Each writes the sums of its rows, image by image, to part[(image * bpi + b) *
// 2 * reals].
struct Deal {
    int64_t n, hw;
    int bpi, ipb, grid;
};

// With G the whole gradient at out (dout and the norm's of dh), m dropout's
// factors and yhat = y / rms(y) (or y):
//   dx = G,  u = G m scale gate gamma,  dy = (u - yhat mean(u yhat)) / rms(y),
//   Q[image] = sum over rows of G m yhat,  N = sum over rows of dh out / rms(out);
// Q carries the gradients of gate, scale and gamma, N that of next_gamma; a lane
// adds up its rows in fp32, what lies beyond a work-group's sums is fp64.
// Bound by HBM: four maps read and two written, 12 bytes per real in bf16 (64 x
// 56 x 56, 64 channels: 617 MB in 134 us, 4.6 TB/s, and 10 us for the sums).
template <typename T, bool BLOCK, bool HAS_Y, bool HAS_H>
__global__ void __launch_bounds__(BLOCK ? kBlockThreads : kThreads)
residual_backward_kernel(Deal deal, int reals, int lpr, bool whole, ResidualBackward a, Drop drop, float eps,
                         float *__restrict__ part)
{
    __shared__ float lds[2 * kBlockWaves];
    __shared__ float cols[BLOCK ? 1 : kWaves * 512];
    const Lane l(lpr, BLOCK);
    const int per = BLOCK ? 1 : kThreads / lpr, col = 8 * l.chunk, valid = l.valid(reals);
    const float mean = 1.0f / float(reals);
    const bool normed = HAS_Y && a.gamma != nullptr;
    uint64_t seed = 0, offset = 0;
    if (HAS_Y && drop.cut) {
        seed = drop.rng[0];
        offset = drop.rng[1];
    }
    f32x8 f, next;
    if (HAS_Y)
        f = param8(a.gamma, col, valid) * param8(a.scale, col, valid);
    if (HAS_H)
        next = param8(a.next_gamma, col, valid);
    const T *y = static_cast<const T *>(a.y), *dout = static_cast<const T *>(a.dout);
    const T *out = static_cast<const T *>(a.out), *dh = static_cast<const T *>(a.dh);
    const T *gate = static_cast<const T *>(a.gate);
    T *dx = static_cast<T *>(a.dx), *dy = static_cast<T *>(a.dy);

    const int64_t img0 = int64_t(blockIdx.x) / deal.bpi * deal.ipb;
    const int64_t b = int64_t(blockIdx.x) % deal.bpi;
    for (int64_t img = img0; img < img0 + deal.ipb && img < deal.n; ++img) {
        f32x8 acc_q = 0.0f, acc_n = 0.0f, fg = 1.0f;
        if (HAS_Y) {
            fg = f;
            if (gate != nullptr)
                fg *= load8(gate, img * reals + col, valid, whole);
        }
        for (int64_t base = b * per; base < deal.hw; base += int64_t(deal.bpi) * per) {
            const int v = base + l.row < deal.hw ? valid : 0;
            const int64_t row = img * deal.hw + base + l.row, at = row * reals + col;
            f32x8 yv, g = 0.0f, ov, hv;
            if (HAS_H) {
                ov = load8(out, at, v, whole);
                hv = load8(dh, at, v, whole);
            }
            if (HAS_Y)
                yv = load8(y, at, v, whole);
            if (dout != nullptr)
                g = load8(dout, at, v, whole);
            float s[3] = {0.0f, 0.0f, 0.0f};
            if (HAS_Y)
                s[0] = dot8(yv, yv);
            if (HAS_H) {
                s[1] = dot8(ov, ov);
                s[2] = dot8(hv * next, ov);
            }
            row_sums3<BLOCK, HAS_Y, HAS_H>(s, lpr, lds);
            if (HAS_H) {
                const float r = inv_sqrt(fmaf(s[1], mean, eps));
                const f32x8 hat = ov * r;
                acc_n += hv * hat;
                g += hv * next * r - hat * (s[2] * mean * r * r);
            }
            store8(dx + at, g, v, whole);
            if (HAS_Y) {
                const float r = normed ? inv_sqrt(fmaf(s[0], mean, eps)) : 1.0f;
                if (drop.cut)
                    drop8(g, unsigned(l.chunk), unsigned(row), seed, offset, drop);
                acc_q += g * (yv * r);
                g *= fg;
                if (normed) {
                    float t[1] = {dot8(g, yv)};
                    row_sums<BLOCK>(t, lpr, lds);
                    g = g * r - yv * (t[0] * mean * r * r * r);
                }
                store8(dy + at, g, v, whole);
            }
        }
        // the work-group's sums of the image, in a fixed order
        float *dst = part + (img * deal.bpi + b) * 2 * reals;
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            if (which == 0 ? !HAS_Y : !HAS_H)
                continue;
            const f32x8 acc = which == 0 ? acc_q : acc_n;
            if (BLOCK) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (e < valid)
                        dst[which * reals + col + e] = acc[e];
                continue;
            }
            __syncthreads();  // cols has been read
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float v = acc[e];
                for (int m = lpr; m < 64; m <<= 1)
                    v += __shfl_xor(v, m, 64);
                if ((threadIdx.x & 63) < unsigned(lpr))
                    cols[(threadIdx.x >> 6) * 512 + col + e] = v;
            }
            __syncthreads();
            for (int c = threadIdx.x; c < reals; c += kThreads) {
                float v = 0.0f;
#pragma unroll
                for (int w = 0; w < kWaves; ++w)
                    v += cols[w * 512 + c];
                dst[which * reals + c] = v;
            }
        }
    }
}

// Sums of `parts` partial sums per image, in fp64: part [n][parts][2][reals]
// -> sums [n][2][reals].  One work-group per 8 columns of both kinds and image.
constexpr int kCols = 8, kSlots = kThreads / kCols;
__global__ void __launch_bounds__(kThreads)
image_sums_kernel(const float *__restrict__ part, double *__restrict__ sums, int parts, int reals)
{
    __shared__ double lds[kSlots][kCols];
    const int col = blockIdx.x * kCols + threadIdx.x % kCols, slot = threadIdx.x / kCols;
    double s = 0.0;
    if (col < 2 * reals)
        for (int p = slot; p < parts; p += kSlots)
            s += double(part[(int64_t(blockIdx.y) * parts + p) * 2 * reals + col]);
    lds[slot][threadIdx.x % kCols] = s;
    __syncthreads();
    if (slot == 0 && col < 2 * reals) {
        s = 0.0;
        for (int i = 0; i < kSlots; ++i)
            s += lds[i][threadIdx.x];
        sums[int64_t(blockIdx.y) * 2 * reals + col] = s;
    }
}

// The parameters' gradients from Q and N of `entries` images (or of as many
// parts of all images where there is no gate), in fp64:
//   dgate = scale gamma Q,  dscale = sum gate gamma Q,  dgamma = sum gate scale Q.
template <typename T, typename S>
__global__ void __launch_bounds__(kThreads)
param_gradient_kernel(const S *__restrict__ sums, int64_t entries, int reals, ResidualBackward a)
{
    __shared__ double lds[2][kSlots][kCols];
    const int i = threadIdx.x % kCols, col = blockIdx.x * kCols + i, slot = threadIdx.x / kCols;
    const T *gate = static_cast<const T *>(a.gate);
    T *dgate = static_cast<T *>(a.dgate);
    double q = 0.0, nx = 0.0;
    float gamma = 1.0f, scale = 1.0f;
    if (col < reals) {
        if (a.gamma != nullptr)
            gamma = a.gamma[col];
        if (a.scale != nullptr)
            scale = a.scale[col];
        for (int64_t e = slot; e < entries; e += kSlots) {
            if (a.y != nullptr) {
                const double v = double(sums[e * 2 * reals + col]);
                if (gate != nullptr) {
                    q += v * double(float(gate[e * reals + col]));
                    dgate[e * reals + col] = T(float(v * double(gamma) * double(scale)));
                } else {
                    q += v;
                }
            }
            if (a.next_gamma != nullptr)
                nx += double(sums[e * 2 * reals + reals + col]);
        }
    }
    lds[0][slot][i] = q;
    lds[1][slot][i] = nx;
    __syncthreads();
    if (slot == 0 && col < reals) {
        q = nx = 0.0;
        for (int s = 0; s < kSlots; ++s) {
            q += lds[0][s][i];
            nx += lds[1][s][i];
        }
        if (a.dgamma != nullptr)
            a.dgamma[col] = float(q * double(scale));
        if (a.dscale != nullptr)
            a.dscale[col] = float(q * double(gamma));
        if (a.dnext_gamma != nullptr)
            a.dnext_gamma[col] = float(nx);
    }
}

// ------------------------------------------------------------------- dropout

// Bound by HBM, the mask being cheap enough: 14 products of 32 x 32 bits per
// chunk of 8 reals (128 x 32 x 32, 16 channels: 34 MB in 6.9 us, 4.9 TB/s).  out
// may be x: a chunk is read and written by one lane, in that order.
template <typename T>
__global__ void __launch_bounds__(kThreads)
dropout_kernel(int64_t rows, int reals, int lpr, bool whole, const T *x, T *out, Drop drop)
{
    const int first = threadIdx.x & (lpr - 1);
    const int per = kThreads / lpr, chunks = (reals + 7) / 8;
    const uint64_t seed = drop.cut ? drop.rng[0] : 0, offset = drop.cut ? drop.rng[1] : 0;
    for (int64_t row = int64_t(blockIdx.x) * per + threadIdx.x / lpr; row < rows; row += int64_t(gridDim.x) * per)
        for (int c = first; c < chunks; c += lpr) {
            const int v = min(8, reals - 8 * c);
            const int64_t p = row * reals + 8 * c;
            f32x8 t = load8(x, p, v, whole);
            if (drop.cut)
                drop8(t, unsigned(c), unsigned(row), seed, offset, drop);
            store8(out + p, t, v, whole);
        }
}

// ---------------------------------------------------------------------- host

int lanes_per_row(int reals)
{
    const int chunks = (reals + 7) / 8;
    int l = 1;
    while (l < chunks && l < 64)
        l <<= 1;
    return l;
}

// Rows of up to 512 reals are a wave's or a part of one's, wider ones a
// work-group's of as many waves as they have chunks for.
bool block_rows(int reals)
{
    return reals > 512;
}
int group_threads(int reals)
{
    return !block_rows(reals) ? kThreads : reals <= 1024 ? 128 : reals <= 2048 ? 256 : kBlockThreads;
}
static_assert(4 * kRowsMaxChannels <= 8 * kBlockThreads, "a work-group holds the widest row");

// The work-groups that the chip holds at once, forward several times over, so
// that the last round is short.  (A gradient's have partial sums to write: one
// time over.)
constexpr int kForwardGroups = 256 * 8;
int backward_groups(int reals)
{
    return 256 * 1024 / group_threads(reals);
}

Deal deal_rows(const RowsGeom &g, bool by_image)
{
    Deal d;
    d.n = by_image ? g.n : 1;
    d.hw = by_image ? g.hw : g.n * g.hw;
    const int reals = 4 * g.c, groups = backward_groups(reals);
    const int per = block_rows(reals) ? 1 : kThreads / lanes_per_row(reals);
    const int64_t most = (d.hw + per - 1) / per;
    d.bpi = int(std::max<int64_t>(1, std::min<int64_t>(groups / d.n, most)));
    d.ipb = int((d.n + groups - 1) / groups);
    d.grid = int((d.n + d.ipb - 1) / d.ipb) * d.bpi;
    return d;
}

// The smallest eps that is added: the root takes smaller numbers as 0.  (Here, not
// at each root: a comparison there that lets NaN through, which fmaxf does not, took
// the gradients of 64 x 56 x 56, 64 channels, from 143 to 205 us.)
float normal_eps(float eps)
{
    return std::max(eps, 1.17549435e-38f);
}

template <typename T, bool HAS_Y, bool HAS_H>
hipError_t forward_launch(const RowsGeom &g, const ResidualForward &a, const Drop &drop, float eps, hipStream_t s)
{
    const int reals = 4 * g.c, lpr = lanes_per_row(reals);
    const int64_t rows = g.n * g.hw;
    const bool whole = reals % 8 == 0;
    const int per = block_rows(reals) ? 1 : kThreads / lpr;
    const dim3 grid(unsigned(std::min<int64_t>((rows + per - 1) / per, kForwardGroups)));
    const FastDiv by(int(g.hw));
    if (block_rows(reals))
        residual_forward_kernel<T, true, HAS_Y, HAS_H><<<grid, group_threads(reals), 0, s>>>(rows, by, reals, lpr, whole, a, drop, eps);
    else
        residual_forward_kernel<T, false, HAS_Y, HAS_H><<<grid, kThreads, 0, s>>>(rows, by, reals, lpr, whole, a, drop, eps);
    return hipGetLastError();
}

template <typename T, bool HAS_Y, bool HAS_H>
hipError_t backward_launch(const RowsGeom &g, const ResidualBackward &a, const Drop &drop, float eps, void *work,
                           hipStream_t s)
{
    const int reals = 4 * g.c, lpr = lanes_per_row(reals);
    const bool whole = reals % 8 == 0;
    const Deal d = deal_rows(g, a.gate != nullptr);
    float *part = static_cast<float *>(work);
    if (block_rows(reals))
        residual_backward_kernel<T, true, HAS_Y, HAS_H><<<d.grid, group_threads(reals), 0, s>>>(d, reals, lpr, whole, a, drop, eps, part);
    else
        residual_backward_kernel<T, false, HAS_Y, HAS_H><<<d.grid, kThreads, 0, s>>>(d, reals, lpr, whole, a, drop, eps, part);
    if (hipError_t e = hipGetLastError())
        return e;
    if (a.dgate == nullptr && a.dgamma == nullptr && a.dscale == nullptr && a.dnext_gamma == nullptr)
        return hipSuccess;
    const int64_t entries = a.gate != nullptr ? d.n : d.bpi;
    const dim3 grid(unsigned((reals + kCols - 1) / kCols));
    if (a.gate != nullptr && d.bpi > 1) {
        // (bpi > 1 only where n < backward_groups: n fits the grid)
        double *sums = reinterpret_cast<double *>(part + d.n * d.bpi * 2 * reals);
        image_sums_kernel<<<dim3(unsigned((2 * reals + kCols - 1) / kCols), unsigned(d.n)), kThreads, 0, s>>>(
            part, sums, d.bpi, reals);
        if (hipError_t e = hipGetLastError())
            return e;
        param_gradient_kernel<T, double><<<grid, kThreads, 0, s>>>(sums, entries, reals, a);
    } else {
        param_gradient_kernel<T, float><<<grid, kThreads, 0, s>>>(part, entries, reals, a);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t residual_forward_run(const RowsGeom &g, DType dt, const ResidualForward &a, const Drop &drop, float eps,
                                hipStream_t s)
{
    const bool has_y = a.y != nullptr, has_h = a.h != nullptr;
    eps = normal_eps(eps);
    if (dt == DType::BF16)
        return has_y ? has_h ? forward_launch<__bf16, true, true>(g, a, drop, eps, s)
                             : forward_launch<__bf16, true, false>(g, a, drop, eps, s)
                     : forward_launch<__bf16, false, true>(g, a, drop, eps, s);
    return has_y ? has_h ? forward_launch<float, true, true>(g, a, drop, eps, s)
                         : forward_launch<float, true, false>(g, a, drop, eps, s)
                 : forward_launch<float, false, true>(g, a, drop, eps, s);
}

size_t residual_backward_work_bytes(const RowsGeom &g, const ResidualBackward &a)
{
    // enough for every smaller batch and map: n images take at most
    // max(n, backward_groups) rows of partial sums, and of sums by image
    const size_t row = size_t(8) * g.c, n = a.gate != nullptr ? size_t(g.n) : 1;
    const size_t groups = size_t(backward_groups(4 * g.c));
    return (std::max(n, groups) * sizeof(float) + std::min(n, groups) * sizeof(double)) * row;
}

hipError_t residual_backward_run(const RowsGeom &g, DType dt, const ResidualBackward &a, const Drop &drop, float eps,
                                 void *work, hipStream_t s)
{
    const bool has_y = a.y != nullptr, has_h = a.dh != nullptr;
    eps = normal_eps(eps);
    if (dt == DType::BF16)
        return has_y ? has_h ? backward_launch<__bf16, true, true>(g, a, drop, eps, work, s)
                             : backward_launch<__bf16, true, false>(g, a, drop, eps, work, s)
                     : backward_launch<__bf16, false, true>(g, a, drop, eps, work, s);
    return has_y ? has_h ? backward_launch<float, true, true>(g, a, drop, eps, work, s)
                         : backward_launch<float, true, false>(g, a, drop, eps, work, s)
                 : backward_launch<float, false, true>(g, a, drop, eps, work, s);
}

hipError_t dropout_run(const RowsGeom &g, DType dt, const void *x, void *out, const Drop &drop, hipStream_t s)
{
    const int reals = 4 * g.c, lpr = lanes_per_row(reals), per = kThreads / lpr;
    const int64_t rows = g.n * g.hw;
    const dim3 grid(unsigned(std::min<int64_t>((rows + per - 1) / per, kForwardGroups)));
    const bool whole = reals % 8 == 0;
    if (dt == DType::BF16)
        dropout_kernel<<<grid, kThreads, 0, s>>>(rows, reals, lpr, whole, static_cast<const __bf16 *>(x),
                                                 static_cast<__bf16 *>(out), drop);
    else
        dropout_kernel<<<grid, kThreads, 0, s>>>(rows, reals, lpr, whole, static_cast<const float *>(x),
                                                 static_cast<float *>(out), drop);
    return hipGetLastError();
}

}  // namespace quan
