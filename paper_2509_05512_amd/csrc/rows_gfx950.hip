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

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// 8 reals of a row from `p`, of which the first `valid` (0, 4 or 8: rows are
// whole quaternions per channel, 4C reals) exist.  `whole` rows are multiples
// of 8 reals, so that every chunk is 16-byte aligned; others are aligned to 4
// reals.
__device__ __forceinline__ f32x8 load8(const __bf16 *p, int valid, bool whole)
{
    f32x8 v = 0.0f;
    if (whole) {
        if (valid == 8)
            v = __builtin_convertvector(*reinterpret_cast<const bf16x8 *>(p), f32x8);
        return v;
    }
    if (valid >= 4) {
        const f32x4 a = __builtin_convertvector(*reinterpret_cast<const bf16x4 *>(p), f32x4);
        v.lo = a;
    }
    if (valid == 8) {
        const f32x4 a = __builtin_convertvector(*reinterpret_cast<const bf16x4 *>(p + 4), f32x4);
        v.hi = a;
    }
    return v;
}
__device__ __forceinline__ f32x8 load8(const float *p, int valid, bool)
{
    f32x8 v = 0.0f;
    if (valid >= 4)
        v.lo = *reinterpret_cast<const f32x4 *>(p);
    if (valid == 8)
        v.hi = *reinterpret_cast<const f32x4 *>(p + 4);
    return v;
}
__device__ __forceinline__ void store8(__bf16 *p, const f32x8 &v, int valid, bool whole)
{
    const bf16x8 b = __builtin_convertvector(v, bf16x8);
    if (whole) {
        if (valid == 8)
            *reinterpret_cast<bf16x8 *>(p) = b;
        return;
    }
    if (valid >= 4)
        *reinterpret_cast<bf16x4 *>(p) = b.lo;
    if (valid == 8)
        *reinterpret_cast<bf16x4 *>(p + 4) = b.hi;
}
__device__ __forceinline__ void store8(float *p, const f32x8 &v, int valid, bool)
{
    if (valid >= 4)
        *reinterpret_cast<f32x4 *>(p) = v.lo;
    if (valid == 8)
        *reinterpret_cast<f32x4 *>(p + 4) = v.hi;
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

// The 8 factors (0 or 1 / (1 - p)) of a chunk: see Drop.
struct Mask {
    unsigned w[4];
    unsigned cut;
    float factor;
    __device__ __forceinline__ float apply(float v, int e) const
    {
        const unsigned bits = e & 1 ? w[e >> 1] >> 16 : w[e >> 1] & 0xffffu;
        return bits >= cut ? v * factor : 0.0f;
    }
};
__device__ __forceinline__ Mask mask8(unsigned chunk, unsigned pixel, uint64_t seed, uint64_t offset, const Drop &d)
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
    return {{c0, c1, c2, c3}, d.cut, d.factor};
}

// Sums over the lanes of a row; BLOCK: over the work-group.
template <bool BLOCK, int N>
__device__ __forceinline__ void row_sums(float (&s)[N], int lpr, float *lds)
{
    for (int m = 1; m < lpr; m <<= 1)
#pragma unroll
        for (int i = 0; i < N; ++i)
            s[i] += __shfl_xor(s[i], m, 64);
    if (BLOCK) {
        __syncthreads();  // the last sums have been read
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i)
                lds[i * kWaves + (threadIdx.x >> 6)] = s[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            s[i] = 0.0f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w)
                s[i] += lds[i * kWaves + w];
        }
    }
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

// A lane's place in its row.
struct Lane {
    int at, row, lpr;  // among the row's lanes; the work-group's row; lanes that hold a row
    int step;          // lanes between chunks of a lane
    __device__ __forceinline__ Lane(int lpr_, bool block)
        : at(block ? threadIdx.x : threadIdx.x & (lpr_ - 1)), row(block ? 0 : threadIdx.x / lpr_), lpr(lpr_),
          step(block ? kThreads : lpr_)
    {
    }
    __device__ __forceinline__ int chunk(int k) const { return at + k * step; }
    __device__ __forceinline__ int valid(int k, int reals) const { return max(0, min(8, reals - 8 * chunk(k))); }
};

// ------------------------------------------------------------------- forward

// Bound by HBM: two maps read and two written, 8 bytes per real in bf16.
template <typename T, int CH, bool BLOCK, bool HAS_Y, bool HAS_H>
__global__ void __launch_bounds__(kThreads)
residual_forward_kernel(int64_t rows, FastDiv by_hw, int reals, int lpr, bool whole, ResidualForward a, Drop drop,
                        float eps)
{
    __shared__ float lds[kWaves];
    const Lane l(lpr, BLOCK);
    const int per = BLOCK ? 1 : kThreads / lpr;
    const float mean = 1.0f / float(reals);
    const bool normed = HAS_Y && a.gamma != nullptr;
    uint64_t seed = 0, offset = 0;
    if (HAS_Y && drop.cut) {
        seed = drop.rng[0];
        offset = drop.rng[1];
    }
    f32x8 f[CH], next[CH];
    int valid[CH];
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        valid[k] = l.valid(k, reals);
        const int col = 8 * l.chunk(k);
        if (HAS_Y)
            f[k] = param8(a.gamma, col, valid[k]) * param8(a.scale, col, valid[k]);
        if (HAS_H)
            next[k] = param8(a.next_gamma, col, valid[k]);
    }
    const T *x = static_cast<const T *>(a.x), *y = static_cast<const T *>(a.y), *gate = static_cast<const T *>(a.gate);
    T *out = static_cast<T *>(a.out), *h = static_cast<T *>(a.h);
    for (int64_t base = int64_t(blockIdx.x) * per; base < rows; base += int64_t(gridDim.x) * per) {
        const int64_t row = base + l.row;
        const bool here = row < rows;
        const int64_t at = (here ? row : 0) * reals;
        f32x8 xv[CH], yv[CH];
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int v = here ? valid[k] : 0;
            xv[k] = load8(x + at + 8 * l.chunk(k), v, whole);
            if (HAS_Y)
                yv[k] = load8(y + at + 8 * l.chunk(k), v, whole);
        }
        if (HAS_Y) {
            float r = 1.0f;
            if (normed) {
                float s[1] = {0.0f};
#pragma unroll
                for (int k = 0; k < CH; ++k)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        s[0] = fmaf(yv[k][e], yv[k][e], s[0]);
                row_sums<BLOCK>(s, lpr, lds);
                r = 1.0f / sqrtf(fmaf(s[0], mean, eps));
            }
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                const int v = here ? valid[k] : 0;
                f32x8 z = yv[k] * r * f[k];
                if (drop.cut) {
                    const Mask m = mask8(unsigned(l.chunk(k)), unsigned(row), seed, offset, drop);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        z[e] = m.apply(z[e], e);
                }
                if (gate != nullptr) {
                    const int64_t img = here ? fast_div(int(row), by_hw) : 0;
                    z *= load8(gate + img * reals + 8 * l.chunk(k), v, whole);
                }
                xv[k] += z;
                store8(out + at + 8 * l.chunk(k), xv[k], v, whole);
            }
        }
        if (HAS_H) {
            float s[1] = {0.0f};
#pragma unroll
            for (int k = 0; k < CH; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    s[0] = fmaf(xv[k][e], xv[k][e], s[0]);
            row_sums<BLOCK>(s, lpr, lds);
            const float r = 1.0f / sqrtf(fmaf(s[0], mean, eps));
#pragma unroll
            for (int k = 0; k < CH; ++k)
                store8(h + at + 8 * l.chunk(k), xv[k] * r * next[k], here ? valid[k] : 0, whole);
        }
    }
}

// ------------------------------------------------------------------ backward

// How a gradient's rows are dealt to work-groups: `bpi` work-groups share each
// image (of `n` with `hw` rows; all rows are one image where no gate asks for
// sums by image), or a work-group takes `ipb` images.  Each writes the sums of
// its rows, image by image, to part[(image * bpi + b) * 2 * reals].
struct Deal {
    int64_t n, hw;
    int bpi, ipb, grid;
    int64_t rows;  // of a work-group in an image
};

// With G the whole gradient at out (dout and the norm's of dh), m dropout's
// factors and yhat = y / rms(y) (or y):
//   dx = G,  u = G m scale gate gamma,  dy = (u - yhat mean(u yhat)) / rms(y),
//   Q[image] = sum over rows of G m yhat,  N = sum over rows of dh out / rms(out);
// Q carries the gradients of gate, scale and gamma, N that of next_gamma.
// Bound by HBM: four maps read and two written, 12 bytes per real in bf16.
template <typename T, int CH, bool BLOCK, bool HAS_Y, bool HAS_H>
__global__ void __launch_bounds__(kThreads)
residual_backward_kernel(Deal deal, int reals, int lpr, bool whole, ResidualBackward a, Drop drop, float eps,
                         float *__restrict__ part)
{
    __shared__ float lds[2 * kWaves];
    __shared__ float cols[BLOCK ? 1 : kWaves * CH * 512];
    const Lane l(lpr, BLOCK);
    const int per = BLOCK ? 1 : kThreads / lpr;
    const float mean = 1.0f / float(reals);
    const bool normed = HAS_Y && a.gamma != nullptr;
    uint64_t seed = 0, offset = 0;
    if (HAS_Y && drop.cut) {
        seed = drop.rng[0];
        offset = drop.rng[1];
    }
    f32x8 f[CH], next[CH];
    int valid[CH];
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        valid[k] = l.valid(k, reals);
        const int col = 8 * l.chunk(k);
        if (HAS_Y)
            f[k] = param8(a.gamma, col, valid[k]) * param8(a.scale, col, valid[k]);
        if (HAS_H)
            next[k] = param8(a.next_gamma, col, valid[k]);
    }
    const T *y = static_cast<const T *>(a.y), *dout = static_cast<const T *>(a.dout);
    const T *out = static_cast<const T *>(a.out), *dh = static_cast<const T *>(a.dh);
    const T *gate = static_cast<const T *>(a.gate);
    T *dx = static_cast<T *>(a.dx), *dy = static_cast<T *>(a.dy);

    const int64_t img0 = int64_t(blockIdx.x) / deal.bpi * deal.ipb;
    const int64_t b = int64_t(blockIdx.x) % deal.bpi;
    for (int64_t img = img0; img < img0 + deal.ipb && img < deal.n; ++img) {
        f32x8 acc_q[CH], acc_n[CH], fg[CH];
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            acc_q[k] = 0.0f;
            acc_n[k] = 0.0f;
            if (HAS_Y) {
                fg[k] = f[k];
                if (gate != nullptr)
                    fg[k] *= load8(gate + img * reals + 8 * l.chunk(k), valid[k], whole);
            }
        }
        const int64_t last = min((b + 1) * deal.rows, deal.hw);
        for (int64_t base = b * deal.rows; base < last; base += per) {
            const bool here = base + l.row < last;
            const int64_t row = img * deal.hw + (here ? base + l.row : 0);
            const int64_t at = row * reals;
            f32x8 yv[CH], g[CH], ov[CH], hv[CH];
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                const int v = here ? valid[k] : 0;
                const int64_t p = at + 8 * l.chunk(k);
                if (HAS_H) {
                    ov[k] = load8(out + p, v, whole);
                    hv[k] = load8(dh + p, v, whole);
                }
                if (HAS_Y)
                    yv[k] = load8(y + p, v, whole);
                if (dout != nullptr)
                    g[k] = load8(dout + p, v, whole);
                else
                    g[k] = 0.0f;
            }
            float s[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int k = 0; k < CH; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if (HAS_Y)
                        s[0] = fmaf(yv[k][e], yv[k][e], s[0]);
                    if (HAS_H) {
                        s[1] = fmaf(ov[k][e], ov[k][e], s[1]);
                        s[2] = fmaf(hv[k][e] * next[k][e], ov[k][e], s[2]);
                    }
                }
            row_sums3<BLOCK, HAS_Y, HAS_H>(s, lpr, lds);
            if (HAS_H) {
                const float r = 1.0f / sqrtf(fmaf(s[1], mean, eps));
                const float t = s[2] * mean * r * r;
#pragma unroll
                for (int k = 0; k < CH; ++k)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float hat = ov[k][e] * r;
                        acc_n[k][e] = fmaf(hv[k][e], hat, acc_n[k][e]);
                        g[k][e] += r * hv[k][e] * next[k][e] - hat * t;
                    }
            }
#pragma unroll
            for (int k = 0; k < CH; ++k)
                store8(dx + at + 8 * l.chunk(k), g[k], here ? valid[k] : 0, whole);
            if (HAS_Y) {
                const float r = normed ? 1.0f / sqrtf(fmaf(s[0], mean, eps)) : 1.0f;
                float t[1] = {0.0f};
#pragma unroll
                for (int k = 0; k < CH; ++k) {
                    if (drop.cut) {
                        const Mask m = mask8(unsigned(l.chunk(k)), unsigned(row), seed, offset, drop);
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            g[k][e] = m.apply(g[k][e], e);
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        acc_q[k][e] = fmaf(g[k][e], yv[k][e] * r, acc_q[k][e]);
                        g[k][e] *= fg[k][e];
                        t[0] = fmaf(g[k][e], yv[k][e], t[0]);
                    }
                }
                if (normed) {
                    row_sums<BLOCK>(t, lpr, lds);
                    const float c = t[0] * mean * r * r * r;
#pragma unroll
                    for (int k = 0; k < CH; ++k)
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            g[k][e] = r * g[k][e] - yv[k][e] * c;
                }
#pragma unroll
                for (int k = 0; k < CH; ++k)
                    store8(dy + at + 8 * l.chunk(k), g[k], here ? valid[k] : 0, whole);
            }
        }
        // the work-group's sums of the image, in a fixed order
        float *dst = part + (img * deal.bpi + b) * 2 * reals;
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            if (which == 0 ? !HAS_Y : !HAS_H)
                continue;
            if (BLOCK) {
#pragma unroll
                for (int k = 0; k < CH; ++k)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (e < valid[k])
                            dst[which * reals + 8 * l.chunk(k) + e] = which == 0 ? acc_q[k][e] : acc_n[k][e];
                continue;
            }
            __syncthreads();  // cols has been read
#pragma unroll
            for (int k = 0; k < CH; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float v = which == 0 ? acc_q[k][e] : acc_n[k][e];
                    for (int m = lpr; m < 64; m <<= 1)
                        v += __shfl_xor(v, m, 64);
                    if ((threadIdx.x & 63) < unsigned(lpr))
                        cols[(threadIdx.x >> 6) * CH * 512 + 8 * l.chunk(k) + e] = v;
                }
            __syncthreads();
            for (int c = threadIdx.x; c < reals; c += kThreads) {
                float v = 0.0f;
#pragma unroll
                for (int w = 0; w < kWaves; ++w)
                    v += cols[w * CH * 512 + c];
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

// Bound by HBM where the mask is cheap enough: one product of 32 x 32 bits per
// 4/7 of a real (14 per chunk of 8).
template <typename T>
__global__ void __launch_bounds__(kThreads)
dropout_kernel(int64_t rows, int reals, int lpr, bool whole, const T *__restrict__ x, T *__restrict__ out, Drop drop)
{
    const Lane l(lpr, false);
    const int per = kThreads / lpr, chunks = (reals + 7) / 8;
    const uint64_t seed = drop.cut ? drop.rng[0] : 0, offset = drop.cut ? drop.rng[1] : 0;
    for (int64_t row = int64_t(blockIdx.x) * per + l.row; row < rows; row += int64_t(gridDim.x) * per)
        for (int c = l.at; c < chunks; c += lpr) {
            const int v = min(8, reals - 8 * c);
            const int64_t p = row * reals + 8 * c;
            f32x8 t = load8(x + p, v, whole);
            if (drop.cut) {
                const Mask m = mask8(unsigned(c), unsigned(row), seed, offset, drop);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    t[e] = m.apply(t[e], e);
            }
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

// Rows of up to 1024 reals are a wave's, wider ones a work-group's.
bool block_rows(int reals)
{
    return reals > 1024;
}

// The work-groups that the chip holds at once, several times over, so that
// the last round is short.
constexpr int kForwardGroups = 256 * 8;
constexpr int kBackwardGroups = 256 * 4;

Deal deal_rows(const RowsGeom &g, bool by_image)
{
    Deal d;
    d.n = by_image ? g.n : 1;
    d.hw = by_image ? g.hw : g.n * g.hw;
    const int reals = 4 * g.c;
    const int per = block_rows(reals) ? 1 : kThreads / lanes_per_row(reals);
    const int64_t most = (d.hw + per - 1) / per;
    d.bpi = int(std::max<int64_t>(1, std::min<int64_t>(kBackwardGroups / std::max<int64_t>(1, d.n), most)));
    d.ipb = int((d.n + kBackwardGroups - 1) / kBackwardGroups);
    d.rows = ((most + d.bpi - 1) / d.bpi) * per;
    d.bpi = int((d.hw + d.rows - 1) / d.rows);
    d.grid = int((d.n + d.ipb - 1) / d.ipb) * d.bpi;
    return d;
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
    if (reals <= 512)
        residual_forward_kernel<T, 1, false, HAS_Y, HAS_H><<<grid, kThreads, 0, s>>>(rows, by, reals, lpr, whole, a, drop, eps);
    else if (reals <= 1024)
        residual_forward_kernel<T, 2, false, HAS_Y, HAS_H><<<grid, kThreads, 0, s>>>(rows, by, reals, lpr, whole, a, drop, eps);
    else if (reals <= 2048)
        residual_forward_kernel<T, 1, true, HAS_Y, HAS_H><<<grid, kThreads, 0, s>>>(rows, by, reals, lpr, whole, a, drop, eps);
    else
        residual_forward_kernel<T, 2, true, HAS_Y, HAS_H><<<grid, kThreads, 0, s>>>(rows, by, reals, lpr, whole, a, drop, eps);
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
    if (reals <= 512)
        residual_backward_kernel<T, 1, false, HAS_Y, HAS_H><<<d.grid, kThreads, 0, s>>>(d, reals, lpr, whole, a, drop, eps, part);
    else if (reals <= 1024)
        residual_backward_kernel<T, 2, false, HAS_Y, HAS_H><<<d.grid, kThreads, 0, s>>>(d, reals, lpr, whole, a, drop, eps, part);
    else if (reals <= 2048)
        residual_backward_kernel<T, 1, true, HAS_Y, HAS_H><<<d.grid, kThreads, 0, s>>>(d, reals, lpr, whole, a, drop, eps, part);
    else
        residual_backward_kernel<T, 2, true, HAS_Y, HAS_H><<<d.grid, kThreads, 0, s>>>(d, reals, lpr, whole, a, drop, eps, part);
    if (hipError_t e = hipGetLastError())
        return e;
    if (a.dgate == nullptr && a.dgamma == nullptr && a.dscale == nullptr && a.dnext_gamma == nullptr)
        return hipSuccess;
    const int64_t entries = a.gate != nullptr ? d.n : d.bpi;
    const dim3 grid(unsigned((reals + kCols - 1) / kCols));
    if (a.gate != nullptr && d.bpi > 1) {
        // (bpi > 1 only where n < kBackwardGroups: n fits the grid)
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
    // max(n, kBackwardGroups) rows of partial sums, and of sums by image
    const size_t row = size_t(8) * g.c, n = a.gate != nullptr ? size_t(g.n) : 1;
    return (std::max<size_t>(n, kBackwardGroups) * sizeof(float) +
            std::min<size_t>(n, kBackwardGroups) * sizeof(double)) * row;
}

hipError_t residual_backward_run(const RowsGeom &g, DType dt, const ResidualBackward &a, const Drop &drop, float eps,
                                 void *work, hipStream_t s)
{
    const bool has_y = a.y != nullptr, has_h = a.dh != nullptr;
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
