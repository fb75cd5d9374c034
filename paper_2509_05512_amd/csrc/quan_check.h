// What the C ABI's files check their arguments with: maps given as descriptors,
// spans of memory that may not overlap.  Host only, nothing here calls HIP.
#pragma once

#include <hip/hip_runtime_api.h>

#include <initializer_list>

#include "quan.h"
#include "quan_block.h"

namespace {

using quan::report;

bool misaligned(const void *p, size_t a)
{
    return reinterpret_cast<uintptr_t>(p) % a != 0;
}

// A range of device memory, and what lies in it: everything, or the channels
// of a map (for which strides are multiples of the component stride, or not).
struct Span {
    const char *what;
    const void *p;
    size_t bytes;
    int64_t period = 0, width = 0;  // bytes: the range's [k period, k period + width) alone, 0: all of it
};

bool overlap(const Span &a, const Span &b)
{
    if (a.p == nullptr || b.p == nullptr)
        return false;
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a.p), b0 = reinterpret_cast<uintptr_t>(b.p);
    if (!(a0 < b0 + b.bytes && b0 < a0 + a.bytes))
        return false;
    if (a.period > 0 && a.period == b.period) {
        // slices of one map: disjoint where their channels are
        const int64_t p = a.period;
        const int64_t d = ((int64_t(b0) - int64_t(a0)) % p + p) % p;
        return !(d >= a.width && d + b.width <= p);
    }
    return true;
}

int check_dtype(const char *fn, int32_t dtype)
{
    if (dtype != QUAN_F32 && dtype != QUAN_BF16)
        return report(QUAN_ERR_DTYPE, "%s: dtype %d is neither QUAN_F32 (0) nor QUAN_BF16 (1)", fn, dtype);
    return QUAN_OK;
}

size_t elem_size(int32_t dtype)
{
    return dtype == QUAN_BF16 ? 2 : 4;
}

quan::DType to_dt(int32_t dtype)
{
    return dtype == QUAN_BF16 ? quan::DType::BF16 : quan::DType::F32;
}

constexpr int64_t kMaxSpan = int64_t(1) << 48;  // elements from a map's first to its last
constexpr int64_t kMaxPixels = (int64_t(1) << 31) - 1, kMaxImagePixels = int64_t(1) << 24;
// Work-groups of 256 lanes (in eights) that a launch may have: a grid's axis holds
// less than 2^32 lanes.
constexpr int64_t kMaxLanes = (int64_t(1) << 32) - 1, kMaxGroups = kMaxLanes / 256 / 8 * 8;

// `out` against everything else; `same` are those it may equal.
int check_alias(const char *fn, const Span &out, std::initializer_list<Span> others,
                std::initializer_list<const void *> same = {})
{
    for (const Span &o : others) {
        bool allowed = false;
        for (const void *s : same)
            allowed = allowed || (s != nullptr && o.p == s && out.p == s);
        if (!allowed && overlap(out, o))
            return report(QUAN_ERR_ALIAS, "%s: %s overlaps %s", fn, out.what, o.what);
    }
    return QUAN_OK;
}

// A map descriptor: logical [N, 4, C, H, W], channels side by side, pixels at
// one stride, images, pixels and components nested in that order.
int check_map(const char *fn, const char *what, const quan_tensor *t, int32_t dtype, const int64_t want[5],
              quan::AttnMap *m, Span *span)
{
    if (t == nullptr || t->data == nullptr)
        return report(QUAN_ERR_NULL, "%s: %s must be non-NULL", fn, what);
    if (t->ndim != 5)
        return report(QUAN_ERR_SHAPE, "%s: %s has %d axes, not 5 ([N, 4, C, H, W])", fn, what, t->ndim);
    if (t->dtype != dtype)
        return report(QUAN_ERR_DTYPE, "%s: %s has dtype %d, q %d", fn, what, t->dtype, dtype);
    for (int i = 0; i < 5; ++i)
        if (want[i] >= 0 && t->shape[i] != want[i])
            return report(QUAN_ERR_SHAPE, "%s: %s has extent %lld on axis %d, not %lld", fn, what,
                          (long long)t->shape[i], i, (long long)want[i]);
    for (int i = 0; i < 5; ++i)
        if (t->shape[i] < 1)
            return report(QUAN_ERR_SHAPE, "%s: %s has an axis of extent %lld", fn, what, (long long)t->shape[i]);
        else if (t->shape[i] > kMaxPixels)
            return report(QUAN_ERR_UNSUPPORTED, "%s: %s has an extent of 2^31 or more", fn, what);
    const int64_t n = t->shape[0], c = t->shape[2], h = t->shape[3], w = t->shape[4];
    if (h * w > kMaxImagePixels)
        return report(QUAN_ERR_UNSUPPORTED, "%s: images of %s have more than 2^24 pixels", fn, what);
    for (int i = 0; i < 5; ++i)
        if (t->shape[i] > 1 && (t->strides[i] < 1 || t->strides[i] > int64_t(1) << 40))
            return report(QUAN_ERR_LAYOUT, "%s: %s has stride %lld on axis %d", fn, what, (long long)t->strides[i], i);
    const int64_t s_p = t->strides[1];
    const int64_t s_t = w > 1 ? t->strides[4] : h > 1 ? t->strides[3] : 4 * s_p;
    // (nothing below leaves 64 bits)
    if (s_t > kMaxSpan / (h * w) || (n > 1 && t->strides[0] > kMaxSpan / n))
        return report(QUAN_ERR_UNSUPPORTED, "%s: %s spans more than 2^48 elements", fn, what);
    const int64_t s_n = n > 1 ? t->strides[0] : h * w * s_t;
    if ((c > 1 && t->strides[2] != 1) || (h > 1 && w > 1 && t->strides[3] != w * s_t) || s_p < c ||
        s_t < 3 * s_p + c || s_n < (h * w - 1) * s_t + 3 * s_p + c)
        return report(QUAN_ERR_LAYOUT,
                      "%s: %s must have its channels side by side, its pixels in row order at one stride, and "
                      "ascending strides of components, pixels and images",
                      fn, what);
    const size_t es = elem_size(dtype);
    if (misaligned(t->data, es))
        return report(QUAN_ERR_ALIGN, "%s: %s must be aligned to its element", fn, what);
    const int64_t chunk = 16 / int64_t(es);
    *m = {t->data, s_n, s_t, s_p,
          !misaligned(t->data, 16) && s_n % chunk == 0 && s_t % chunk == 0 && s_p % chunk == 0, 0};
    const int64_t last = (n - 1) * s_n + (h * w - 1) * s_t + 3 * s_p + c;
    *span = {what, t->data, size_t(last) * es};
    if ((n == 1 || s_n % s_p == 0) && s_t % s_p == 0) {
        span->period = s_p * int64_t(es);
        span->width = c * int64_t(es);
    }
    return QUAN_OK;
}

// A lane takes 8 reals of a head at a time.
void for_heads(quan::AttnMap *m, int dq)
{
    m->s_h = dq;
    m->vec = m->vec && dq % 8 == 0;
}

// A bias by buckets, and the memory that it lies in.
int check_relpos(const char *fn, const quan_relpos *relpos, int32_t heads, quan::AttnBias *bias, Span *table, Span *by,
                 Span *bx)
{
    if (relpos->table == nullptr)
        return report(QUAN_ERR_NULL, "%s: relpos->table must be non-NULL", fn);
    if (relpos->buckets_y < 1 || relpos->buckets_x < 1 || relpos->radius_y < 0 || relpos->radius_x < 0)
        return report(QUAN_ERR_SHAPE, "%s: relpos needs at least one bucket per axis and radii >= 0", fn);
    if (relpos->buckets_y > quan::kAttnMaxBuckets || relpos->buckets_x > quan::kAttnMaxBuckets ||
        relpos->radius_y > kMaxImagePixels || relpos->radius_x > kMaxImagePixels)
        return report(QUAN_ERR_UNSUPPORTED, "%s: at most %d buckets per axis and radii of 2^24", fn,
                      quan::kAttnMaxBuckets);
    if (misaligned(relpos->table, 4) || misaligned(relpos->bucket_y, 4) || misaligned(relpos->bucket_x, 4))
        return report(QUAN_ERR_ALIGN, "%s: relpos's arrays must be 4-byte aligned", fn);
    *bias = {relpos->table,     relpos->bucket_y, relpos->bucket_x, relpos->buckets_y,
             relpos->buckets_x, relpos->radius_y, relpos->radius_x};
    *table = {"relpos->table", relpos->table, size_t(heads) * relpos->buckets_y * relpos->buckets_x * 4};
    *by = {"relpos->bucket_y", relpos->bucket_y, (size_t(2) * relpos->radius_y + 1) * 4};
    *bx = {"relpos->bucket_x", relpos->bucket_x, (size_t(2) * relpos->radius_x + 1) * 4};
    return QUAN_OK;
}

int launched(hipError_t e, const char *fn)
{
    if (e != hipSuccess)
        return report(QUAN_ERR_HIP, "%s launch: %s (%d)", fn, hipGetErrorString(e), int(e));
    return QUAN_OK;
}

}  // namespace
