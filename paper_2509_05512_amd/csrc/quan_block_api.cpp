// C ABI of the attention block: argument validation and dispatch.  As in
// quan_api.cpp, everything is checked on the host before the first HIP call.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cmath>
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

// ------------------------------------------------------------------ the rows

int check_rows(const char *fn, int32_t n, int32_t c, int32_t h, int32_t w, int32_t dtype, float eps,
               int32_t max_channels, quan::RowsGeom *g)
{
    if (int rc = check_dtype(fn, dtype))
        return rc;
    if (n < 1 || c < 1 || h < 1 || w < 1)
        return report(QUAN_ERR_SHAPE, "%s: sizes must be >= 1 (n=%d c=%d h=%d w=%d)", fn, n, c, h, w);
    if (!(eps > 0.0f) || std::isinf(eps))
        return report(QUAN_ERR_SHAPE, "%s: eps must be > 0 and finite (got %g)", fn, double(eps));
    if (c > max_channels)
        return report(QUAN_ERR_UNSUPPORTED, "%s: %d channels, at most %d are supported", fn, c, max_channels);
    // (n * h * w overflows no 64-bit integer before the first comparison)
    const int64_t hw = int64_t(h) * w;
    if (hw > kMaxPixels || hw * n > kMaxPixels)
        return report(QUAN_ERR_UNSUPPORTED, "%s: more than 2^31-1 pixels", fn);
    *g = {n, hw, c};
    return QUAN_OK;
}

int check_drop(const char *fn, float p, const uint64_t *rng, quan::Drop *d)
{
    if (!(p >= 0.0f && p < 1.0f))
        return report(QUAN_ERR_SHAPE, "%s: p must be in [0, 1) (got %g)", fn, double(p));
    if (p > 0.0f && rng == nullptr)
        return report(QUAN_ERR_NULL, "%s: rng must be non-NULL with p > 0", fn);
    if (misaligned(rng, 8))
        return report(QUAN_ERR_ALIGN, "%s: rng must be 8-byte aligned", fn);
    long cut = std::lrint(double(p) * 65536.0);
    if (cut > 65535)
        cut = 65535;
    *d = {rng, unsigned(cut), float(65536.0 / double(65536 - cut))};
    return QUAN_OK;
}

int check_maps(const char *fn, std::initializer_list<Span> maps)
{
    for (const Span &m : maps)
        if (misaligned(m.p, 16))
            return report(QUAN_ERR_ALIGN, "%s: %s must be 16-byte aligned", fn, m.what);
    return QUAN_OK;
}

int check_params(const char *fn, std::initializer_list<Span> params)
{
    for (const Span &m : params)
        if (misaligned(m.p, 4))
            return report(QUAN_ERR_ALIGN, "%s: %s must be 4-byte aligned", fn, m.what);
    return QUAN_OK;
}

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

struct ForwardRows {
    quan::RowsGeom g;
    quan::DType dt;
    quan::ResidualForward a;
    quan::Drop drop;
    float eps;
};
hipError_t run_forward_rows(const ForwardRows &r, void *stream)
{
    return quan::residual_forward_run(r.g, r.dt, r.a, r.drop, r.eps, static_cast<hipStream_t>(stream));
}

struct BackwardRows {
    quan::RowsGeom g;
    quan::DType dt;
    quan::ResidualBackward a;
    quan::Drop drop;
    float eps;
};
hipError_t run_backward_rows(void *args, void *work, void *, hipStream_t s)
{
    const BackwardRows &r = *static_cast<BackwardRows *>(args);
    return quan::residual_backward_run(r.g, r.dt, r.a, r.drop, r.eps, work, s);
}

int launched(hipError_t e, const char *fn)
{
    if (e != hipSuccess)
        return report(QUAN_ERR_HIP, "%s launch: %s (%d)", fn, hipGetErrorString(e), int(e));
    return QUAN_OK;
}

// ------------------------------------------------------------- the attention

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

struct Spans {
    Span q, k, v, table, by, bx, kv_len, pos;
};

// What both directions share.
int check_call(const char *fn, const quan_tensor *q, const quan_tensor *k, const quan_tensor *v,
               const quan_relpos *relpos, const int32_t *kv_len, const int32_t *pos, float scale, int32_t heads,
               quan::AttnCall *a, Spans *s)
{
    if (q == nullptr || k == nullptr || v == nullptr)
        return report(QUAN_ERR_NULL, "%s: q, k and v must be non-NULL", fn);
    const int32_t dtype = q->dtype;
    if (int rc = check_dtype(fn, dtype))
        return rc;
    const int64_t q_want[5] = {-1, 4, -1, -1, -1};
    if (int rc = check_map(fn, "q", q, dtype, q_want, &a->q, &s->q))
        return rc;
    const int64_t k_want[5] = {q->shape[0], 4, -1, -1, -1};
    if (int rc = check_map(fn, "k", k, dtype, k_want, &a->k, &s->k))
        return rc;
    const int64_t v_want[5] = {k->shape[0], 4, k->shape[2], k->shape[3], k->shape[4]};
    if (int rc = check_map(fn, "v", v, dtype, v_want, &a->v, &s->v))
        return rc;
    const int64_t c = q->shape[2], ckv = k->shape[2];
    if (heads < 1 || c % heads != 0)
        return report(QUAN_ERR_SHAPE, "%s: %d heads do not divide %lld channels", fn, heads, (long long)c);
    const int64_t dq = c / heads;
    if (dq > quan::kAttnMaxDq)
        return report(QUAN_ERR_UNSUPPORTED, "%s: heads of %lld quaternion channels, at most %d are supported", fn,
                      (long long)dq, quan::kAttnMaxDq);
    if (ckv % dq != 0 || heads % (ckv / dq) != 0)
        return report(QUAN_ERR_SHAPE, "%s: %lld channels of k are no whole number of heads that divides %d", fn,
                      (long long)ckv, heads);
    if (heads > 65535)
        return report(QUAN_ERR_UNSUPPORTED, "%s: more than 65535 heads", fn);
    if (!std::isfinite(scale))
        return report(QUAN_ERR_SHAPE, "%s: scale must be finite", fn);
    if (misaligned(kv_len, 4) || misaligned(pos, 4))
        return report(QUAN_ERR_ALIGN, "%s: kv_len and pos must be 4-byte aligned", fn);
    quan::AttnGeom &g = a->g;
    g = {int(q->shape[0]), heads,           int(ckv / dq),    int(dq), int(q->shape[3]),
         int(q->shape[4]), int(k->shape[3]), int(k->shape[4]), scale};
    // a work-group takes 128 queries of a head and image, or a part of one's keys
    const int64_t blocks = (std::max(g.lq(), g.lk()) + 63) / 64;
    if (blocks * g.n > kMaxPixels / 2 / heads || (g.lq() + 127) / 128 * int64_t(g.n) * heads > kMaxGroups)
        return report(QUAN_ERR_UNSUPPORTED, "%s: too many work-groups", fn);
    for (quan::AttnMap *m : {&a->q, &a->k, &a->v})
        for_heads(m, g.dq);
    a->kv_len = kv_len;
    a->pos = pos;
    a->bias = {};
    s->kv_len = {"kv_len", kv_len, size_t(g.n) * 4};
    s->pos = {"pos", pos, size_t(g.n) * 8};
    s->table = s->by = s->bx = {"relpos", nullptr, 0};
    if (relpos != nullptr) {
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
        if ((g.hq > 1 || g.hk > 1) && std::max(g.wq, g.wk) > quan::kAttnMaxWidth)
            return report(QUAN_ERR_UNSUPPORTED, "%s: with a bias, maps of several rows may be %d pixels wide", fn,
                          quan::kAttnMaxWidth);
        if (int64_t(g.hk + g.hq) * (g.wk + g.wq) > kMaxPixels)
            return report(QUAN_ERR_UNSUPPORTED, "%s: too many offsets between q's and k's pixels", fn);
        a->bias = {relpos->table,     relpos->bucket_y,  relpos->bucket_x, relpos->buckets_y,
                   relpos->buckets_x, relpos->radius_y, relpos->radius_x};
        s->table = {"relpos->table", relpos->table, size_t(heads) * relpos->buckets_y * relpos->buckets_x * 4};
        s->by = {"relpos->bucket_y", relpos->bucket_y, (size_t(2) * relpos->radius_y + 1) * 4};
        s->bx = {"relpos->bucket_x", relpos->bucket_x, (size_t(2) * relpos->radius_x + 1) * 4};
    }
    return QUAN_OK;
}

// A tile's offsets have to fit in LDS: narrow maps against wide ones have many.
int check_offsets(const char *fn, bool fits, const char *of)
{
    if (!fits)
        return report(QUAN_ERR_UNSUPPORTED,
                      "%s: the offsets between 128 pixels of one map and a tile of the other do not fit in a "
                      "work-group's memory%s",
                      fn, of);
    return QUAN_OK;
}

struct ForwardCall {
    quan::AttnCall a;
    quan::DType dt;
    quan::AttnMap out;
    void *rest;
    float *stats;
};
hipError_t run_forward(void *args, void *work, void *extra, hipStream_t s)
{
    const ForwardCall &c = *static_cast<ForwardCall *>(args);
    return quan::attention_forward_run(c.a, c.dt, c.out, c.rest, c.stats, work, extra, s);
}

struct BackwardCall {
    quan::AttnCall a;
    quan::DType dt;
    quan::AttnGradients g;
};
hipError_t run_backward(void *args, void *work, void *, hipStream_t s)
{
    const BackwardCall &c = *static_cast<BackwardCall *>(args);
    return quan::attention_backward_run(c.a, c.dt, c.g, work, s);
}

size_t dense_bytes(const quan_tensor *t)
{
    return size_t(t->shape[0]) * 4 * t->shape[2] * t->shape[3] * t->shape[4] * elem_size(t->dtype);
}

}  // namespace

extern "C" {

QUAN_API int quan_relpos_buckets(int32_t radius, int32_t buckets, int32_t *map)
{
    quan::clear_error();
    if (map == nullptr)
        return report(QUAN_ERR_NULL, "relpos_buckets: map must be non-NULL");
    if (radius < 0 || buckets < 1)
        return report(QUAN_ERR_SHAPE, "relpos_buckets: radius must be >= 0 and buckets >= 1");
    if (radius > kMaxImagePixels || buckets > quan::kAttnMaxBuckets)
        return report(QUAN_ERR_UNSUPPORTED, "relpos_buckets: at most a radius of 2^24 and %d buckets",
                      quan::kAttnMaxBuckets);
    const int half = buckets / 2, near = half / 2 > 1 ? half / 2 : 1;
    for (int d = -radius; d <= radius; ++d) {
        int b;
        if (buckets >= 2 * radius + 1) {
            b = d + radius;
        } else if (half < 1) {
            b = 0;
        } else {
            const int a = d < 0 ? -d : d;
            b = a;
            if (a >= near && radius > near)
                b = near + int(std::log(double(a) / near) / std::log(double(radius) / near) * (half - near));
            b = (b < half - 1 ? b : half - 1) + (d > 0 ? half : 0);
        }
        map[d + radius] = b;
    }
    return QUAN_OK;
}

QUAN_API int quan_attention_forward(const quan_tensor *q, const quan_tensor *k, const quan_tensor *v,
                                    const quan_relpos *relpos, const int32_t *kv_len, const int32_t *pos,
                                    float scale, int32_t heads, quan_tensor *out, void *rest, float *stats,
                                    void *stream)
{
    const char *fn = "attention_forward";
    quan::clear_error();
    ForwardCall c{};
    Spans s;
    if (int rc = check_call(fn, q, k, v, relpos, kv_len, pos, scale, heads, &c.a, &s))
        return rc;
    Span out_span;
    if (int rc = check_map(fn, "out", out, q->dtype, q->shape, &c.out, &out_span))
        return rc;
    if (rest != nullptr && q->dtype != QUAN_BF16)
        return report(QUAN_ERR_DTYPE, "%s: rest is for bf16 maps", fn);
    if (misaligned(rest, 16))
        return report(QUAN_ERR_ALIGN, "%s: rest must be 16-byte aligned", fn);
    if (misaligned(stats, 4))
        return report(QUAN_ERR_ALIGN, "%s: stats must be 4-byte aligned", fn);
    c.dt = to_dt(q->dtype);
    if (int rc = check_offsets(fn, quan::attention_forward_fits(c.a, c.dt), ""))
        return rc;
    if (stats != nullptr)
        if (int rc = check_offsets(fn, quan::attention_backward_fits(c.a, c.dt, {}), " (of its backward pass)"))
            return rc;
    const Span rest_span{"rest", rest, dense_bytes(q)};
    const Span stats_span{"stats", stats, size_t(c.a.g.n) * heads * c.a.g.lq() * 8};
    for (const Span &o : {out_span, rest_span, stats_span})
        if (int rc = check_alias(fn, o, {s.q, s.k, s.v, s.table, s.by, s.bx, s.kv_len, s.pos}))
            return rc;
    if (int rc = check_alias(fn, out_span, {rest_span, stats_span}))
        return rc;
    if (int rc = check_alias(fn, rest_span, {stats_span}))
        return rc;
    for_heads(&c.out, c.a.g.dq);
    c.rest = rest;
    c.stats = stats;
    const size_t bytes = quan::attention_forward_work_bytes(c.a, c.dt);
    const size_t extra = quan::attention_forward_extra_bytes(c.a, c.dt);
    if (bytes == 0 && extra == 0)
        return launched(run_forward(&c, nullptr, nullptr, static_cast<hipStream_t>(stream)), fn);
    return quan::run_on_stream(stream, bytes, extra, run_forward, &c, fn);
}

QUAN_API int quan_attention_backward(const quan_tensor *q, const quan_tensor *k, const quan_tensor *v,
                                     const quan_relpos *relpos, const int32_t *kv_len, const int32_t *pos,
                                     float scale, int32_t heads, const quan_tensor *out, const void *rest,
                                     const float *stats, const quan_tensor *dout, quan_tensor *dq,
                                     quan_tensor *dk, quan_tensor *dv, float *dtable, void *stream)
{
    const char *fn = "attention_backward";
    quan::clear_error();
    BackwardCall c{};
    Spans s;
    if (int rc = check_call(fn, q, k, v, relpos, kv_len, pos, scale, heads, &c.a, &s))
        return rc;
    Span out_span, dout_span, dq_span, dk_span, dv_span;
    if (int rc = check_map(fn, "out", out, q->dtype, q->shape, &c.g.out, &out_span))
        return rc;
    if (int rc = check_map(fn, "dout", dout, q->dtype, q->shape, &c.g.dout, &dout_span))
        return rc;
    if (int rc = check_map(fn, "dq", dq, q->dtype, q->shape, &c.g.dq, &dq_span))
        return rc;
    if (int rc = check_map(fn, "dk", dk, q->dtype, k->shape, &c.g.dk, &dk_span))
        return rc;
    if (int rc = check_map(fn, "dv", dv, q->dtype, k->shape, &c.g.dv, &dv_span))
        return rc;
    if (stats == nullptr)
        return report(QUAN_ERR_NULL, "%s: stats must be non-NULL", fn);
    if (dtable != nullptr && relpos == nullptr)
        return report(QUAN_ERR_NULL, "%s: dtable without relpos", fn);
    if (rest != nullptr && q->dtype != QUAN_BF16)
        return report(QUAN_ERR_DTYPE, "%s: rest is for bf16 maps", fn);
    if (misaligned(rest, 16))
        return report(QUAN_ERR_ALIGN, "%s: rest must be 16-byte aligned", fn);
    const quan::AttnGeom &g = c.a.g;
    if ((g.lk() + 127) / 128 * int64_t(g.n) * g.kv_heads > kMaxGroups)
        return report(QUAN_ERR_UNSUPPORTED, "%s: too many work-groups", fn);
    // (4 lanes per offset, 512 per row of buckets)
    if (dtable != nullptr && (int64_t(g.hk + g.hq) * (g.wk + g.wq) > kMaxLanes / 4 - 64 ||
                              int64_t(heads) * relpos->buckets_y > kMaxLanes / 512))
        return report(QUAN_ERR_UNSUPPORTED, "%s: too many offsets or buckets for dtable", fn);
    if (misaligned(stats, 4) || misaligned(dtable, 4))
        return report(QUAN_ERR_ALIGN, "%s: stats and dtable must be 4-byte aligned", fn);
    const Span rest_span{"rest", rest, dense_bytes(q)};
    const Span stats_span{"stats", stats, size_t(c.a.g.n) * heads * c.a.g.lq() * 8};
    const Span dtable_span{"dtable", dtable, s.table.bytes};
    c.dt = to_dt(q->dtype);
    c.g.dtable = dtable;
    if (int rc = check_offsets(fn, quan::attention_backward_fits(c.a, c.dt, c.g), dtable != nullptr ? " (with dtable)" : ""))
        return rc;
    for (const Span &o : {dq_span, dk_span, dv_span, dtable_span})
        if (int rc = check_alias(fn, o, {s.q, s.k, s.v, s.table, s.by, s.bx, s.kv_len, s.pos, out_span, rest_span,
                                         stats_span, dout_span}))
            return rc;
    if (int rc = check_alias(fn, dq_span, {dk_span, dv_span, dtable_span}))
        return rc;
    if (int rc = check_alias(fn, dk_span, {dv_span, dtable_span}))
        return rc;
    if (int rc = check_alias(fn, dv_span, {dtable_span}))
        return rc;
    for (quan::AttnMap *m : {&c.g.out, &c.g.dout, &c.g.dq, &c.g.dk, &c.g.dv})
        for_heads(m, c.a.g.dq);
    c.g.rest = rest;
    c.g.stats = stats;
    return quan::run_on_stream(stream, quan::attention_backward_work_bytes(c.a, c.dt, c.g), 0, run_backward, &c, fn);
}

QUAN_API int quan_rmsnorm_forward(const void *x, const float *gamma, float eps, void *out, int32_t n, int32_t c,
                                  int32_t h, int32_t w, int32_t dtype, void *stream)
{
    const char *fn = "rmsnorm_forward";
    quan::clear_error();
    if (!x || !gamma || !out)
        return report(QUAN_ERR_NULL, "%s: x, gamma and out must be non-NULL", fn);
    ForwardRows r{};
    if (int rc = check_rows(fn, n, c, h, w, dtype, eps, quan::kRowsMaxChannels, &r.g))
        return rc;
    const size_t bytes = size_t(r.g.n) * r.g.hw * 4 * c * elem_size(dtype), row = size_t(16) * c;
    const Span xs{"x", x, bytes}, os{"out", out, bytes}, gs{"gamma", gamma, row};
    if (int rc = check_maps(fn, {xs, os}))
        return rc;
    if (int rc = check_params(fn, {gs}))
        return rc;
    if (int rc = check_alias(fn, os, {xs, gs}, {x}))
        return rc;
    r.dt = to_dt(dtype);
    r.a.x = x;
    r.a.next_gamma = gamma;
    r.a.h = out;
    r.eps = eps;
    return launched(run_forward_rows(r, stream), fn);
}

QUAN_API int quan_rmsnorm_backward(const void *x, const void *dout, const float *gamma, const void *dres, float eps,
                                   void *dx, float *dgamma, int32_t n, int32_t c, int32_t h, int32_t w,
                                   int32_t dtype, void *stream)
{
    const char *fn = "rmsnorm_backward";
    quan::clear_error();
    if (!x || !dout || !gamma || !dx || !dgamma)
        return report(QUAN_ERR_NULL, "%s: x, dout, gamma, dx and dgamma must be non-NULL", fn);
    BackwardRows r{};
    if (int rc = check_rows(fn, n, c, h, w, dtype, eps, quan::kRowsMaxChannels, &r.g))
        return rc;
    const size_t bytes = size_t(r.g.n) * r.g.hw * 4 * c * elem_size(dtype), row = size_t(16) * c;
    const Span xs{"x", x, bytes}, ds{"dout", dout, bytes}, rs{"dres", dres, bytes}, dxs{"dx", dx, bytes};
    const Span gs{"gamma", gamma, row}, dgs{"dgamma", dgamma, row};
    if (int rc = check_maps(fn, {xs, ds, rs, dxs}))
        return rc;
    if (int rc = check_params(fn, {gs, dgs}))
        return rc;
    if (int rc = check_alias(fn, dxs, {xs, ds, rs, gs, dgs}, {dres, dout}))
        return rc;
    if (int rc = check_alias(fn, dgs, {xs, ds, rs, gs}))
        return rc;
    r.dt = to_dt(dtype);
    r.a.out = x;
    r.a.dh = dout;
    r.a.dout = dres;
    r.a.next_gamma = gamma;
    r.a.dx = dx;
    r.a.dnext_gamma = dgamma;
    r.eps = eps;
    return quan::run_on_stream(stream, quan::residual_backward_work_bytes(r.g, r.a), 0, run_backward_rows, &r, fn);
}

QUAN_API int quan_residual_forward(const void *x, const void *y, const void *gate, const float *gamma,
                                   const float *scale, const float *next_gamma, float p, const uint64_t *rng,
                                   float eps, void *out, void *h, int32_t n, int32_t c, int32_t height, int32_t w,
                                   int32_t dtype, void *stream)
{
    const char *fn = "residual_forward";
    quan::clear_error();
    if (!x || !y || !out)
        return report(QUAN_ERR_NULL, "%s: x, y and out must be non-NULL", fn);
    if ((h == nullptr) != (next_gamma == nullptr))
        return report(QUAN_ERR_NULL, "%s: h and next_gamma come together", fn);
    ForwardRows r{};
    if (int rc = check_rows(fn, n, c, height, w, dtype, eps, quan::kRowsMaxChannels, &r.g))
        return rc;
    if (int rc = check_drop(fn, p, rng, &r.drop))
        return rc;
    const size_t es = elem_size(dtype), bytes = size_t(r.g.n) * r.g.hw * 4 * c * es, row = size_t(16) * c;
    const Span xs{"x", x, bytes}, ys{"y", y, bytes}, gts{"gate", gate, size_t(n) * 4 * c * es};
    const Span os{"out", out, bytes}, hs{"h", h, bytes}, rs{"rng", rng, 16};
    const Span gs{"gamma", gamma, row}, ss{"scale", scale, row}, ns{"next_gamma", next_gamma, row};
    if (int rc = check_maps(fn, {xs, ys, gts, os, hs}))
        return rc;
    if (int rc = check_params(fn, {gs, ss, ns}))
        return rc;
    if (int rc = check_alias(fn, os, {xs, ys, gts, hs, rs, gs, ss, ns}, {x, y}))
        return rc;
    if (int rc = check_alias(fn, hs, {xs, ys, gts, rs, gs, ss, ns}))
        return rc;
    r.dt = to_dt(dtype);
    r.a = {x, y, gamma, scale, next_gamma, gate, out, h};
    r.eps = eps;
    return launched(run_forward_rows(r, stream), fn);
}

QUAN_API int quan_residual_backward(const void *y, const void *dout, const void *out, const void *dh,
                                    const void *gate, const float *gamma, const float *scale,
                                    const float *next_gamma, float p, const uint64_t *rng, float eps, void *dx,
                                    void *dy, void *dgate, float *dgamma, float *dscale, float *dnext_gamma,
                                    int32_t n, int32_t c, int32_t h, int32_t w, int32_t dtype, void *stream)
{
    const char *fn = "residual_backward";
    quan::clear_error();
    if (!y || !dout || !dx || !dy)
        return report(QUAN_ERR_NULL, "%s: y, dout, dx and dy must be non-NULL", fn);
    const bool following = next_gamma != nullptr;
    if ((out != nullptr) != following || (dh != nullptr) != following || (dnext_gamma != nullptr) != following)
        return report(QUAN_ERR_NULL, "%s: out, dh, next_gamma and dnext_gamma come together", fn);
    if ((dgate != nullptr) != (gate != nullptr) || (dgamma != nullptr) != (gamma != nullptr) ||
        (dscale != nullptr) != (scale != nullptr))
        return report(QUAN_ERR_NULL, "%s: gate, gamma and scale come with their gradients", fn);
    BackwardRows r{};
    if (int rc = check_rows(fn, n, c, h, w, dtype, eps, quan::kRowsMaxChannels, &r.g))
        return rc;
    if (int rc = check_drop(fn, p, rng, &r.drop))
        return rc;
    const size_t es = elem_size(dtype), bytes = size_t(r.g.n) * r.g.hw * 4 * c * es, row = size_t(16) * c;
    const size_t gate_bytes = size_t(n) * 4 * c * es;
    const Span ys{"y", y, bytes}, ds{"dout", dout, bytes}, os{"out", out, bytes}, hs{"dh", dh, bytes};
    const Span gts{"gate", gate, gate_bytes}, rs{"rng", rng, 16};
    const Span gs{"gamma", gamma, row}, ss{"scale", scale, row}, ns{"next_gamma", next_gamma, row};
    const Span dxs{"dx", dx, bytes}, dys{"dy", dy, bytes}, dgts{"dgate", dgate, gate_bytes};
    const Span dgs{"dgamma", dgamma, row}, dss{"dscale", dscale, row}, dns{"dnext_gamma", dnext_gamma, row};
    if (int rc = check_maps(fn, {ys, ds, os, hs, gts, dxs, dys, dgts}))
        return rc;
    if (int rc = check_params(fn, {gs, ss, ns, dgs, dss, dns}))
        return rc;
    if (int rc = check_alias(fn, dxs, {ys, ds, os, hs, gts, rs, gs, ss, ns, dys, dgts, dgs, dss, dns}, {dout, dh}))
        return rc;
    if (int rc = check_alias(fn, dys, {ys, ds, os, hs, gts, rs, gs, ss, ns, dgts, dgs, dss, dns}, {y}))
        return rc;
    if (int rc = check_alias(fn, dgts, {ys, ds, os, hs, gts, rs, gs, ss, ns, dgs, dss, dns}))
        return rc;
    if (int rc = check_alias(fn, dgs, {ys, ds, os, hs, gts, rs, gs, ss, ns, dss, dns}))
        return rc;
    if (int rc = check_alias(fn, dss, {ys, ds, os, hs, gts, rs, gs, ss, ns, dns}))
        return rc;
    if (int rc = check_alias(fn, dns, {ys, ds, os, hs, gts, rs, gs, ss, ns}))
        return rc;
    r.dt = to_dt(dtype);
    r.a = {y, dout, out, dh, gamma, scale, next_gamma, gate, dx, dy, dgate, dgamma, dscale, dnext_gamma};
    r.eps = eps;
    return quan::run_on_stream(stream, quan::residual_backward_work_bytes(r.g, r.a), 0, run_backward_rows, &r, fn);
}

QUAN_API int quan_dropout(const void *x, float p, const uint64_t *rng, void *out, int32_t n, int32_t c, int32_t h,
                          int32_t w, int32_t dtype, void *stream)
{
    const char *fn = "dropout";
    quan::clear_error();
    if (!x || !out)
        return report(QUAN_ERR_NULL, "%s: x and out must be non-NULL", fn);
    quan::RowsGeom g;
    quan::Drop drop;
    if (int rc = check_rows(fn, n, c, h, w, dtype, 1.0f, 1 << 28, &g))
        return rc;
    if (int rc = check_drop(fn, p, rng, &drop))
        return rc;
    const size_t bytes = size_t(g.n) * g.hw * 4 * c * elem_size(dtype);
    const Span xs{"x", x, bytes}, os{"out", out, bytes}, rs{"rng", rng, 16};
    if (int rc = check_maps(fn, {xs, os}))
        return rc;
    if (int rc = check_alias(fn, os, {xs, rs}, {x}))
        return rc;
    return launched(quan::dropout_run(g, to_dt(dtype), x, out, drop, static_cast<hipStream_t>(stream)), fn);
}

}  // extern "C"
