// C ABI of the operators on sequences of pixels: argument validation and
// dispatch.  Everything is checked on the host before the first HIP call.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "quan_check.h"
#include "quan_sequence.h"

namespace {

constexpr int64_t kMaxInt = (int64_t(1) << 31) - 1;

int check_format(const char *fn, int32_t dq, int32_t format)
{
    if (format != QUAN_CACHE_F32 && format != QUAN_CACHE_BF16 && format != QUAN_CACHE_E4M3)
        return report(QUAN_ERR_DTYPE, "%s: format %d is no quan_cache_format", fn, format);
    if (dq < 1)
        return report(QUAN_ERR_SHAPE, "%s: heads of %d quaternion channels", fn, dq);
    if (dq > quan::kAttnMaxDq)
        return report(QUAN_ERR_UNSUPPORTED, "%s: heads of %d quaternion channels, at most %d are supported", fn, dq,
                      quan::kAttnMaxDq);
    return QUAN_OK;
}

struct CacheSpans {
    Span keys, values, key_exp, value_exp, table;
};

int check_cache(const char *fn, const quan_cache *c, int32_t dtype, quan::Cache *out, CacheSpans *s)
{
    if (c == nullptr || c->keys == nullptr || c->values == nullptr || c->table == nullptr)
        return report(QUAN_ERR_NULL, "%s: the cache and its keys, values and table must be non-NULL", fn);
    if (int rc = check_format(fn, c->dq, c->format))
        return rc;
    const bool e4m3 = c->format == QUAN_CACHE_E4M3;
    if (e4m3 && (c->key_exp == nullptr || c->value_exp == nullptr))
        return report(QUAN_ERR_NULL, "%s: an 8-bit cache needs key_exp and value_exp", fn);
    if (!e4m3 && c->format != dtype)
        return report(QUAN_ERR_DTYPE, "%s: a cache of format %d with maps of dtype %d", fn, c->format, dtype);
    if (c->pages < 1 || c->page_tokens < 1 || c->heads < 1 || c->sequences < 1 || c->table_pages < 1)
        return report(QUAN_ERR_SHAPE,
                      "%s: sizes of the cache must be >= 1 (pages=%d page_tokens=%d heads=%d sequences=%d table_pages=%d)",
                      fn, c->pages, c->page_tokens, c->heads, c->sequences, c->table_pages);
    if (c->heads > 65535 || c->page_tokens > kMaxImagePixels)
        return report(QUAN_ERR_UNSUPPORTED, "%s: at most 65535 heads and 2^24 tokens of a page", fn);
    // (65535 * 2^24 leaves room for the comparison)
    const int64_t page_rows = int64_t(c->heads) * c->page_tokens;
    if (page_rows > kMaxInt || page_rows * c->pages > kMaxInt || int64_t(c->sequences) * c->table_pages > kMaxInt)
        return report(QUAN_ERR_UNSUPPORTED, "%s: the cache has 2^31 or more rows or entries of its table", fn);
    // (what a work-group adds to a position stays an int)
    if (int64_t(c->table_pages) * c->page_tokens > int64_t(1) << 30)
        return report(QUAN_ERR_UNSUPPORTED, "%s: a sequence has more than 2^30 positions", fn);
    if (misaligned(c->keys, 16) || misaligned(c->values, 16))
        return report(QUAN_ERR_ALIGN, "%s: the cache's keys and values must be 16-byte aligned", fn);
    if (misaligned(c->table, 4))
        return report(QUAN_ERR_ALIGN, "%s: the cache's table must be 4-byte aligned", fn);
    const auto form = static_cast<quan::CacheForm>(c->format);
    const int row = quan::cache_row_bytes(c->dq, form);
    *out = {static_cast<unsigned char *>(c->keys),
            static_cast<unsigned char *>(c->values),
            c->key_exp,
            c->value_exp,
            c->table,
            form,
            c->pages,
            c->page_tokens,
            c->heads,
            c->dq,
            c->sequences,
            c->table_pages,
            row,
            quan::FastDiv(c->page_tokens)};
    const size_t rows = size_t(page_rows) * c->pages;
    s->keys = {"the cache's keys", c->keys, rows * row};
    s->values = {"the cache's values", c->values, rows * row};
    s->key_exp = {"key_exp", e4m3 ? c->key_exp : nullptr, rows};
    s->value_exp = {"value_exp", e4m3 ? c->value_exp : nullptr, rows};
    s->table = {"the cache's table", c->table, size_t(c->sequences) * c->table_pages * 4};
    return QUAN_OK;
}

// Where a map's sequences lie.
int check_sequences(const char *fn, const char *what, const quan_tensor *t, const int32_t *first, int32_t sequences,
                    quan::Sequences *s, Span *span)
{
    const int64_t n = t->shape[0], hw = t->shape[3] * t->shape[4];
    if (sequences < 1)
        return report(QUAN_ERR_SHAPE, "%s: %d sequences", fn, sequences);
    if (first != nullptr ? n != 1 : n != sequences)
        return report(QUAN_ERR_SHAPE, "%s: %s has %lld images, not %d", fn, what, (long long)n,
                      first != nullptr ? 1 : sequences);
    if (n * hw > kMaxInt)
        return report(QUAN_ERR_UNSUPPORTED, "%s: %s has 2^31 or more pixels", fn, what);
    if (misaligned(first, 4))
        return report(QUAN_ERR_ALIGN, "%s: the sequences of %s must be 4-byte aligned", fn, what);
    *s = {first, sequences, int(hw)};
    *span = {"the array of sequences", first, (size_t(sequences) + 1) * 4};
    return QUAN_OK;
}

int check_ints(const char *fn, std::initializer_list<Span> arrays)
{
    for (const Span &a : arrays)
        if (misaligned(a.p, 4))
            return report(QUAN_ERR_ALIGN, "%s: %s must be 4-byte aligned", fn, a.what);
    return QUAN_OK;
}

struct CopySpans {
    CacheSpans cache;
    Span k, v, first, start, kv_len;
};

int check_copy(const char *fn, const quan_tensor *k, const quan_tensor *v, const int32_t *first, const int32_t *start,
               const int32_t *kv_len, const quan_cache *cache, quan::CacheCopy *c, quan::DType *dt, CopySpans *s)
{
    if (k == nullptr || v == nullptr)
        return report(QUAN_ERR_NULL, "%s: k and v must be non-NULL", fn);
    if (int rc = check_dtype(fn, k->dtype))
        return rc;
    if (int rc = check_cache(fn, cache, k->dtype, &c->cache, &s->cache))
        return rc;
    const int64_t want[5] = {-1, 4, int64_t(cache->heads) * cache->dq, -1, -1};
    if (int rc = check_map(fn, "k", k, k->dtype, want, &c->k, &s->k))
        return rc;
    if (int rc = check_map(fn, "v", v, k->dtype, k->shape, &c->v, &s->v))
        return rc;
    if (int rc = check_sequences(fn, "k", k, first, cache->sequences, &c->seq, &s->first))
        return rc;
    if (k->shape[0] * k->shape[3] * k->shape[4] * 2 * cache->heads > kMaxInt)
        return report(QUAN_ERR_UNSUPPORTED, "%s: 2^31 or more rows of tokens and heads", fn);
    s->start = {"start", start, size_t(cache->sequences) * 4};
    s->kv_len = {"kv_len", kv_len, size_t(cache->sequences) * 4};
    if (int rc = check_ints(fn, {s->start, s->kv_len}))
        return rc;
    c->start = start;
    c->kv_len = kv_len;
    for_heads(&c->k, cache->dq);
    for_heads(&c->v, cache->dq);
    if (quan::cache_copy_groups(*c) > kMaxGroups)
        return report(QUAN_ERR_UNSUPPORTED, "%s: too many work-groups", fn);
    *dt = to_dt(k->dtype);
    return QUAN_OK;
}

struct AttentionCall {
    quan::CacheAttention a;
    quan::DType dt;
};
hipError_t run_attention(void *args, void *, void *extra, hipStream_t s)
{
    const AttentionCall &c = *static_cast<AttentionCall *>(args);
    return quan::cache_attention_run(c.a, c.dt, extra, s);
}

struct PackedSpans {
    Span q, k, v, q_first, k_first;
};

int check_packed(const char *fn, const quan_tensor *q, const quan_tensor *k, const quan_tensor *v, const int32_t *q_first,
                 const int32_t *k_first, int32_t sequences, int32_t causal, float scale, int32_t heads,
                 quan::PackedCall *c, quan::DType *dt, PackedSpans *s)
{
    if (q == nullptr || k == nullptr || v == nullptr)
        return report(QUAN_ERR_NULL, "%s: q, k and v must be non-NULL", fn);
    const int32_t dtype = q->dtype;
    if (int rc = check_dtype(fn, dtype))
        return rc;
    const int64_t q_want[5] = {-1, 4, -1, -1, -1};
    if (int rc = check_map(fn, "q", q, dtype, q_want, &c->q, &s->q))
        return rc;
    const int64_t k_want[5] = {q->shape[0], 4, -1, -1, -1};
    if (int rc = check_map(fn, "k", k, dtype, k_want, &c->k, &s->k))
        return rc;
    if (int rc = check_map(fn, "v", v, dtype, k->shape, &c->v, &s->v))
        return rc;
    const int64_t channels = q->shape[2], ckv = k->shape[2];
    if (heads < 1 || channels % heads != 0)
        return report(QUAN_ERR_SHAPE, "%s: %d heads do not divide %lld channels", fn, heads, (long long)channels);
    const int64_t dq = channels / heads;
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
    if (causal != 0 && causal != 1)
        return report(QUAN_ERR_SHAPE, "%s: causal must be 0 or 1 (got %d)", fn, causal);
    if (q_first == nullptr && k_first != nullptr)
        return report(QUAN_ERR_NULL, "%s: k_first without q_first", fn);
    if (q_first != nullptr && k_first == nullptr) {
        if (q->shape[3] * q->shape[4] != k->shape[3] * k->shape[4])
            return report(QUAN_ERR_SHAPE, "%s: without k_first, q and k must have as many pixels", fn);
        k_first = q_first;
    }
    if (int rc = check_sequences(fn, "q", q, q_first, sequences, &c->qs, &s->q_first))
        return rc;
    if (int rc = check_sequences(fn, "k", k, k_first, sequences, &c->ks, &s->k_first))
        return rc;
    c->images = int(q->shape[0]);
    c->heads = heads;
    c->kv_heads = int(ckv / dq);
    c->dq = int(dq);
    c->causal = causal == 1;
    c->scale = scale;
    // (work-groups of 512 lanes, in whole turns of the XCDs)
    constexpr int64_t kMost = kMaxLanes / 512 - 128;
    if (quan::packed_blocks(c->qs) > kMost / heads || quan::packed_blocks(c->ks) > kMost / c->kv_heads ||
        c->q_tokens() > kMaxInt * 4 / heads)
        return report(QUAN_ERR_UNSUPPORTED, "%s: too many work-groups", fn);
    for (quan::AttnMap *m : {&c->q, &c->k, &c->v})
        for_heads(m, c->dq);
    *dt = to_dt(dtype);
    return QUAN_OK;
}

// What the forward pass keeps for the backward one.
int check_saved(const char *fn, const quan_tensor *q, const void *rest, const float *stats, int32_t heads,
                const quan::PackedCall &c, Span *rest_span, Span *stats_span)
{
    if (rest != nullptr && q->dtype != QUAN_BF16)
        return report(QUAN_ERR_DTYPE, "%s: rest is for bf16 maps", fn);
    if (misaligned(rest, 16))
        return report(QUAN_ERR_ALIGN, "%s: rest must be 16-byte aligned", fn);
    if (misaligned(stats, 4))
        return report(QUAN_ERR_ALIGN, "%s: stats must be 4-byte aligned", fn);
    *rest_span = {"rest", rest, size_t(c.q_tokens()) * 4 * q->shape[2] * 2};
    *stats_span = {"stats", stats, size_t(heads) * c.q_tokens() * 8};
    return QUAN_OK;
}

struct PackedForward {
    quan::PackedCall c;
    quan::DType dt;
    quan::AttnMap out;
    void *rest;
    float *stats;
};
hipError_t run_packed_forward(void *args, void *work, void *extra, hipStream_t s)
{
    const PackedForward &p = *static_cast<PackedForward *>(args);
    return quan::packed_forward_run(p.c, p.dt, p.out, p.rest, p.stats, work, extra, s);
}

struct PackedBackward {
    quan::PackedCall c;
    quan::DType dt;
    quan::PackedGradients g;
};
hipError_t run_packed_backward(void *args, void *work, void *, hipStream_t s)
{
    const PackedBackward &p = *static_cast<PackedBackward *>(args);
    return quan::packed_backward_run(p.c, p.dt, p.g, work, s);
}

}  // namespace

extern "C" {

QUAN_API int64_t quan_cache_row_bytes(int32_t dq, int32_t format)
{
    quan::clear_error();
    if (int rc = check_format("cache_row_bytes", dq, format))
        return rc;
    return quan::cache_row_bytes(dq, static_cast<quan::CacheForm>(format));
}

QUAN_API int quan_cache_write(const quan_tensor *k, const quan_tensor *v, const int32_t *first, const int32_t *start,
                              const int32_t *kv_len, const quan_cache *cache, void *stream)
{
    const char *fn = "cache_write";
    quan::clear_error();
    quan::CacheCopy c{};
    quan::DType dt;
    CopySpans s;
    if (int rc = check_copy(fn, k, v, first, start, kv_len, cache, &c, &dt, &s))
        return rc;
    const CacheSpans &o = s.cache;
    for (const Span &out : {o.keys, o.values, o.key_exp, o.value_exp})
        if (int rc = check_alias(fn, out, {s.k, s.v, s.first, s.start, s.kv_len, o.table}))
            return rc;
    if (int rc = check_alias(fn, o.keys, {o.values, o.key_exp, o.value_exp}))
        return rc;
    if (int rc = check_alias(fn, o.values, {o.key_exp, o.value_exp}))
        return rc;
    if (int rc = check_alias(fn, o.key_exp, {o.value_exp}))
        return rc;
    return launched(quan::cache_write_run(c, dt, static_cast<hipStream_t>(stream)), fn);
}

QUAN_API int quan_cache_read(const quan_cache *cache, const int32_t *first, const int32_t *start, const int32_t *kv_len,
                             quan_tensor *k, quan_tensor *v, void *stream)
{
    const char *fn = "cache_read";
    quan::clear_error();
    quan::CacheCopy c{};
    quan::DType dt;
    CopySpans s;
    if (int rc = check_copy(fn, k, v, first, start, kv_len, cache, &c, &dt, &s))
        return rc;
    const CacheSpans &o = s.cache;
    for (const Span &out : {s.k, s.v})
        if (int rc = check_alias(fn, out, {o.keys, o.values, o.key_exp, o.value_exp, o.table, s.first, s.start, s.kv_len}))
            return rc;
    if (int rc = check_alias(fn, s.k, {s.v}))
        return rc;
    return launched(quan::cache_read_run(c, dt, static_cast<hipStream_t>(stream)), fn);
}

QUAN_API int quan_cache_attention(const quan_tensor *q, const quan_cache *cache, const quan_relpos *relpos,
                                  int32_t width, const int32_t *kv_len, const int32_t *pos, float scale, int32_t heads,
                                  quan_tensor *out, void *stream)
{
    const char *fn = "cache_attention";
    quan::clear_error();
    AttentionCall c{};
    CacheSpans s;
    if (q == nullptr)
        return report(QUAN_ERR_NULL, "%s: q must be non-NULL", fn);
    if (int rc = check_dtype(fn, q->dtype))
        return rc;
    if (int rc = check_cache(fn, cache, q->dtype, &c.a.cache, &s))
        return rc;
    if (heads < 1 || heads % cache->heads != 0)
        return report(QUAN_ERR_SHAPE, "%s: %d heads are no multiple of the cache's %d", fn, heads, cache->heads);
    if (heads > 65535)
        return report(QUAN_ERR_UNSUPPORTED, "%s: more than 65535 heads", fn);
    const int64_t want[5] = {cache->sequences, 4, int64_t(heads) * cache->dq, 1, 1};
    Span q_span, out_span;
    if (int rc = check_map(fn, "q", q, q->dtype, want, &c.a.q, &q_span))
        return rc;
    if (int rc = check_map(fn, "out", out, q->dtype, want, &c.a.out, &out_span))
        return rc;
    if (!std::isfinite(scale))
        return report(QUAN_ERR_SHAPE, "%s: scale must be finite", fn);
    if (int64_t(cache->sequences) * heads > kMaxLanes / 512)  // (work-groups of 512 lanes)
        return report(QUAN_ERR_UNSUPPORTED, "%s: too many work-groups", fn);
    const Span len_span{"kv_len", kv_len, size_t(cache->sequences) * 4};
    const Span pos_span{"pos", pos, size_t(cache->sequences) * 8};
    if (int rc = check_ints(fn, {len_span, pos_span}))
        return rc;
    Span table{"relpos", nullptr, 0}, by = table, bx = table;
    c.a.bias = {};
    c.a.width = 1;
    if (relpos != nullptr) {
        if (int rc = check_relpos(fn, relpos, heads, &c.a.bias, &table, &by, &bx))
            return rc;
        if (width < 1)
            return report(QUAN_ERR_SHAPE, "%s: width must be >= 1 with a bias (got %d)", fn, width);
        c.a.width = width;
    }
    if (int rc = check_alias(fn, out_span, {q_span, s.keys, s.values, s.key_exp, s.value_exp, s.table, len_span, pos_span,
                                            table, by, bx}))
        return rc;
    for_heads(&c.a.q, cache->dq);
    for_heads(&c.a.out, cache->dq);
    c.a.kv_len = kv_len;
    c.a.pos = pos;
    c.a.n = cache->sequences;
    c.a.heads = heads;
    c.a.by_width = quan::FastDiv(c.a.width);
    c.a.scale = scale;
    c.dt = to_dt(q->dtype);
    const size_t extra = quan::cache_attention_extra_bytes(c.a, c.dt);
    if (extra == 0)
        return launched(run_attention(&c, nullptr, nullptr, static_cast<hipStream_t>(stream)), fn);
    return quan::run_on_stream(stream, 0, extra, run_attention, &c, fn);
}

QUAN_API int quan_packed_attention_forward(const quan_tensor *q, const quan_tensor *k, const quan_tensor *v,
                                           const int32_t *q_first, const int32_t *k_first, int32_t sequences,
                                           int32_t causal, float scale, int32_t heads, quan_tensor *out, void *rest,
                                           float *stats, void *stream)
{
    const char *fn = "packed_attention_forward";
    quan::clear_error();
    PackedForward p{};
    PackedSpans s;
    if (int rc = check_packed(fn, q, k, v, q_first, k_first, sequences, causal, scale, heads, &p.c, &p.dt, &s))
        return rc;
    Span out_span;
    if (int rc = check_map(fn, "out", out, q->dtype, q->shape, &p.out, &out_span))
        return rc;
    Span rest_span, stats_span;
    if (int rc = check_saved(fn, q, rest, stats, heads, p.c, &rest_span, &stats_span))
        return rc;
    for (const Span &o : {out_span, rest_span, stats_span})
        if (int rc = check_alias(fn, o, {s.q, s.k, s.v, s.q_first, s.k_first}))
            return rc;
    if (int rc = check_alias(fn, out_span, {rest_span, stats_span}))
        return rc;
    if (int rc = check_alias(fn, rest_span, {stats_span}))
        return rc;
    for_heads(&p.out, p.c.dq);
    p.rest = rest;
    p.stats = stats;
    const size_t bytes = quan::packed_forward_work_bytes(p.c, p.dt), extra = quan::packed_forward_extra_bytes(p.c, p.dt);
    if (bytes == 0 && extra == 0)
        return launched(run_packed_forward(&p, nullptr, nullptr, static_cast<hipStream_t>(stream)), fn);
    return quan::run_on_stream(stream, bytes, extra, run_packed_forward, &p, fn);
}

QUAN_API int quan_packed_attention_backward(const quan_tensor *q, const quan_tensor *k, const quan_tensor *v,
                                            const int32_t *q_first, const int32_t *k_first, int32_t sequences,
                                            int32_t causal, float scale, int32_t heads, const quan_tensor *out,
                                            const void *rest, const float *stats, const quan_tensor *dout, quan_tensor *dq,
                                            quan_tensor *dk, quan_tensor *dv, void *stream)
{
    const char *fn = "packed_attention_backward";
    quan::clear_error();
    PackedBackward p{};
    PackedSpans s;
    if (int rc = check_packed(fn, q, k, v, q_first, k_first, sequences, causal, scale, heads, &p.c, &p.dt, &s))
        return rc;
    Span out_span, dout_span, dq_span, dk_span, dv_span;
    if (int rc = check_map(fn, "out", out, q->dtype, q->shape, &p.g.out, &out_span))
        return rc;
    if (int rc = check_map(fn, "dout", dout, q->dtype, q->shape, &p.g.dout, &dout_span))
        return rc;
    if (int rc = check_map(fn, "dq", dq, q->dtype, q->shape, &p.g.dq, &dq_span))
        return rc;
    if (int rc = check_map(fn, "dk", dk, q->dtype, k->shape, &p.g.dk, &dk_span))
        return rc;
    if (int rc = check_map(fn, "dv", dv, q->dtype, k->shape, &p.g.dv, &dv_span))
        return rc;
    if (stats == nullptr)
        return report(QUAN_ERR_NULL, "%s: stats must be non-NULL", fn);
    Span rest_span, stats_span;
    if (int rc = check_saved(fn, q, rest, stats, heads, p.c, &rest_span, &stats_span))
        return rc;
    for (const Span &o : {dq_span, dk_span, dv_span})
        if (int rc = check_alias(fn, o, {s.q, s.k, s.v, s.q_first, s.k_first, out_span, rest_span, stats_span, dout_span}))
            return rc;
    if (int rc = check_alias(fn, dq_span, {dk_span, dv_span}))
        return rc;
    if (int rc = check_alias(fn, dk_span, {dv_span}))
        return rc;
    for (quan::AttnMap *m : {&p.g.out, &p.g.dout, &p.g.dq, &p.g.dk, &p.g.dv})
        for_heads(m, p.c.dq);
    p.g.rest = rest;
    p.g.stats = stats;
    return quan::run_on_stream(stream, quan::packed_backward_work_bytes(p.c, p.dt, p.g), 0, run_packed_backward, &p, fn);
}

}  // extern "C"
