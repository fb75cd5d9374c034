"""Attention of one new token per sequence over a paged cache, on the GPU."""
import numpy as np
import pytest
import torch

import sequence_reference as ref
from parity import say
from paper_2509_05512_amd import quan
from test_gpu_cache import BF, DEV, E4M3, F32, FORMS, ints, make_table, rand_map

pytestmark = pytest.mark.gpu


def fill(seed, lens, page, heads, dq, dtype, form, spare_nan=True):
    """A cache of sequences of `lens` tokens; slots that hold none are NaN."""
    rng = np.random.default_rng(seed)
    table, pages = make_table(rng, lens, page)
    cache = quan.empty_cache(pages, page, heads, dq, table, form)
    for t in (cache.keys, cache.values):
        t.view(torch.uint8).fill_(0x7f if form == E4M3 else 0xff)
    for t in (cache.key_exp, cache.value_exp):
        if t is not None:
            t.fill_(255)
    tokens = max(1, sum(lens))
    k, v = (rand_map(seed + s, 1, heads * dq, 1, tokens, dtype) for s in (1, 2))
    quan.quan_cache_write(cache, k, v, first=ints(ref.starts(lens).tolist()))
    return cache


def values_of(cache):
    """Per sequence and position the fp64 rows [heads, d] that the cache holds,
    None where there is no page: for keys and for values."""
    out = []
    table, d = cache.table.cpu().numpy(), 4 * cache.dq
    for t, e in ((cache.keys, cache.key_exp), (cache.values, cache.value_exp)):
        x = t.float().cpu().numpy().astype(np.float64)[..., :d]
        if e is not None:
            x = x * 2.0 ** (e.cpu().numpy().astype(np.float64) - 127.0)[..., None]
        seqs = []
        for row in table:
            at = []
            for p in row:
                at += [x[p, :, s] for s in range(cache.page_tokens)] if 0 <= p < len(x) else [None] * cache.page_tokens
            seqs.append(at)
        out.append(seqs)
    return out


def run(cache, q, lens, heads, relpos=None, pos=None, width=None, scale=None, what="", **kw):
    out = quan.quan_cache_attention(q, cache, None if lens is None else ints(lens), heads, relpos=relpos,
                                    pos=None if pos is None else ints(pos), width=width, scale=scale, **kw)
    keys, values = values_of(cache)
    n, full = q.shape[0], cache.table.shape[1] * cache.page_tokens
    rows = ref.rows_of(q.float().cpu().numpy().astype(np.float64), heads)
    named = {} if relpos is None else dict(zip(("table", "by", "bx"), (None if t is None else t.cpu().numpy().astype(
        np.float64 if t.dtype == F32 else np.int64) for t in relpos)))
    if relpos is not None and named["table"].ndim == 2:
        named["table"] = named["table"][:, None, :]
    want, err, size = ref.cache_attention(rows, keys, values, [full] * n if lens is None else lens, heads, pos=pos,
                                          width=width or 1, scale=scale, **named)
    got = ref.rows_of(out.float().cpu().numpy().astype(np.float64), heads)
    ref.check(got, want, (err, ref.F32 * max(size, 1e-30)), q.dtype == BF, what)
    return out


@pytest.mark.parametrize("dtype,form", FORMS, ids=["bf16-e4m3", "fp32-e4m3", "bf16", "fp32"])
@pytest.mark.parametrize("dq,heads,kv_heads,page", [
    (16, 8, 2, 16), (16, 4, 4, 64), (8, 3, 3, 7), (32, 4, 1, 64), (5, 6, 2, 1), (12, 40, 2, 5), (1, 2, 1, 3), (24, 2, 2, 33)])
def test_attention(dtype, form, dq, heads, kv_heads, page):
    say(f"cache attention {dtype} {form} dq {dq} heads {heads}/{kv_heads} page {page}")
    lens = [0, 1, 2, 15, 16, 17, 63, 64, 65, 130, 300, 777]
    cache = fill(dq, lens, page, kv_heads, dq, dtype, form)
    q = rand_map(9, len(lens), heads * dq, 1, 1, dtype)
    out = run(cache, q, lens, heads, what="out")
    assert not bool(out[0].any())


@pytest.mark.parametrize("dtype,form", FORMS, ids=["bf16-e4m3", "fp32-e4m3", "bf16", "fp32"])
@pytest.mark.parametrize("heads,kv_heads,ny,nx,ry,rx,width", [
    (4, 2, 5, 7, 2, 3, 9), (3, 3, 1, 16, 0, 64, 5000), (8, 1, 31, 31, 15, 15, 20), (2, 2, 64, 96, 40, 60, 11), (33, 1, 1, 1, 0, 0, 1)])
def test_bias(dtype, form, heads, kv_heads, ny, nx, ry, rx, width):
    say(f"cache attention bias {dtype} {form} heads {heads}/{kv_heads} {ny} x {nx}")
    lens, dq = [0, 1, 100, 1000, 37], 8
    cache = fill(5, lens, 16, kv_heads, dq, dtype, form)
    g = torch.Generator().manual_seed(2)
    table = torch.randn((heads, ny, nx), generator=g).to(DEV)
    table[0, ny // 2] = -3.4028234663852886e38
    by = quan.quan_relpos_buckets(ry, ny, DEV) if ny > 1 else None
    bx = quan.quan_relpos_buckets(rx, nx, DEV) if nx > 1 else None
    pos = [[0, 0], [3, 4], [50, -7], [-2147483648, 2147483647], [max(0, 36 // width), 36 % width]]
    q = rand_map(3, 5, heads * dq, 1, 1, dtype)
    run(cache, q, lens, heads, (table, by, bx), pos, width, what="out")
    run(cache, q, lens, heads, (table, by, bx), None, width, scale=0.3, what="out without places")


def test_bias_that_leaves_nothing():
    """-infinity in every bucket: 0; in some: the others alone."""
    say("cache attention, biases of -infinity")
    lens, heads, dq = [70, 70, 70], 2, 16
    for dtype, form in FORMS:
        cache = fill(6, lens, 8, heads, dq, dtype, form)
        table = torch.zeros((heads, 1, 3), device=DEV)
        table[0] = -torch.inf
        table[1, 0, 0] = -torch.inf
        bx = quan.quan_relpos_buckets(1, 3, DEV)
        q = rand_map(1, 3, heads * dq, 1, 1, dtype)
        out = run(cache, q, lens, heads, (table, None, bx), [[0, 0], [0, 30], [0, 500]], 100, what="out")
        assert not bool(out[:, :, :dq].any()) and not bool(out[2].any())
        assert bool(out[:2, :, dq:].any())


def test_lengths_and_bad_pages():
    """Lengths beyond the table or below 0; pages that are none in the middle; one
    page for several sequences."""
    say("cache attention, bad pages")
    for dtype, form in FORMS:
        lens, heads, dq, page = [40, 40, 40, 40], 2, 16, 8
        cache = fill(8, lens, page, heads, dq, dtype, form)
        table = cache.table.clone()
        table[0, 1], table[0, 3], table[1, 0], table[2, 4] = -1, 2147483647, cache.keys.shape[0], -2147483648
        table[3] = table[1]
        table[3, 0] = table[2, 0]
        cache = cache._replace(table=table)
        q = rand_map(4, 4, heads * dq, 1, 1, dtype)
        run(cache, q, [40, 40, 33, 2147483647], heads, what="bad pages")
        run(cache, q, [-5, -2147483648, 8, 39], heads, what="lengths")
        run(cache, q, None, heads, what="no lengths")
        cache = cache._replace(table=torch.full_like(table, -1))
        assert not bool(run(cache, q, lens, heads, what="no pages").any())


@pytest.mark.parametrize("dtype,form", FORMS, ids=["bf16-e4m3", "fp32-e4m3", "bf16", "fp32"])
def test_long_sequences(dtype, form):
    """Sequences that are dealt out to work-groups, beside short ones."""
    say(f"cache attention, long sequences {dtype} {form}")
    lens, dq = [9000, 3, 0, 4097, 64], 16
    cache = fill(11, lens, 64, 1, dq, dtype, form)
    q = rand_map(5, 5, 2 * dq, 1, 1, dtype)
    run(cache, q, lens, 2, what="out")
    one = cache._replace(table=cache.table[:1].contiguous())
    run(one, q[:1], lens[:1], 2, what="one sequence")


@pytest.mark.parametrize("count", [1, 64, 65, 257, 1500])
def test_many_sequences(count):
    say(f"cache attention of {count} sequences")
    rng = np.random.default_rng(count)
    lens = rng.integers(0, 90, count).tolist()
    cache = fill(count, lens, 16, 2, 8, BF, E4M3)
    run(cache, rand_map(1, count, 4 * 8, 1, 1, BF), lens, 4, what="out")


def test_scores_of_any_size():
    """Scores of hundreds, where all but one key vanish; NaN and infinities in what
    is masked or beyond the length change nothing, in a key they reach its sequence
    alone."""
    say("cache attention, large scores and NaN")
    for dtype, form in FORMS:
        lens, heads, dq = [100, 100], 1, 16
        cache = fill(12, lens, 16, heads, dq, dtype, form)
        q = rand_map(2, 2, dq, 1, 1, dtype)
        run(cache, q, lens, heads, scale=20.0, what="large scores")
        clean = run(cache, q, [90, 90], heads, what="shorter")
        page, slot = int(cache.table[0, 90 // 16]), 90 % 16
        for t in (cache.keys, cache.values):
            t[page, :, slot:].view(torch.uint8).fill_(0x7f if form == E4M3 else 0xff)
        again = quan.quan_cache_attention(q, cache, ints([90, 90]), heads)
        assert torch.equal(clean, again)
        got = quan.quan_cache_attention(q, cache, ints([91, 91]), heads)
        assert bool(torch.isnan(got[0]).all()) and not bool(torch.isnan(got[1]).any())


def test_unaligned_queries_and_slices():
    say("cache attention, slices")
    lens, heads, dq = [50, 20, 7], 4, 8
    for dtype in (BF, F32):
        cache = fill(13, lens, 16, 2, dq, dtype, E4M3)
        wide = rand_map(3, 3, 3 + 2 * heads * dq, 1, 1, dtype)
        run(cache, wide[:, :, 3:3 + heads * dq], lens, heads, out=wide[:, :, 3 + heads * dq:], what="out")


def test_read_back_attention_is_the_same():
    """The cache's attention against quan_attention_forward over what is read
    back: a bf16 step of the largest value apart (8-bit values are bf16 numbers)."""
    say("cache attention against the maps' attention")
    lens, heads, dq, width = [200, 1, 77, 0], 4, 16, 20
    cache = fill(14, lens, 16, 2, dq, BF, E4M3)
    room = cache.table.shape[1] * 16
    k, v = (torch.zeros((4, 1, room, 4, 2 * dq), dtype=BF, device=DEV).permute(0, 3, 4, 1, 2) for _ in range(2))
    quan.quan_cache_read(cache, k, v, kv_len=ints(lens))
    q = rand_map(3, 4, heads * dq, 1, 1, BF)
    a = quan.quan_cache_attention(q, cache, ints(lens), heads)
    b = quan.quan_attention_forward(q, k, v, heads, kv_len=ints(lens))
    assert float((a.float() - b.float()).abs().max()) <= 2.0 ** -7 * float(b.float().abs().max())


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("dq,heads,kv_heads", [(16, 4, 2), (8, 3, 3), (32, 16, 1), (5, 2, 1)])
@pytest.mark.parametrize("lens", [[100, 1, 65], [5000, 70, 0]], ids=["short", "long"])
def test_infinite_values(dtype, dq, heads, kv_heads, lens):
    """An infinity in a value is the result's, both signs in one place are NaN, as is a
    NaN; the other reals keep their bounds."""
    say(f"cache attention, infinite values {dtype} dq {dq} heads {heads}/{kv_heads} {lens}")
    cache = fill(21, lens, 16, kv_heads, dq, dtype, dtype)
    q = rand_map(3, len(lens), heads * dq, 1, 1, dtype)
    odd = [(0, 3, np.inf), (1, 7, -np.inf), (2, 9, np.inf), (2, lens[0] - 1, -np.inf), (3, 40, np.nan), (4 * dq - 1, 64, np.inf),
           (4 * dq - 2, 5, np.inf), (4 * dq - 2, 50, np.nan), (4 * dq - 2, 51, np.inf)]
    zeros = cache._replace(values=cache.values.clone())
    extra = np.zeros((len(lens), heads, 4 * dq))
    for real, token, value in odd:
        page = int(cache.table[0, token // 16])
        cache.values[page, 0, token % 16, real] = value
        zeros.values[page, 0, token % 16, real] = 0.0
        with np.errstate(invalid="ignore"):
            extra[0, :heads // kv_heads, real] += value
    got = ref.rows_of(quan.quan_cache_attention(q, cache, ints(lens), heads).float().cpu().numpy().astype(np.float64), heads)
    keys, values = values_of(zeros)
    rows = ref.rows_of(q.float().cpu().numpy().astype(np.float64), heads)
    want, err, size = ref.cache_attention(rows, keys, values, lens, heads)
    hit = ~np.isfinite(extra)
    assert np.array_equal(got[hit], extra[hit], equal_nan=True)
    ref.check(np.where(hit, want, got), want, (err, ref.F32 * max(size, 1e-30)), dtype == BF, "the others")


@pytest.mark.parametrize("dtype,form", FORMS, ids=["bf16-e4m3", "fp32-e4m3", "bf16", "fp32"])
@pytest.mark.parametrize("count", [65, 129, 200])
def test_many_sequences_dealt_out(dtype, form, count):
    """Sequences in several sets of 64, empty ones among them, with long ones behind the
    first set that work-groups share."""
    say(f"cache attention of {count} sequences, dealt out {dtype} {form}")
    lens = np.random.default_rng(count).integers(0, 60, count).tolist()
    lens[3], lens[64], lens[count - 1] = 0, 3000, 5001
    lens[count // 2 + 20] = 1
    cache = fill(count, lens, 64, 1, 8, dtype, form)
    run(cache, rand_map(1, count, 8, 1, 1, dtype), lens, 1, what="out")


@pytest.mark.parametrize("dtype,form", FORMS, ids=["bf16-e4m3", "fp32-e4m3", "bf16", "fp32"])
@pytest.mark.parametrize("dq,heads,kv_heads", [(32, 16, 1), (24, 32, 2), (20, 33, 1)])
def test_many_wide_heads_of_a_key(dtype, form, dq, heads, kv_heads):
    """16 query heads and more than 64 reals to a head of keys, whose results take more
    than 64 KiB where the waves' are joined."""
    say(f"cache attention {dtype} {form} dq {dq} heads {heads}/{kv_heads}")
    lens = [0, 1, 70, 700]
    cache = fill(31, lens, 16, kv_heads, dq, dtype, form)
    q = rand_map(4, len(lens), heads * dq, 1, 1, dtype)
    run(cache, q, lens, heads, what="out")
    g = torch.Generator().manual_seed(6)
    table = torch.randn((heads, 1, 9), generator=g).to(DEV)
    run(cache, q, lens, heads, (table, None, quan.quan_relpos_buckets(30, 9, DEV)), [[0, 5]] * 4, 50, what="out with a bias")
