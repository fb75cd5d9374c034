"""The operators on sequences of pixels together, as a model that reads and writes
them one after another calls them: whole prompts, prompts continued from a cache,
single pixels; captured graphs, streams, threads."""
import threading

import numpy as np
import pytest
import torch

import sequence_reference as ref
from parity import say
from paper_2509_05512_amd import quan
from paper_2509_05512_amd.attention_block import AttentionBlock
from test_gpu_cache import BF, DEV, E4M3, F32, ints, make_table, rand_map
from test_gpu_packed_attention import compare, step

pytestmark = pytest.mark.gpu


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


@pytest.mark.parametrize("dtype,form", [(BF, BF), (F32, F32), (BF, E4M3), (F32, E4M3)],
                         ids=["bf16", "fp32", "bf16-e4m3", "fp32-e4m3"])
def test_a_sequence_in_pieces(dtype, form):
    """Prompts, their continuation from the cache and single tokens against whole
    sequences over the keys and values that the cache holds.  Bounds: those of the
    packed attention; a single token's are within them."""
    say(f"sequences in pieces {dtype} {form}")
    heads, kv_heads, dq, lens = 4, 2, 16, [70, 0, 133, 9]
    pieces = [[40, 0, 64, 1], [20, 0, 68, 7], [10, 0, 1, 1]]  # the last one token by token
    n = len(lens)
    table, pages = make_table(np.random.default_rng(1), lens, 16)
    cache = quan.empty_cache(pages, 16, kv_heads, dq, table, form)
    q, kv = rand_map(1, 1, heads * dq, 1, sum(lens), dtype), rand_map(2, 1, 2 * kv_heads * dq, 1, sum(lens), dtype)
    k, v = kv[:, :, :kv_heads * dq], kv[:, :, kv_heads * dq:]
    at = ref.starts(lens)
    outs = torch.zeros_like(q)

    def take(t, where):
        return quan.to_device_layout(t[..., torch.tensor(where, dtype=torch.long, device=DEV)])
    past = [0] * n
    for p, counts in enumerate(pieces):
        for counts in ([counts] if p < 2 else [[int(past[i] + s < lens[i]) for i in range(n)] for s in range(10)]):
            where = [at[i] + past[i] + j for i in range(n) for j in range(counts[i])]
            if not where:
                continue
            first = ints(ref.starts(counts).tolist())
            quan.quan_cache_write(cache, take(k, where), take(v, where), ints(past), first=first)
            upto = [a + b for a, b in zip(past, counts)]
            if p < 2:
                back = torch.zeros((1, 1, sum(upto), 4, 2 * kv_heads * dq), dtype=dtype, device=DEV).permute(0, 3, 4, 1, 2)
                k_first = ints(ref.starts(upto).tolist())
                keys, values = quan.quan_cache_read(cache, back[:, :, :kv_heads * dq], back[:, :, kv_heads * dq:], first=k_first)
                got = quan.quan_packed_attention_forward(take(q, where), keys, values, first, heads, k_first=k_first)
            else:
                one = torch.zeros((n, 1, 1, 4, heads * dq), dtype=dtype, device=DEV).permute(0, 3, 4, 1, 2)
                for i in range(n):
                    if counts[i]:
                        one[i, ..., 0] = q[0, ..., at[i] + past[i]]
                got = quan.quan_cache_attention(one, cache, ints(upto), heads)
                assert not bool(got[1].any())
                got = torch.cat([got[i:i + 1] for i in range(n) if counts[i]], 4)
            for g, w in enumerate(where):
                outs[..., w] = got[..., g]
            past = upto
    assert past == lens
    whole = torch.zeros_like(kv)
    keys, values = quan.quan_cache_read(cache, whole[:, :, :kv_heads * dq], whole[:, :, kv_heads * dq:],
                                        first=ints(at.tolist()))
    rows = [ref.rows_of(f64(t), h) for t, h in ((q, heads), (keys, kv_heads), (values, kv_heads))]
    want, err = ref.packed(*rows, lens, lens)
    ref.check(ref.rows_of(f64(outs), heads), want["out"], err["out"], dtype == BF, "pieces")


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
def test_causal_block(dtype):
    """A causal block's whole map against its pixels in pieces from a cache in the
    map's own type: their sums are split and rounded elsewhere, and two convolutions
    and two norms pass it on (bf16: 2^-8 of the largest value at each of four
    roundings; fp32: 1e-5)."""
    say(f"causal block {dtype}")
    n, c, heads, h, w = 3, 32, 4, 6, 7
    block = AttentionBlock(c, heads, kv_heads=2, dtype=dtype, causal=True, seed=3)
    x, hh = rand_map(1, n, c, h, w, dtype), rand_map(2, n, c, h, w, dtype)
    whole, whole_h = block.forward(x, hh)
    cache = block.pages(n, h, w, page_tokens=5, dtype=dtype)
    tol = (4 * 2.0 ** -8 if dtype == BF else 1e-5)

    def near(got, want):
        assert float((got.float() - want.float()).abs().max()) <= tol * float(want.float().abs().max())
    for row, rows in ((0, 1), (1, 3), (4, 1)):
        z = slice(row, row + rows)
        out, out_h = block.extend(cache, *(quan.to_device_layout(t[:, :, :, z]) for t in (x, hh)), [row * w] * n)
        near(out, whole[:, :, :, z])
        near(out_h, whole_h[:, :, :, z])
    for j in range(w):  # the last row pixel by pixel
        px, ph = (quan.to_device_layout(t[:, :, :, 5:6, j:j + 1]) for t in (x, hh))
        _, k, v = block._parts(block._conv("qkv", ph))
        quan.quan_cache_write(cache, k, v, torch.full((n,), 5 * w + j, dtype=torch.int32, device=DEV))
        out, out_h = block.query(cache, px, ph, None, kv_len=torch.full((n,), 5 * w + j + 1, dtype=torch.int32, device=DEV))
        near(out, whole[:, :, :, 5:6, j:j + 1])
        near(out_h, whole_h[:, :, :, 5:6, j:j + 1])


def test_causal_block_gradients():
    """In fp32, along random directions of its inputs and kernels: central
    differences with h = 2^-7 are off by the third derivative's h^2 / 6 (1e-5 for
    terms of order 1) and by the forward's rounding, 2^-24 of sums of a thousand terms
    over h: 1e-3 of the sums of absolute products leaves room for both."""
    say("causal block, differences")
    c, heads = 16, 2
    block = AttentionBlock(c, heads, kv_heads=1, dtype=F32, causal=True, seed=5)
    x, hh, dout, dh_out = (rand_map(s, 2, c, 3, 5, F32) for s in range(4))
    out, h_out, saved = block.forward(x, hh, save=True)
    dx, dh, _, grads = block.backward(saved, dout, dh_out)
    assert "table" not in grads
    step_ = 2.0 ** -7

    def value(x, hh):
        o, h = block.forward(x, hh)
        return float((o.double() * dout.double()).sum() + (h.double() * dh_out.double()).sum())

    def check(grad, way, up, down, what):
        slope = (up - down) / (2 * step_)
        p = grad.double() * way.double()
        assert abs(slope - float(p.sum())) <= 1e-3 * float(p.abs().sum()), (what, slope, float(p.sum()))
    way = rand_map(8, 2, c, 3, 5, F32)
    check(dh, way, value(x, hh + step_ * way), value(x, hh - step_ * way), "h")
    check(dx, way, value(x + step_ * way, hh), value(x - step_ * way, hh), "x")
    for name in ("qkv", "proj"):
        held = block.params[name].clone()
        way = torch.randn(held.shape, generator=torch.Generator().manual_seed(9)).to(DEV) * 0.1
        vals = []
        for s in (1, -1):
            block.params[name] = held + s * step_ * way
            block.load()
            vals.append(value(x, hh))
        block.params[name] = held
        block.load()
        check(grads[name], way, *vals, name)


def test_block_with_pages():
    """A block with a bias asked single pixels from a cache of pages, in the maps'
    own type: as from the cache of maps, up to bf16's last place of the largest."""
    say("block with pages")
    n, c, heads, side = 3, 32, 4, 8
    block = AttentionBlock(c, heads, radius=side - 1, buckets=9, seed=4)
    x, h = rand_map(1, n, c, side, side, BF), rand_map(2, n, c, side, side, BF)
    maps, pages = block.cache(n, side, side), block.pages(n, side, side, page_tokens=6, dtype=BF)
    for row in (0, 3):
        for cache in (maps, pages):
            block.write(cache, quan.to_device_layout(h[:, :, :, row:row + 3]), row)
    pos = ints([[2, 3], [5, 0], [7, 7]])
    lens = ints([6 * side, 20, 1])
    px, ph = (quan.to_device_layout(t[..., 2:3, 3:4]) for t in (x, h))
    a = block.query(maps, px, ph, pos, kv_len=lens)
    b = block.query(pages, px, ph, pos, kv_len=lens, width=side)
    for p, q in zip(a, b):
        assert float((p.float() - q.float()).abs().max()) <= 2.0 ** -7 * float(p.float().abs().max())


def calls(seed=0, dtype=BF):
    """A serving step and a training step of some size, as one function of nothing,
    and its results."""
    heads, kv_heads, dq, lens = 4, 2, 16, [700, 3, 0, 2100]
    table, pages = make_table(np.random.default_rng(seed), [v + 1 for v in lens], 16)
    cache = quan.empty_cache(pages, 16, kv_heads, dq, table)
    kv = rand_map(seed + 1, 1, 2 * kv_heads * dq, 1, sum(lens), dtype)
    new = rand_map(seed + 2, len(lens), 2 * kv_heads * dq, 1, 1, dtype)
    ckv = kv_heads * dq
    q1, qp, do = rand_map(seed + 3, len(lens), heads * dq, 1, 1, dtype), rand_map(seed + 4, 1, heads * dq, 1, sum(lens), dtype), \
        rand_map(seed + 5, 1, heads * dq, 1, sum(lens), dtype)
    first, start, after = ints(ref.starts(lens).tolist()), ints(lens), ints([v + 1 for v in lens])

    def run():
        quan.quan_cache_write(cache, kv[:, :, :ckv], kv[:, :, ckv:], first=first)
        quan.quan_cache_write(cache, new[:, :, :ckv], new[:, :, ckv:], start)
        one = quan.quan_cache_attention(q1, cache, after, heads)
        back = torch.zeros_like(kv)
        k, v = quan.quan_cache_read(cache, back[:, :, :ckv], back[:, :, ckv:], first=first)
        out, saved = quan.quan_packed_attention_forward(qp, k, v, first, heads, save=True)
        return (one, back, out, *quan.quan_packed_attention_backward(qp, k, v, out, saved, do, first, heads))
    return run


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
def test_captured(dtype):
    """Replays of a captured step, with the program's own eager work and waits in
    between, give the eager result's bits; two graphs of one stream share its
    workspace one after the other."""
    say(f"sequences captured {dtype}")
    stream = torch.cuda.Stream()
    runs = [calls(s, dtype) for s in (0, 7)]
    with torch.cuda.stream(stream):
        want = [[t.clone() for t in r()] for r in runs]
        graphs, outs = [], []
        for r in runs:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                outs.append(r())
            graphs.append(g)
    torch.cuda.synchronize()
    for turn in range(3):
        for i in (0, 1, 0) if turn % 2 else (1, 0):
            for t in outs[i]:
                t.fill_(float("nan"))
            torch.cuda.synchronize()
            with torch.cuda.stream(stream):
                graphs[i].replay()
                eager = runs[1 - i]()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outs[i], want[i])), (turn, i)
            assert all(torch.equal(a, b) for a, b in zip(eager, want[1 - i])), (turn, i)


def test_streams_and_threads():
    """Calls of several threads, on streams of their own and on one stream."""
    say("sequences on streams")
    runs = [calls(s) for s in (1, 2, 3, 4)]
    want = [[t.clone() for t in r()] for r in runs]
    torch.cuda.synchronize()
    shared = torch.cuda.Stream()
    streams = [torch.cuda.Stream(), torch.cuda.Stream(), shared, shared]
    got, errors = [None] * 4, []

    def work(i):
        try:
            with torch.cuda.stream(streams[i]):
                for _ in range(5):
                    got[i] = runs[i]()
                streams[i].synchronize()
        except Exception as e:  # noqa: BLE001
            errors.append(e)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    torch.cuda.synchronize()
    assert not errors, errors
    for g, w in zip(got, want):
        assert all(torch.equal(a, b) for a, b in zip(g, w))


def test_repeats():
    """The same calls give the same bits."""
    say("sequences repeat")
    for dtype in (BF, F32):
        run = calls(5, dtype)
        a = [t.clone() for t in run()]
        assert all(torch.equal(x, y) for x, y in zip(a, run()))


def test_long_packed_backward_against_one_sequence():
    """A sequence packed among others is what it is alone."""
    say("packed against alone")
    heads, dq, lens = 2, 16, [300, 900, 64]
    maps = [rand_map(s, 1, heads * dq, 1, sum(lens), BF) for s in range(4)]
    got = step(*maps, ints(ref.starts(lens).tolist()), heads)
    compare(*maps, lens, lens, heads, got, "packed")
    for i, a in enumerate(ref.starts(lens)[:-1]):
        alone = [quan.to_device_layout(t[..., a:a + lens[i]]) for t in maps]
        compare(*alone, [lens[i]], [lens[i]], heads, step(*alone, ints([0, lens[i]]), heads), f"alone {i}")


@pytest.mark.parametrize("dtype", [None, BF], ids=["e4m3", "bf16"])
@pytest.mark.parametrize("side,page", [(20, 64), (8, 6), (8, 16)])
def test_pages_of_whole_maps(dtype, side, page):
    """Without lengths a query reads a map's pixels, as from the cache of maps, and
    not the slots behind them on the last page, which are NaN here: a bf16 step of the
    largest value from the same keys and values in maps (8-bit ones are bf16 numbers)."""
    say(f"block, pages of whole maps {dtype} {side} {page}")
    n, c, heads = 3, 32, 4
    block = AttentionBlock(c, heads, kv_heads=2, radius=side - 1, buckets=9, seed=4)
    x, h = rand_map(1, n, c, side, side, BF), rand_map(2, n, c, side, side, BF)
    pages = block.pages(n, side, side, page_tokens=page, **({} if dtype is None else {"dtype": dtype}))
    for t in pages[:4]:
        if t is not None:
            t.view(torch.uint8).fill_(0x7f if t.dtype == E4M3 else 0xff)
    block.write(pages, h, 0)
    maps = block.cache(n, side, side)
    quan.quan_cache_read(pages, *maps)
    pos = ints([[2, 3], [5, 0], [7, 7]])
    px, ph = (quan.to_device_layout(t[..., 2:3, 3:4]) for t in (x, h))
    want = block.query(maps, px, ph, pos)
    whole = torch.full((n,), side * side, dtype=torch.int32, device=DEV)
    for got in (block.query(pages, px, ph, pos, width=side), block.query(pages, px, ph, pos, kv_len=whole, width=side),
                block.query(pages._replace(table=pages.table.clone()), px, ph, pos, width=side)):
        for p, q in zip(want, got):
            assert float((p.float() - q.float()).abs().max()) <= 2.0 ** -7 * float(p.float().abs().max())
