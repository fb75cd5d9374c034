"""Attention between the pixels of maps with a learned bias by buckets of the
relative position, against the formulas in 64 bits (tests/block_reference.py
derives the bounds)."""
import numpy as np
import pytest
import torch

from block_reference import attention, check
from parity import f64, say
from paper_2509_05512_amd import quan

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def rand_map(seed, n, c, h, w, dtype, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (std * torch.randn((n, h, w, 4, c), generator=g)).to(dtype).permute(0, 3, 4, 1, 2)


def bias_of(seed, heads, hq, wq, hk, wk, ny, nx, ry=None, rx=None):
    """(table [heads, ny, nx], by, bx) with buckets from the library's map, or
    random ones where there are more buckets than it needs."""
    g = torch.Generator().manual_seed(seed)
    ry = max(hq, hk) - 1 if ry is None else ry
    rx = max(wq, wk) - 1 if rx is None else rx
    table = torch.randn((heads, ny, nx), generator=g)
    return table, quan.quan_relpos_buckets(ry, ny), quan.quan_relpos_buckets(rx, nx)


def run(q, k, v, heads, relpos=None, kv_len=None, pos=None, scale=None, dout=None, wide=False):
    """Forward, and with dout backward, on the GPU; wide: q, k, v and their
    gradients are channel slices of one map."""
    dev = torch.device("cuda")
    c, ckv = q.shape[2], k.shape[2]

    def up(t):
        return None if t is None else t.to(dev)
    rp = None if relpos is None else tuple(up(t) for t in relpos)
    kw = dict(relpos=rp, kv_len=up(kv_len), pos=up(pos), scale=scale)
    if wide:
        whole = quan.to_device_layout(torch.cat([q, k, v], 2).to(dev))
        qd, kd, vd = whole[:, :, :c], whole[:, :, c:c + ckv], whole[:, :, c + ckv:]
        assert not quan.is_device_layout(qd) or q.shape[2] == whole.shape[2]
    else:
        qd, kd, vd = (quan.to_device_layout(t.to(dev)) for t in (q, k, v))
    if dout is None:
        return {"out": quan.quan_attention_forward(qd, kd, vd, heads, **kw)}
    out, stats, rest = quan.quan_attention_forward(qd, kd, vd, heads, save=True, **kw)
    grads = {}
    if wide:
        dw = torch.full_like(whole, float("nan"))
        grads = dict(dq=dw[:, :, :c], dk=dw[:, :, c:c + ckv], dv=dw[:, :, c + ckv:])
    dq, dk, dv, dtable = quan.quan_attention_backward(qd, kd, vd, out, stats, rest, quan.to_device_layout(dout.to(dev)),
                                                      heads, **grads, **kw)
    torch.cuda.synchronize()
    return {"out": out, "stats": stats, "dq": dq, "dk": dk, "dv": dv, "dtable": dtable}


def compare(res, q, k, v, heads, relpos=None, kv_len=None, pos=None, scale=None, dout=None):
    arrays = [None, None, None] if relpos is None else [None if t is None else t.numpy() for t in relpos]
    table = None if arrays[0] is None else arrays[0].astype(np.float64)
    ref, err = attention(f64(q), f64(k), f64(v), heads, table, arrays[1], arrays[2],
                         None if kv_len is None else kv_len.numpy(), None if pos is None else pos.numpy(), scale,
                         None if dout is None else f64(dout))
    bf = q.dtype == BF
    for name in ("out", "dq", "dk", "dv"):
        if name in res:
            check(f64(res[name]), ref[name], err[name], bf, name)
    if res.get("dtable") is not None:
        check(f64(res["dtable"]), ref["dtable"], err["dtable"], bf, "dtable")
    if "stats" in res:
        st = f64(res["stats"])
        with np.errstate(divide="ignore"):
            lse = (st[..., 0] + np.log2(st[..., 1])) * np.log(2.0)
        assert np.array_equal(np.isneginf(lse), np.isneginf(ref["lse"]))
        # (a maximum below the type's lowest, in units of log 2, is that)
        ok = np.isfinite(lse) & (ref["lse"] > -2e38)
        assert np.all(lse[np.isfinite(lse) & ~ok] < -2e38)
        assert np.all(np.abs(lse[ok] - ref["lse"][ok]) <= 1e-5 * (1 + np.abs(ref["lse"][ok])))
    return ref


# n, (hq, wq), (hk, wk), heads, kv_heads, dq, (ny, nx): tiles are 128 queries or
# keys and 64 (fp32: 32) of the other side
SELF = [
    (1, (1, 1), (1, 1), 1, 1, 1, (1, 1)),
    (2, (1, 2), (1, 2), 2, 1, 2, (1, 3)),
    (1, (1, 63), (1, 63), 1, 1, 8, (1, 16)),
    (1, (1, 65), (1, 65), 2, 2, 16, (1, 129)),
    (2, (1, 129), (1, 129), 1, 1, 32, (1, 8)),
    (2, (5, 7), (5, 7), 4, 2, 5, (9, 13)),
    (1, (7, 9), (7, 9), 4, 1, 12, (4, 6)),
    (3, (8, 8), (8, 8), 2, 2, 8, (15, 15)),
    (2, (13, 20), (13, 20), 2, 1, 16, (8, 8)),
    (1, (14, 14), (14, 14), 3, 3, 24, (27, 27)),
    (1, (20, 33), (20, 33), 1, 1, 7, (5, 65)),
]


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("case", SELF, ids=str)
@pytest.mark.parametrize("wide", [False, True], ids=["maps", "slices"])
def test_training_step(case, dtype, wide):
    n, (hq, wq), (hk, wk), heads, kvh, dq, (ny, nx) = case
    say(f"training step {case} {dtype} {wide}")
    q, do = (rand_map(s, n, heads * dq, hq, wq, dtype) for s in (1, 4))
    k, v = (rand_map(s, n, kvh * dq, hk, wk, dtype) for s in (2, 3))
    relpos = bias_of(5, heads, hq, wq, hk, wk, ny, nx)
    compare(run(q, k, v, heads, relpos, dout=do, wide=wide), q, k, v, heads, relpos, dout=do)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
def test_without_bias(dtype):
    say(f"no bias {dtype}")
    q, k, v, do = (rand_map(s, 2, 24, 9, 11, dtype) for s in (1, 2, 3, 4))
    compare(run(q, k, v, 3, dout=do), q, k, v, 3, dout=do)
    compare(run(q, k, v, 3), q, k, v, 3)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("shape", [((3, 5), (6, 9)), ((1, 7), (4, 40)), ((6, 6), (1, 70)), ((2, 2), (1, 1))], ids=str)
def test_other_maps_of_keys(shape, dtype):
    """Queries of a map of their own, placed in the keys' map by pos (outside
    it too), lengths of keys from none to more than there are."""
    (hq, wq), (hk, wk) = shape
    say(f"cross {shape} {dtype}")
    n, heads = 4, 2
    q, do = (rand_map(s, n, heads * 8, hq, wq, dtype) for s in (1, 4))
    k, v = (rand_map(s, n, heads * 8, hk, wk, dtype) for s in (2, 3))
    relpos = bias_of(5, heads, hq, wq, hk, wk, 6, 7, 5, 4)
    pos = torch.tensor([[0, 0], [1, 3], [-2, 100], [hk - 1, wk - 1]], dtype=torch.int32)
    lens = torch.tensor([0, 1, hk * wk + 5, max(1, hk * wk - 1)], dtype=torch.int32)
    compare(run(q, k, v, heads, relpos, lens, pos, dout=do), q, k, v, heads, relpos, lens, pos, dout=do)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
def test_what_lies_behind_the_keys_is_not_read(dtype):
    """NaN and infinities behind kv_len change nothing, and their gradients are
    zero."""
    say(f"behind kv_len {dtype}")
    n, heads, L = 3, 2, 150
    q, do = (rand_map(s, n, 16, 1, L, dtype) for s in (1, 4))
    k, v = (rand_map(s, n, 16, 1, L, dtype) for s in (2, 3))
    lens = torch.tensor([0, 70, 149], dtype=torch.int32)
    relpos = bias_of(5, heads, 1, L, 1, L, 1, 16, 0, 32)
    clean = run(q, k, v, heads, relpos, lens, dout=do)
    one = run(q[..., :1], k, v, heads, relpos, lens)["out"]
    kn, vn = k.clone(), v.clone()
    for i, m in enumerate(lens.tolist()):
        kn[i, :, :, :, m:] = float("nan")
        vn[i, :, :, :, m:] = float("inf")
    dirty = run(q, kn, vn, heads, relpos, lens, dout=do)
    for name in ("out", "dq", "dk", "dv", "dtable"):
        assert torch.equal(clean[name], dirty[name]), name
    assert torch.equal(one, run(q[..., :1], kn, vn, heads, relpos, lens)["out"])
    for i, m in enumerate(lens.tolist()):
        assert not dirty["dk"][i, ..., m:].any() and not dirty["dv"][i, ..., m:].any()
    assert not dirty["out"][0].any() and not dirty["dq"][0].any()
    compare(dirty, q, k, v, heads, relpos, lens, dout=do)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("lq", [100, 1])
def test_bias_that_masks(dtype, lq):
    """-infinity keeps pairs apart, rows that it empties give zeros; the type's
    lowest value gives a row of nothing else an even softmax."""
    say(f"masking bias {dtype} {lq}")
    L, heads = 100, 3
    q, do = (rand_map(s, 1, 24, 1, lq, dtype) for s in (1, 4))
    k, v = (rand_map(s, 1, 24, 1, L, dtype) for s in (2, 3))
    low = torch.finfo(torch.float32).min
    # head 0: earlier keys alone (query 0 sees itself), head 1: keys at a
    # distance of 60 and more alone (queries 40..59 see none), head 2: lowest
    # for all but keys 90 and more to the right (queries 10.. see lowest alone)
    d = torch.arange(-(L - 1), L)
    table = torch.zeros((heads, 1, 2 * L - 1))
    table[0, 0, d > 0] = -float("inf")
    table[1, 0, d.abs() < 60] = -float("inf")
    table[2, 0, d < 90] = low
    relpos = (table, None, torch.arange(2 * L - 1, dtype=torch.int32))
    pos = None if lq > 1 else torch.tensor([[0, 50]], dtype=torch.int32)
    dout = do if lq > 1 else None
    res = run(q, k, v, heads, relpos, pos=pos, dout=dout)
    compare(res, q, k, v, heads, relpos, pos=pos, dout=dout)
    out = f64(res["out"])[0, :, 8:16, 0]
    assert not np.any(out[..., 40:60] if lq > 1 else out)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("heads,kvh,dq", [(1, 1, 8), (4, 4, 16), (8, 2, 16), (6, 2, 12), (5, 1, 3), (16, 2, 32), (3, 3, 32)])
@pytest.mark.parametrize("hw", [(1, 1), (3, 5), (1, 700), (37, 41)], ids=str)
def test_one_query(heads, kvh, dq, hw, dtype):
    """The form for single queries, its keys split over work-groups."""
    say(f"one query {heads} {kvh} {dq} {hw} {dtype}")
    h, w = hw
    n = 3
    q, do = (rand_map(s, n, heads * dq, 1, 1, dtype) for s in (1, 4))
    k, v = (rand_map(s, n, kvh * dq, h, w, dtype) for s in (2, 3))
    relpos = bias_of(5, heads, 1, 1, h, w, 5, 8, 3, 20)
    pos = torch.tensor([[0, 0], [h // 2, w // 2], [h - 1, w - 1]], dtype=torch.int32)
    lens = torch.tensor([h * w, max(0, h * w - 130), 0], dtype=torch.int32)
    compare(run(q, k, v, heads, relpos, lens, pos), q, k, v, heads, relpos, lens, pos)
    compare(run(q, k, v, heads, relpos, lens, pos, dout=do, wide=False), q, k, v, heads, relpos, lens, pos, dout=do)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("lq", [2, 33])
def test_few_queries_many_keys(dtype, lq):
    """Few rows: the keys are split over work-groups and joined."""
    say(f"few queries {lq} {dtype}")
    heads, L = 2, 1500
    q, do = (rand_map(s, 1, 32, 1, lq, dtype) for s in (1, 4))
    k, v = (rand_map(s, 1, 32, 1, L, dtype) for s in (2, 3))
    relpos = bias_of(5, heads, 1, lq, 1, L, 1, 32, 0, 128)
    pos = torch.tensor([[0, L - lq]], dtype=torch.int32)
    compare(run(q, k, v, heads, relpos, None, pos, dout=do), q, k, v, heads, relpos, None, pos, dout=do)


def test_unaligned_slices():
    """Slices that start between 16-byte chunks, components at odd strides."""
    say("unaligned slices")
    n, h, w, heads = 2, 6, 11, 2
    base = torch.randn((n, h, w, 4, 55), generator=torch.Generator().manual_seed(1)).to(BF).cuda().permute(0, 3, 4, 1, 2)
    q, k, v, do = base[:, :, 1:17], base[:, :, 18:34], base[:, :, 35:51], rand_map(2, n, 16, h, w, BF)
    dw = torch.full_like(base, 7.0)
    relpos = bias_of(5, heads, h, w, h, w, 5, 6)
    rp = tuple(t.cuda() for t in relpos)
    out, stats, rest = quan.quan_attention_forward(q, k, v, heads, relpos=rp, save=True, out=dw[:, :, 0:16])
    dq, dk, dv, dt = quan.quan_attention_backward(q, k, v, out, stats, rest, quan.to_device_layout(do.cuda()), heads,
                                                  relpos=rp, dk=dw[:, :, 17:33], dv=dw[:, :, 34:50])
    compare({"out": out, "dq": dq, "dk": dk, "dv": dv, "dtable": dt}, q.cpu(), k.cpu(), v.cpu(), heads, relpos, dout=do)
    for c in (16, 33, 50, 51, 54):
        assert bool((dw[:, :, c] == 7.0).all()), "channels beside the slices are untouched"


def test_wide_maps_and_scale():
    """Rows as wide as they may be with a bias, several segments of offsets, a
    scale of one's own."""
    say("wide maps")
    n, heads, h, w = 1, 1, 2, 700
    q, k, v, do = (rand_map(s, n, 8, h, w, BF) for s in (1, 2, 3, 4))
    relpos = bias_of(5, heads, h, w, h, w, 3, 33, 1, 300)
    compare(run(q, k, v, heads, relpos, scale=0.3, dout=do), q, k, v, heads, relpos, scale=0.3, dout=do)
    q, k, v, do = (rand_map(s, n, 8, 2, 1792, BF) for s in (1, 2, 3, 4))
    relpos = bias_of(5, heads, 2, 1792, 2, 1792, 3, 9)
    compare(run(q, k, v, heads, relpos, dout=do), q, k, v, heads, relpos, dout=do)


def test_large_and_small_values():
    """The sums by offset meet terms that differ by many orders of magnitude,
    the larger ones later and earlier; equal scores and peaked ones."""
    say("ranges of values")
    L, heads = 400, 1
    for order in (1, -1):
        q, k, v, do = (rand_map(s, 2, 16, 1, L, F32) for s in (1, 2, 3, 4))
        steps = torch.logspace(-12, 3, L)
        steps = steps if order > 0 else steps.flip(0)
        v = v * steps
        do[1] *= 1e-20
        q[0] *= 3.0
        relpos = bias_of(5, heads, 1, L, 1, L, 1, 32, 0, 100)
        compare(run(q, k, v, heads, relpos, dout=do), q, k, v, heads, relpos, dout=do)


def test_nan_reaches_its_rows_and_the_bias():
    say("NaN in a query")
    L = 200
    q, k, v, do = (rand_map(s, 2, 8, 1, L, BF) for s in (1, 2, 3, 4))
    relpos = bias_of(5, 1, 1, L, 1, L, 1, 16)
    clean = run(q, k, v, 1, relpos, dout=do)
    q[1, 0, 0, 0, 7] = float("nan")
    res = run(q, k, v, 1, relpos, dout=do)
    keep = torch.arange(L) != 7
    assert torch.equal(res["out"][..., keep.cuda()], clean["out"][..., keep.cuda()])
    assert bool(res["out"][1, ..., 7].isnan().all()) and bool(res["dq"][1, ..., 7].isnan().all())
    assert bool(res["dk"][1].isnan().any()) and not bool(res["dk"][0].isnan().any())
    assert bool(res["dtable"].isnan().any())


def test_deterministic():
    say("determinism")
    q, k, v, do = (rand_map(s, 4, 32, 20, 23, BF) for s in (1, 2, 3, 4))
    relpos = bias_of(5, 4, 20, 23, 20, 23, 8, 8)
    a, b = (run(q, k, v, 4, relpos, dout=do) for _ in range(2))
    for name in ("out", "dq", "dk", "dv", "dtable"):
        assert torch.equal(a[name], b[name]), name


def test_gradients_against_differences():
    """<gradient, direction> of every input against central differences of the
    loss in 64 bits, step 1e-4: their error is 1e-8 of the third derivative."""
    say("differences")
    n, h, w, heads, dq = 2, 4, 5, 2, 3
    q, k, v, do = (rand_map(s, n, heads * dq, h, w, F32) for s in (1, 2, 3, 4))
    table, by, bx = bias_of(5, heads, h, w, h, w, 4, 5)
    lens = torch.tensor([20, 13], dtype=torch.int32)
    res = run(q, k, v, heads, (table, by, bx), lens, dout=do)
    args = {"dq": f64(q), "dk": f64(k), "dv": f64(v), "dtable": table.numpy().astype(np.float64)}
    go = f64(do)

    def loss(a):
        r, _ = attention(a["dq"], a["dk"], a["dv"], heads, a["dtable"], by.numpy(), bx.numpy(), lens.numpy())
        return float((r["out"] * go).sum())
    rng = np.random.default_rng(0)
    for name in args:
        d = rng.standard_normal(args[name].shape)
        up, down = ({**args, name: args[name] + s * 1e-4 * d} for s in (1, -1))
        want = (loss(up) - loss(down)) / 2e-4
        got = float((f64(res[name]) * d).sum())
        assert abs(got - want) <= 1e-5 * (1 + np.abs(f64(res[name]) * d).sum()), name


def test_offsets_beyond_32_bits():
    """A cache whose elements' offsets pass 2^31, in bytes 2^33: the last keys
    are found, by one query and by a tile of them."""
    say("offsets beyond 32 bits")
    L, c_all, dq = 4_300_000, 128, 8
    cache = torch.zeros((1, 1, L, 4, c_all), dtype=BF, device="cuda").permute(0, 3, 4, 1, 2)
    assert cache.numel() > 2 ** 31
    tail = 300
    g = torch.Generator().manual_seed(3)
    kv = torch.randn((1, 1, tail, 4, 2 * dq), generator=g).to(BF).permute(0, 3, 4, 1, 2)
    cache[:, :, 100:100 + 2 * dq, :, L - tail:] = kv.cuda()
    k, v = cache[:, :, 100:100 + dq], cache[:, :, 100 + dq:100 + 2 * dq]
    # keys before the tail are kept apart by the bias: -infinity at distances
    # of `tail` and more to the left of the last key
    r = 2 * tail
    table = torch.full((1, 1, 2), -float("inf"))
    table[0, 0, 1] = 0.5
    for lq in (1, 40):
        q = rand_map(4, 1, dq, 1, lq, BF)
        # a query sees its tail - lq predecessors and what follows it
        bx = torch.tensor([1 if -(tail - lq) < d <= r else 0 for d in range(-r, r + 1)], dtype=torch.int32)
        pos = torch.tensor([[0, L - lq]], dtype=torch.int32)
        out = quan.quan_attention_forward(q.cuda(), k, v, 1, relpos=(table.cuda(), None, bx.cuda()), pos=pos.cuda())
        pos_ref = torch.tensor([[0, tail - lq]], dtype=torch.int32)
        compare({"out": out}, q, kv[:, :, :dq], kv[:, :, dq:], 1, (table, None, bx), pos=pos_ref)
    del cache


def test_other_streams_and_graphs():
    """A captured training step replays on new inputs; eager calls and other
    streams between the replays change nothing."""
    say("streams and graphs")
    dev = torch.device("cuda")
    q, k, v, do = (quan.to_device_layout(rand_map(s, 2, 16, 9, 10, BF).to(dev)) for s in (1, 2, 3, 4))
    rp = tuple(t.to(dev) for t in bias_of(5, 2, 9, 10, 9, 10, 6, 6))
    q1 = quan.to_device_layout(rand_map(6, 2, 16, 1, 1, BF).to(dev))

    def step():
        out, stats, rest = quan.quan_attention_forward(q, k, v, 2, relpos=rp, save=True)
        return (out, quan.quan_attention_forward(q1, k, v, 2, relpos=rp),
                *quan.quan_attention_backward(q, k, v, out, stats, rest, do, 2, relpos=rp))
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        want = step()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, step()))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        held = step()
    for rep in range(3):
        q.copy_(rand_map(10 + rep, 2, 16, 9, 10, BF))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want))
