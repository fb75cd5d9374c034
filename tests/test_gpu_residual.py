"""The residual step of a block (norms, gate, scale, dropout), the norm and
dropout by themselves, against the formulas in 64 bits."""
import numpy as np
import pytest
import torch

from block_reference import drop_factors, residual, residual_gradients
from parity import assert_close, f64, say
from paper_2509_05512_amd import quan

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
EPS = 1e-6
SEED, OFFSET = 0x123456789ABCDEF, 0x7FFFFFFF12345678


def rand_map(seed, n, c, h, w, dtype):
    g = torch.Generator().manual_seed(seed)
    return torch.randn((n, h, w, 4, c), generator=g).to(dtype).permute(0, 3, 4, 1, 2)


def param(seed, c):
    return 1.0 + 0.3 * torch.randn((4, c), generator=torch.Generator().manual_seed(seed))


def f(t):
    return None if t is None else f64(t)


def up(t):
    return None if t is None else (quan.to_device_layout(t.cuda()) if t.dim() == 5 else t.cuda())


def rng():
    return torch.tensor([SEED, OFFSET], dtype=torch.int64, device="cuda")


# rows are 4 c reals: parts of a wave, whole waves, work-groups of 2, 4 and 8
# waves, with and without a last half chunk
SHAPES = [(1, 1, 1, 1), (2, 1, 3, 5), (3, 13, 4, 7), (2, 37, 9, 5), (5, 64, 6, 6), (1, 100, 3, 11), (2, 128, 4, 4),
          (2, 129, 2, 3), (1, 256, 5, 5), (1, 300, 3, 3), (2, 512, 2, 2), (1, 1023, 2, 2), (2, 1024, 1, 3)]
PARTS = [dict(), dict(gate=False), dict(post=False), dict(scale=False), dict(following=False),
         dict(gate=False, post=False, scale=False, following=False)]


def inputs(shape, dtype, gate=True, post=True, scale=True, following=True):
    n, c, h, w = shape
    return dict(gamma=param(1, c) if post else None, gate=rand_map(2, n, c, 1, 1, dtype) if gate else None,
                scale=param(3, c) if scale else None, next_gamma=param(4, c) if following else None)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("p", [0.0, 0.3])
def test_forward_and_backward(shape, p, dtype):
    """Results are fp32 sums of 4 c terms rounded once, far inside the bars of
    both types (one bf16 rounding is 2^-8 of a value, the bar 2e-2)."""
    n, c, h, w = shape
    for parts in PARTS:
        say(f"residual {shape} {p} {dtype} {parts}")
        kw = inputs(shape, dtype, **parts)
        x, y, do, dh, o = (rand_map(10 + i, n, c, h, w, dtype) for i in range(5))
        fac = drop_factors(n, c, h, w, p, SEED, OFFSET)
        g = {k: up(t) for k, t in kw.items()}
        out, hh = quan.quan_residual_forward(up(x), up(y), p=p, rng=rng(), eps=EPS, **g)
        r_out, r_h = residual(f(x), f(y), f(kw["gamma"]), f(kw["gate"]), f(kw["scale"]), f(kw["next_gamma"]), fac, EPS)
        assert_close(f64(out), r_out, dtype, "out")
        assert (hh is None) == (r_h is None)
        if hh is not None:
            assert_close(f64(hh), r_h, dtype, "h")
        fol = kw["next_gamma"] is not None
        res = quan.quan_residual_backward(up(y), up(do), out=up(o) if fol else None, dh=up(dh) if fol else None, p=p,
                                          rng=rng(), eps=EPS, **g)
        ref = residual_gradients(f(y), f(do), f(kw["gamma"]), f(kw["gate"]), f(kw["scale"]), f(kw["next_gamma"]),
                                 f(o), f(dh), fac, EPS)
        for name in ("dx", "dy", "dgate"):
            got = getattr(res, name)
            assert (got is None) == (name not in ref)
            if got is not None:
                assert_close(f64(got), ref[name], dtype, name)
        for name in ("dgamma", "dscale", "dnext_gamma"):
            got = getattr(res, name)
            assert (got is None) == (name not in ref)
            if got is not None:
                assert_close(f64(got), ref[name], F32, name)


@pytest.mark.parametrize("shape", [(700, 16, 1, 2), (2100, 4, 1, 1), (3, 16, 70, 90), (1, 256, 60, 60)], ids=str)
@pytest.mark.parametrize("gate", [True, False])
def test_many_images_and_many_pixels(shape, gate):
    """More images than work-groups, several work-groups per image: the sums by
    image and over all."""
    n, c, h, w = shape
    say(f"many {shape} {gate}")
    kw = inputs(shape, F32, gate=gate)
    y, do, dh, o = (rand_map(10 + i, n, c, h, w, F32) for i in range(4))
    res = quan.quan_residual_backward(up(y), up(do), out=up(o), dh=up(dh), eps=EPS, **{k: up(t) for k, t in kw.items()})
    ref = residual_gradients(f(y), f(do), f(kw["gamma"]), f(kw["gate"]), f(kw["scale"]), f(kw["next_gamma"]), f(o),
                             f(dh), 1.0, EPS)
    for name, want in ref.items():
        assert_close(f64(getattr(res, name)), want, F32, name)
    again = quan.quan_residual_backward(up(y), up(do), out=up(o), dh=up(dh), eps=EPS, **{k: up(t) for k, t in kw.items()})
    assert all(torch.equal(a, b) for a, b in zip(res, again) if a is not None)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("shape", SHAPES[:10:3], ids=str)
def test_norm(shape, dtype):
    n, c, h, w = shape
    say(f"norm {shape} {dtype}")
    x, do, dr = (rand_map(20 + i, n, c, h, w, dtype) for i in range(3))
    gamma = param(5, c)
    xs = up(x)
    out = quan.quan_rmsnorm_forward(xs, gamma.cuda(), eps=EPS)
    want = residual(f(x), 0.0 * f(x), None, None, None, f(gamma), 1.0, EPS)[1]
    assert_close(f64(out), want, dtype, "out")
    for res in (None, dr):
        ref = residual_gradients(0.0 * f(x), 0.0 * f(x) if res is None else f(res), None, None, None, f(gamma), f(x),
                                 f(do), 1.0, EPS)
        dx, dgamma = quan.quan_rmsnorm_backward(xs, up(do), gamma.cuda(), dres=up(res), eps=EPS)
        assert_close(f64(dx), ref["dx"], dtype, "dx")
        assert_close(f64(dgamma), ref["dnext_gamma"], F32, "dgamma")
    held = xs.clone(memory_format=torch.preserve_format)
    assert torch.equal(quan.quan_rmsnorm_forward(held, gamma.cuda(), eps=EPS, out=held), out)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.99999, 1e-7])
def test_dropout(shape, p, dtype):
    """The mask is the generator's, word by word; the same call drops a
    gradient; in place."""
    n, c, h, w = shape
    say(f"dropout {shape} {p} {dtype}")
    x = rand_map(1, n, c, h, w, dtype)
    fac = drop_factors(n, c, h, w, p, SEED, OFFSET)
    if p == 0.99999:
        fac = drop_factors(n, c, h, w, 65535 / 65536, SEED, OFFSET)  # the largest p'
    out = quan.quan_dropout(up(x), p, rng())
    assert np.array_equal(f64(out) != 0, (fac != 0) & (f64(x) != 0))
    assert_close(f64(out), f64(x) * fac, dtype, "out")
    t = up(x)
    assert torch.equal(quan.quan_dropout(t, p, rng(), out=t), out)


def test_dropout_rate_and_independence():
    """Of 2^22 reals a share p is dropped to within 5 standard deviations, and
    masks of other offsets agree as often as independent ones."""
    say("dropout statistics")
    x = torch.ones((64, 64, 64, 4, 4), dtype=BF, device="cuda").permute(0, 3, 4, 1, 2)
    n = x.numel()
    masks = []
    for off in range(3):
        m = quan.quan_dropout(x, 0.25, torch.tensor([1, off], dtype=torch.int64, device="cuda")) == 0
        masks.append(m)
        assert abs(float(m.float().mean()) - 0.25) <= 5 * (0.1875 / n) ** 0.5
    for a, b in ((0, 1), (1, 2), (0, 2)):
        both = float((masks[a] & masks[b]).float().mean())
        assert abs(both - 0.0625) <= 5 * (0.0625 * 0.9375 / n) ** 0.5


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
def test_dropped_reals_hide_nan(dtype):
    """A dropped real is zero whatever it was; a kept NaN stays in its pixel."""
    say(f"dropped NaN {dtype}")
    n, c, h, w, p = 1, 8, 4, 4, 0.5
    fac = drop_factors(n, c, h, w, p, SEED, OFFSET)
    x = torch.where(torch.from_numpy(fac == 0), torch.tensor(float("nan")), torch.tensor(1.0)).to(dtype)
    out = quan.quan_dropout(up(x), p, rng())
    assert np.array_equal(f64(out), fac)
    y = rand_map(3, n, c, h, w, dtype)
    y[0, 1, 2, 3, 1] = float("inf")
    got, _ = quan.quan_residual_forward(up(rand_map(4, n, c, h, w, dtype)), up(y), gamma=up(param(1, c)), eps=EPS)
    bad = f64(got)
    assert np.all(np.isfinite(np.delete(bad.reshape(4 * c, -1), 3 * w + 1, 1)))


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
def test_zero_rows(dtype):
    """Rows of zeros: norms are zero, gradients finite."""
    say(f"zero rows {dtype}")
    n, c, h, w = 2, 16, 3, 3
    kw = inputs((n, c, h, w), dtype)
    y, o = torch.zeros_like(rand_map(1, n, c, h, w, dtype)), torch.zeros_like(rand_map(1, n, c, h, w, dtype))
    do, dh = (1e-3 * rand_map(i, n, c, h, w, F32) for i in (2, 3))
    do, dh = do.to(dtype), dh.to(dtype)
    out, hh = quan.quan_residual_forward(up(o), up(y), eps=EPS, **{k: up(t) for k, t in kw.items()})
    assert not out.any() and not hh.any()
    res = quan.quan_residual_backward(up(y), up(do), out=up(o), dh=up(dh), eps=EPS, **{k: up(t) for k, t in kw.items()})
    ref = residual_gradients(f(y), f(do), f(kw["gamma"]), f(kw["gate"]), f(kw["scale"]), f(kw["next_gamma"]), f(o),
                             f(dh), 1.0, EPS)
    for name in ("dx", "dy"):
        assert_close(f64(getattr(res, name)), ref[name], dtype, name)


def test_in_place_forms():
    say("in place")
    shape = (2, 20, 5, 6)
    n, c, h, w = shape
    kw = {k: up(t) for k, t in inputs(shape, BF).items()}
    x, y, do, dh, o = (up(rand_map(i, n, c, h, w, BF)) for i in range(5))
    out, hh = quan.quan_residual_forward(x, y, p=0.2, rng=rng(), **kw)
    for into in (x, y):
        a, b = x.clone(memory_format=torch.preserve_format), y.clone(memory_format=torch.preserve_format)
        got, h2 = quan.quan_residual_forward(a, b, p=0.2, rng=rng(), out=a if into is x else b, **kw)
        assert torch.equal(got, out) and torch.equal(h2, hh)
    want = quan.quan_residual_backward(y, do, out=o, dh=dh, p=0.2, rng=rng(), **kw)
    for which in ("dout", "dh"):
        a, b, d = (t.clone(memory_format=torch.preserve_format) for t in (y, do, dh))
        got = quan.quan_residual_backward(a, b, out=o, dh=d, p=0.2, rng=rng(), dx=b if which == "dout" else d, dy=a, **kw)
        assert all(torch.equal(s, t) for s, t in zip(got, want))


def test_gradients_against_differences():
    """<gradient, direction> against central differences in 64 bits (step
    1e-5), the dropout's mask held."""
    say("differences")
    shape = (2, 5, 3, 4)
    n, c, h, w = shape
    kw = inputs(shape, F32)
    x, y, go, gh = (rand_map(i, n, c, h, w, F32) for i in range(4))
    fac = drop_factors(n, c, h, w, 0.25, SEED, OFFSET)
    a = {"dx": f(x), "dy": f(y), **{"d" + k: f(t) for k, t in kw.items()}}

    def loss(a):
        o, hh = residual(a["dx"], a["dy"], a["dgamma"], a["dgate"], a["dscale"], a["dnext_gamma"], fac, EPS)
        return float((o * f(go)).sum() + (hh * f(gh)).sum())
    g = {k: up(t) for k, t in kw.items()}
    out, _ = quan.quan_residual_forward(up(x), up(y), p=0.25, rng=rng(), eps=EPS, **g)
    res = quan.quan_residual_backward(up(y), up(go), out=out, dh=up(gh), p=0.25, rng=rng(), eps=EPS, **g)
    r = np.random.default_rng(0)
    for name in a:
        d = r.standard_normal(a[name].shape)
        up_, down = ({**a, name: a[name] + s * 1e-5 * d} for s in (1, -1))
        got = f64(getattr(res, name)) * d
        assert abs(got.sum() - (loss(up_) - loss(down)) / 2e-5) <= 1e-5 * (1 + np.abs(got).sum()), name


def test_graph_sees_a_new_seed():
    """rng is read on the device: a replay with another seed drops others."""
    say("graph with a new seed")
    shape = (2, 16, 6, 6)
    n, c, h, w = shape
    kw = {k: up(t) for k, t in inputs(shape, BF).items()}
    x, y, do, dh = (up(rand_map(i, n, c, h, w, BF)) for i in range(4))
    r = rng()

    def step():
        out, hh = quan.quan_residual_forward(x, y, p=0.4, rng=r, **kw)
        g = quan.quan_residual_backward(y, do, out=out, dh=dh, p=0.4, rng=r, **kw)
        return (out, hh, quan.quan_dropout(x, 0.4, r), *g)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        first = step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        held = step()
    for seed in (SEED, 5, 6):
        r.copy_(torch.tensor([seed, 9]))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want))
        assert not torch.equal(held[2], first[2])
