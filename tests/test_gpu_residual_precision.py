"""The residual step's bf16 maps are fp32 results rounded once: off by at most
2^-8 of a value (half of the last of its 8 bits) and fp32's own error, 1e-5 of
the largest sum of the terms' absolute values."""
import numpy as np
import pytest
import torch

from block_reference import drop_factors, residual, residual_gradients
from parity import f64, say
from paper_2509_05512_amd import quan

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
EPS, SEED, OFFSET = 1e-6, 77, 5


def rand_map(seed, n, c, h, w):
    g = torch.Generator().manual_seed(seed)
    return torch.randn((n, h, w, 4, c), generator=g).to(BF).permute(0, 3, 4, 1, 2)


def param(seed, c):
    return 1.0 + 0.3 * torch.randn((4, c), generator=torch.Generator().manual_seed(seed))


def up(t):
    return quan.to_device_layout(t.cuda()) if t.dim() == 5 else t.cuda()


def check(got, ref, size, what):
    off = np.abs(f64(got) - ref) - 2.0 ** -8 * np.abs(ref)
    assert np.all(off <= 1e-5 * np.abs(size).max()), (what, float(off.max()))


@pytest.mark.parametrize("shape", [(2, 1, 3, 5), (3, 13, 4, 7), (5, 64, 6, 6), (2, 129, 2, 3), (1, 300, 3, 3), (2, 1024, 1, 3)],
                         ids=str)
@pytest.mark.parametrize("p", [0.0, 0.3])
def test_one_rounding(shape, p):
    say(f"one rounding {shape} {p}")
    n, c, h, w = shape
    x, y, do, dh, o = (rand_map(10 + i, n, c, h, w) for i in range(5))
    gate, gamma, scale, following = rand_map(2, n, c, 1, 1), param(1, c), param(3, c), param(4, c)
    rng = torch.tensor([SEED, OFFSET], dtype=torch.int64, device="cuda")
    kw = dict(gamma=up(gamma), gate=up(gate), scale=up(scale), next_gamma=up(following), p=p, rng=rng, eps=EPS)
    args = (f64(gamma), f64(gate), f64(scale), f64(following), drop_factors(n, c, h, w, p, SEED, OFFSET), EPS)
    out, hh = quan.quan_residual_forward(up(x), up(y), **kw)
    r_out, r_h = residual(f64(x), f64(y), *args)
    check(out, r_out, np.abs(f64(x)) + np.abs(r_out - f64(x)), "out")
    check(hh, r_h, r_h, "h")
    res = quan.quan_residual_backward(up(y), up(do), out=up(o), dh=up(dh), **kw)
    ref = residual_gradients(f64(y), f64(do), *args[:4], f64(o), f64(dh), *args[4:])
    # (terms: dout, dh and the means that the norms take off, each at most the
    # largest of those, times the parameters)
    check(res.dx, ref["dx"], 3.0 * max(np.abs(ref["dx"]).max(), 1.0), "dx")
    check(res.dy, ref["dy"], 3.0 * max(np.abs(ref["dy"]).max(), 1.0), "dy")
    check(res.dgate, ref["dgate"], 3.0 * h * w * max(np.abs(ref["dx"]).max(), 1.0), "dgate")
