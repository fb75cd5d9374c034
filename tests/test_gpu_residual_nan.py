"""NaN in the rows of the residual step and of the norm: every result that a NaN
enters is NaN, every other one is what it was."""
import pytest
import torch

from parity import say
from paper_2509_05512_amd import quan

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
# rows of half a chunk, parts of a wave, work-groups of 2 and 8 waves
CHANNELS = [1, 13, 64, 256, 1024]
N, H, W = 2, 3, 4


def rand_map(seed, c, dtype):
    g = torch.Generator().manual_seed(seed)
    return torch.randn((N, H, W, 4, c), generator=g).to(dtype).cuda().permute(0, 3, 4, 1, 2)


def param(seed, c):
    return (1.0 + 0.3 * torch.randn((4, c), generator=torch.Generator().manual_seed(seed))).cuda()


def with_nan(t):
    """One NaN, in the pixel (1, 2) of image 1."""
    t = t.clone(memory_format=torch.preserve_format)
    t[1, 2, t.shape[2] // 2, 1, 2] = float("nan")
    return t


def check_pixel(got, clean, what):
    """The pixel is NaN in every channel, the others have not changed."""
    assert bool(got[1, :, :, 1, 2].isnan().all()), what
    rest = got.clone(memory_format=torch.preserve_format)
    rest[1, :, :, 1, 2] = clean[1, :, :, 1, 2]
    assert torch.equal(rest, clean), what


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("c", CHANNELS)
def test_norm(c, dtype):
    say(f"NaN in the norm {c} {dtype}")
    x, do, gamma = rand_map(1, c, dtype), rand_map(2, c, dtype), param(3, c)
    check_pixel(quan.quan_rmsnorm_forward(with_nan(x), gamma), quan.quan_rmsnorm_forward(x, gamma), "out")
    clean = quan.quan_rmsnorm_backward(x, do, gamma)[0]
    dx, dgamma = quan.quan_rmsnorm_backward(with_nan(x), do, gamma)
    check_pixel(dx, clean, "dx")
    assert bool(dgamma.isnan().all())


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("c", CHANNELS)
@pytest.mark.parametrize("p", [0.0, 0.3])
def test_residual_step(c, p, dtype):
    say(f"NaN in the residual step {c} {p} {dtype}")
    x, y, do, dh = (rand_map(s, c, dtype) for s in (1, 2, 3, 4))
    kw = dict(gamma=param(5, c), scale=param(6, c), next_gamma=param(7, c), p=p,
              rng=torch.tensor([3, 4], dtype=torch.int64, device="cuda"),
              gate=quan.to_device_layout(rand_map(8, c, dtype)[..., :1, :1]))
    out, h = quan.quan_residual_forward(x, y, **kw)
    got, got_h = quan.quan_residual_forward(with_nan(x), y, **kw)  # (one channel of out, all of h)
    check_pixel(got_h, h, "h of x")
    assert int(got.isnan().sum()) == 1
    got, got_h = quan.quan_residual_forward(x, with_nan(y), **kw)
    check_pixel(got_h, h, "h of y")
    if p == 0.0:  # (dropped reals are zero whatever they were)
        check_pixel(got, out, "out of y")

    clean = quan.quan_residual_backward(y, do, out=out, dh=dh, **kw)
    # a NaN in out: G is NaN in the pixel, and all that follows from it
    res = quan.quan_residual_backward(y, do, out=with_nan(out), dh=dh, **kw)
    check_pixel(res.dx, clean.dx, "dx")
    assert bool(res.dnext_gamma.isnan().all())
    if p == 0.0:
        for name in ("dgamma", "dscale"):
            assert bool(getattr(res, name).isnan().all()), name
    # a NaN in y: the norm's statistic is, so every channel's gradient
    res = quan.quan_residual_backward(with_nan(y), do, out=out, dh=dh, **kw)
    check_pixel(res.dy, clean.dy, "dy")
    assert torch.equal(res.dx, clean.dx) and torch.equal(res.dnext_gamma, clean.dnext_gamma)
    if p == 0.0:
        for name in ("dgamma", "dscale"):
            assert bool(getattr(res, name).isnan().all()), name
        assert bool(res.dgate[1].isnan().all()) and torch.equal(res.dgate[0], clean.dgate[0])
