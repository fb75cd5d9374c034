"""The bias's gradient is linear in dout over the type's range: a power of two
times dout, whose squares are beyond fp32, gives that power times the gradient
to the bit (every step of it is linear in dout, and rounds alike)."""
import pytest
import torch

from parity import say
from paper_2509_05512_amd import quan

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def rand_map(seed, n, c, h, w, dtype):
    g = torch.Generator().manual_seed(seed)
    return torch.randn((n, h, w, 4, c), generator=g).to(dtype).cuda().permute(0, 3, 4, 1, 2)


def gradient(q, k, v, dout, heads, relpos):
    out, stats, rest = quan.quan_attention_forward(q, k, v, heads, relpos=relpos, save=True)
    return quan.quan_attention_backward(q, k, v, out, stats, rest, dout, heads, relpos=relpos)[3]


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("dq", [8, 32])
@pytest.mark.parametrize("power", [-84, -80, -66, 64, 70])
def test_small_and_large_dout(power, dq, dtype):
    """Scores of 0 and values in pairs v, -v: rows' sums of dout out cancel, so
    that dS is all dP.  Terms are 2^power x 1 .. 1000, far from the type's ends."""
    say(f"dout of 2^{power} {dq} {dtype}")
    heads, length = 2, 16
    q = torch.zeros((1, 1, length, 4, heads * dq), dtype=dtype, device="cuda").permute(0, 3, 4, 1, 2)
    k = rand_map(1, 1, heads * dq, 1, length, dtype)
    v = 64.0 * rand_map(2, 1, heads * dq, 1, length, dtype)
    v[..., length // 2:] = -v[..., :length // 2]
    do = rand_map(3, 1, heads * dq, 1, length, dtype)
    relpos = (torch.zeros((heads, 1, 9), device="cuda"), None, quan.quan_relpos_buckets(4, 9, "cuda"))
    want = gradient(q, k, v, do, heads, relpos)
    assert bool(want.isfinite().all()) and float(want.abs().max()) > 1
    got = gradient(q, k, v, do * 2.0 ** power, heads, relpos)
    assert torch.equal(got, want * 2.0 ** power)
