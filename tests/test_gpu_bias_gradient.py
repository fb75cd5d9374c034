"""The bias's gradient is its sums alone: nothing that earlier calls left in the
stream's workspace reaches it."""
import numpy as np
import pytest
import torch

from block_reference import attention, check
from parity import f64, say
from paper_2509_05512_amd import quan

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def rand_map(seed, n, c, h, w, dtype):
    g = torch.Generator().manual_seed(seed)
    return torch.randn((n, h, w, 4, c), generator=g).to(dtype).permute(0, 3, 4, 1, 2)


def leave_behind(value):
    """Calls of `value` everywhere whose copies of the maps (heads of 5 channels
    are padded to 8) fill the first 65 MB of the workspace."""
    x = torch.full((256, 1, 700, 4, 5), value, dtype=BF, device="cuda").permute(0, 3, 4, 1, 2)
    out, stats, rest = quan.quan_attention_forward(x, x, x, 1, save=True)
    rest.fill_(value)
    quan.quan_attention_backward(x, x, x, x, stats, rest, x, 1)


def step(q, k, v, do, heads, relpos):
    out, stats, rest = quan.quan_attention_forward(q, k, v, heads, relpos=relpos, save=True)
    return out, stats, rest, (lambda: quan.quan_attention_backward(q, k, v, out, stats, rest, do, heads, relpos=relpos)[3])


# maps whose last blocks of queries have fewer offsets to a row of keys than the
# next row lies ahead; n * heads * blocks of 128 queries >= 256, so that a
# work-group walks over all keys
@pytest.mark.parametrize("dtype,h,w", [(BF, 66, 66), (BF, 68, 68), (BF, 69, 69), (BF, 17, 92), (BF, 19, 96),
                                       (F32, 17, 68), (F32, 34, 68), (F32, 76, 76)], ids=str)
def test_offsets_that_a_block_has_not(dtype, h, w):
    say(f"offsets between rows of keys {dtype} {h} {w}")
    heads, dq, blocks = 8, 8, (h * w + 127) // 128
    n = -(-256 // (heads * blocks))
    q, k, v, do = (quan.to_device_layout(rand_map(s, n, heads * dq, h, w, dtype).cuda()) for s in (1, 2, 3, 4))
    b = [quan.quan_relpos_buckets(r - 1, 16, "cuda") for r in (h, w)]
    relpos = (torch.randn((heads, 16, 16), generator=torch.Generator().manual_seed(5)).cuda(), *b)
    *_, gradient = step(q, k, v, do, heads, relpos)
    got = []
    for value in (0.0, float("nan"), 1e30):
        leave_behind(value)
        got.append(gradient())
    assert bool(got[0].isfinite().all())
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])


def test_offsets_that_a_block_has_not_against_the_formula():
    say("offsets between rows of keys, formula")
    n, heads, dq, h, w = 2, 13, 2, 17, 68
    q, k, v, do = (rand_map(s, n, heads * dq, h, w, F32) for s in (1, 2, 3, 4))
    by, bx = (quan.quan_relpos_buckets(r - 1, 7) for r in (h, w))
    table = torch.randn((heads, 7, 7), generator=torch.Generator().manual_seed(5))
    up = [quan.to_device_layout(t.cuda()) for t in (q, k, v, do)]
    *_, gradient = step(*up, heads, (table.cuda(), by.cuda(), bx.cuda()))
    leave_behind(1e30)
    ref, err = attention(f64(q), f64(k), f64(v), heads, table.numpy().astype(np.float64), by.numpy(), bx.numpy(),
                         dout=f64(do))
    check(f64(gradient()), ref["dtable"], err["dtable"], False, "dtable")
