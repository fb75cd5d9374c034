"""A query's place far outside the keys' map, to the ends of its type: offsets
beyond the radius take the end's bucket."""
import numpy as np
import pytest
import torch

from block_reference import attention, check
from parity import f64, say
from paper_2509_05512_amd import quan

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def rand_map(seed, n, c, h, w):
    g = torch.Generator().manual_seed(seed)
    return torch.randn((n, h, w, 4, c), generator=g).to(BF).permute(0, 3, 4, 1, 2)


@pytest.mark.parametrize("hq,wq", [(1, 1), (5, 6)])
def test_places_at_the_ends_of_int32(hq, wq):
    say(f"places at the ends of int32 {hq} {wq}")
    low, high = -2 ** 31, 2 ** 31 - 1
    pos = torch.tensor([[low, 0], [high, 0], [0, low], [0, high], [low, high], [low + 3, high - 3], [1 << 30, -(1 << 30)]],
                       dtype=torch.int32)
    n, heads, dq, h, w = len(pos), 2, 8, 7, 9
    q, do = (rand_map(s, n, heads * dq, hq, wq) for s in (1, 4))
    k, v = (rand_map(s, n, heads * dq, h, w) for s in (2, 3))
    by, bx = (quan.quan_relpos_buckets(4, 5) for _ in range(2))
    table = 3.0 * torch.randn((heads, 5, 5), generator=torch.Generator().manual_seed(5))
    qd, kd, vd, dod = (quan.to_device_layout(t.cuda()) for t in (q, k, v, do))
    kw = dict(relpos=(table.cuda(), by.cuda(), bx.cuda()), pos=pos.cuda())
    out, stats, rest = quan.quan_attention_forward(qd, kd, vd, heads, save=True, **kw)
    grads = quan.quan_attention_backward(qd, kd, vd, out, stats, rest, dod, heads, **kw)
    # (one bucket per query and image: any place as far out is the same)
    near = pos.clamp(-1000, 1000).numpy()
    ref, err = attention(f64(q), f64(k), f64(v), heads, table.numpy().astype(np.float64), by.numpy(), bx.numpy(),
                         pos=near, dout=f64(do))
    for name, got in zip(("out", "dq", "dk", "dv", "dtable"), (out, *grads)):
        check(f64(got), ref[name], err[name], True, name)
