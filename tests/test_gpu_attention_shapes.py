"""Maps of queries that are narrow where the keys' are wide and the reverse, up
to where a tile's offsets fill a work-group's LDS."""
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


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("q_hw,k_hw,dq", [((8, 8), (4, 512), 32), ((90, 1), (50, 60), 8), ((140, 1), (33, 70), 8),
                                          ((33, 70), (140, 1), 8), ((5, 600), (16, 8), 16), ((16, 4), (5, 250), 16),
                                          ((1, 300), (9, 11), 8), ((2, 150), (4, 3), 5)], ids=str)
def test_narrow_and_wide(q_hw, k_hw, dq, dtype):
    say(f"narrow and wide {q_hw} {k_hw} {dq} {dtype}")
    heads = 2
    q, do = (rand_map(s, 1, heads * dq, *q_hw, dtype) for s in (1, 4))
    k, v = (rand_map(s, 1, heads * dq, *k_hw, dtype) for s in (2, 3))
    by, bx = (quan.quan_relpos_buckets(max(a, b) - 1, 9) for a, b in zip(q_hw, k_hw))
    table = torch.randn((heads, 9, 9), generator=torch.Generator().manual_seed(5))
    pos = torch.tensor([[1, 3]], dtype=torch.int32)
    kw = dict(relpos=(table.cuda(), by.cuda(), bx.cuda()), pos=pos.cuda())
    qd, kd, vd, dod = (quan.to_device_layout(t.cuda()) for t in (q, k, v, do))
    out, stats, rest = quan.quan_attention_forward(qd, kd, vd, heads, save=True, **kw)
    grads = quan.quan_attention_backward(qd, kd, vd, out, stats, rest, dod, heads, **kw)
    ref, err = attention(f64(q), f64(k), f64(v), heads, table.numpy().astype(np.float64), by.numpy(), bx.numpy(),
                         pos=pos.numpy(), dout=f64(do))
    for name, got in zip(("out", "dq", "dk", "dv", "dtable"), (out, *grads)):
        check(f64(got), ref[name], err[name], dtype == BF, name)
