"""What a training step in bf16 keeps beyond its outputs' rounding: out and rest
are the fp32 results, and the bias's gradient, fp32, is as far off as fp32 is
(1e-5 of the largest sum of a result's terms, the other operators' slack)."""
import numpy as np
import pytest
import torch

from block_reference import F32 as SLACK
from block_reference import attention, check
from parity import f64, say
from paper_2509_05512_amd import quan

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def rand_map(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(BF)


# one query, a few keys, odd channels, keys dealt out to work-groups, shared heads
@pytest.mark.parametrize("n,q_hw,k_hw,heads,kv_heads,dq", [
    (3, (1, 1), (9, 11), 4, 2, 16), (2, (2, 3), (2, 3), 1, 1, 16), (2, (7, 5), (7, 5), 2, 1, 5),
    (1, (1, 700), (1, 700), 2, 2, 8), (2, (12, 13), (12, 13), 4, 2, 32)])
@pytest.mark.parametrize("scale", [None, 2.0])  # (2: rows of few large probabilities)
def test_out_and_rest_are_fp32(n, q_hw, k_hw, heads, kv_heads, dq, scale):
    say(f"rest {n} {q_hw} {k_hw} {heads} {kv_heads} {dq} {scale}")
    q, do = (rand_map(s, n, 4, heads * dq, *q_hw) for s in (1, 2))
    k, v = (rand_map(s, n, 4, kv_heads * dq, *k_hw) for s in (3, 4))
    by, bx = (quan.quan_relpos_buckets(max(a, b) - 1, 5) for a, b in zip(q_hw, k_hw))
    table = torch.randn((heads, 5, 5), generator=torch.Generator().manual_seed(5))
    rp = tuple(t.cuda() for t in (table, by, bx))
    qd, kd, vd, dod = (quan.to_device_layout(t.cuda()) for t in (q, k, v, do))
    out, stats, rest = quan.quan_attention_forward(qd, kd, vd, heads, relpos=rp, scale=scale, save=True)
    dtable = quan.quan_attention_backward(qd, kd, vd, out, stats, rest, dod, heads, relpos=rp, scale=scale)[3]

    ref, err = attention(f64(q), f64(k), f64(v), heads, table.numpy().astype(np.float64), by.numpy(), bx.numpy(),
                         scale=scale, dout=f64(do))
    high, low = (t.cpu().view(torch.int16).to(torch.int64) for t in (out, rest))
    whole = ((high << 16) + low).to(torch.int32).view(torch.float32)
    assert float((whole.double().numpy() - ref["out"]).__abs__().max()) <= SLACK * float(f64(v).__abs__().max())
    assert torch.equal(whole.to(BF), out.cpu())  # (rounded, they are out)
    check(f64(dtable), ref["dtable"], err["dtable"], False, "dtable")
