"""The attention block that runs the operators together: its output and every
gradient against torch's differentiation of the same formulas in 64 bits on the
CPU, its single pixels against its whole maps."""
import math

import pytest
import torch

from block_reference import drop_factors
from parity import say
from paper_2509_05512_amd import quan
from paper_2509_05512_amd.attention_block import AttentionBlock, Stack, train

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
SIGN = ((1, -1, -1, -1), (1, 1, -1, 1), (1, 1, 1, -1), (1, -1, 1, 1))  # of W_(p xor q) x_q in component p

# Bars on |got - ref| / |ref| (2-norms).  bf16: the chain of two blocks rounds
# each of its ~20 maps once, 2^-9 of a value in the mean; were all of them off
# the same way, 20 x 2^-9 = 0.04 (a gradient of a sum of many of them less).
# fp32: the same with the 2^-24 of its roundings and of sums of up to 1000
# terms (20 x 1000^(1/2) x 2^-24 = 4e-5).
BAR = {BF: 0.04, F32: 4e-5}


def rand_map(seed, *shape, dtype):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


def up(t):
    return quan.to_device_layout(t.cuda())


def hamilton(w, x):
    """w [4, O, C, 1, 1] (x) x [N, 4, C, H, W]"""
    parts = []
    for p in range(4):
        terms = [SIGN[p][q] * torch.einsum("oc,nchw->nohw", w[p ^ q, :, :, 0, 0], x[:, q]) for q in range(4)]
        parts.append(sum(terms))
    return torch.stack(parts, 1)


def norm(x, g):
    return x / torch.sqrt(x.square().mean((1, 2), keepdim=True) + 1e-6) * g[None, :, :, None, None]


def attention(q, k, v, heads, table, bucket):
    n, _, c, h, w = q.shape
    dq = c // heads
    kv = k.shape[2] // dq

    def split(t, count):
        return t.reshape(n, 4, count, dq, h * w).permute(0, 2, 4, 1, 3).reshape(n, count, h * w, 4 * dq)

    Q = split(q, heads)
    K, V = (split(t, kv).repeat_interleave(heads // kv, 1) for t in (k, v))
    ys, xs = torch.arange(h * w) // w, torch.arange(h * w) % w
    r = bucket.numel() // 2
    by, bx = (bucket[(s[None, :] - s[:, None]).clamp(-r, r) + r].long() for s in (ys, xs))
    s = Q @ K.transpose(-1, -2) / math.sqrt(4 * dq) + table[:, by, bx]
    o = torch.softmax(s, -1) @ V
    return o.reshape(n, heads, h * w, 4, dq).permute(0, 3, 1, 4, 2).reshape(n, 4, c, h, w)


def reference(stack, leaves, x, factors):
    """The stack in 64 bits on leaves = [norm_in, params of each block]."""
    h = norm(x, leaves[0])
    for block, at, keep in zip(stack.blocks, leaves[1:], factors):
        c, kv = block.c, block.kv
        qkv = hamilton(at["qkv"], h)
        a = attention(qkv[:, :, :c], qkv[:, :, c:c + kv], qkv[:, :, c + kv:], block.heads, at["table"],
                      block.bucket.cpu())
        y = hamilton(at["proj"], a)
        x = x + at["scale"][None, :, :, None, None] * keep * norm(y, at["gamma"])
        h = norm(x, at["next_gamma"]) if "next_gamma" in at else None
    return x


def close(got, ref, dtype, what):
    off = float((got.double().cpu() - ref).norm() / ref.norm())
    assert off <= BAR[dtype], f"{what}: {off:.3g} of its norm off"


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("shape", [(2, 16, 5, 7, 4, 4), (1, 24, 9, 9, 4, 2), (3, 8, 1, 33, 2, 1), (2, 32, 8, 8, 2, 2)],
                         ids=str)
def test_output_and_gradients(shape, dtype):
    n, c, height, width, heads, kv = shape
    say(f"stack {shape} {dtype}")
    p = 0.2
    stack = Stack(2, c, heads, kv_heads=kv, radius=4, buckets=7, p=p, dtype=dtype, seed=5)
    x, dout = rand_map(1, n, 4, c, height, width, dtype=dtype), rand_map(2, n, 4, c, height, width, dtype=dtype)
    rngs = [torch.tensor([11, i], dtype=torch.int64, device="cuda") for i in range(2)]
    out, saved = stack.forward(up(x), rngs, save=True)
    dx, dnorm, grads = stack.backward(saved, up(dout))

    def leaf(t):
        return t.detach().double().cpu().requires_grad_()

    ref_x = leaf(x)
    leaves = [leaf(stack.norm_in)] + [{name: leaf(b.kernels.get(name, t)) for name, t in b.params.items()}
                                      for b in stack.blocks]
    factors = [torch.from_numpy(drop_factors(n, c, height, width, p, 11, i)) for i in range(2)]
    ref = reference(stack, leaves, ref_x, factors)
    ref.backward(dout.double())
    close(out, ref.detach(), dtype, "out")
    close(dx, ref_x.grad, dtype, "dx")
    close(dnorm, leaves[0].grad, dtype, "dnorm_in")
    for i, g in enumerate(grads):
        assert set(g) == set(stack.blocks[i].params)
        for name, value in g.items():
            close(value, leaves[1 + i][name].grad, dtype, f"block {i}'s d{name}")


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
def test_single_pixels_are_the_whole_maps(dtype):
    """The same operators on one query and on whole maps: apart by roundings."""
    n, c, side, heads = 3, 32, 6, 4
    block = AttentionBlock(c, heads, kv_heads=2, radius=3, buckets=7, dtype=dtype, seed=9)
    x = up(rand_map(3, n, 4, c, side, side, dtype=dtype))
    h = quan.quan_rmsnorm_forward(x, torch.ones((4, c), device="cuda"))
    gate = up(rand_map(4, n, 4, c, 1, 1, dtype=dtype))
    whole = block.forward(x, h, gate=gate)
    cache = block.cache(n, side, side)
    for row in (0, 2, 4):
        block.write(cache, quan.to_device_layout(h[..., row:row + 2, :]), row)
    there = torch.full((n,), side * side, dtype=torch.int32, device="cuda")
    for at_y, at_x in ((0, 0), (5, 2), (3, 5)):
        say(f"pixel {at_y} {at_x} {dtype}")
        px, ph = (quan.to_device_layout(t[..., at_y:at_y + 1, at_x:at_x + 1]) for t in (x, h))
        pos = torch.tensor([[at_y, at_x]] * n, dtype=torch.int32, device="cuda")
        for got, ref in zip(block.query(cache, px, ph, pos, kv_len=there, gate=gate), whole):
            close(got, ref[..., at_y:at_y + 1, at_x:at_x + 1].double().cpu(), dtype, "pixel")


def test_training_lowers_the_loss():
    stack = Stack(2, 16, 2, radius=4, buckets=5, p=0.1, dtype=BF, seed=1)
    x, target = (up(rand_map(s, 4, 4, 16, 6, 6, dtype=BF)) for s in (5, 6))
    losses = train(stack, x, target, steps=20, rate=5.0)
    assert losses[-1] < 0.95 * losses[0], losses


def test_refusals():
    with pytest.raises(ValueError):
        AttentionBlock(30, 4)
    with pytest.raises(ValueError):
        AttentionBlock(32, 4, kv_heads=3)
    block = AttentionBlock(16, 2)
    x = up(rand_map(1, 1, 4, 16, 2, 2, dtype=BF))
    with pytest.raises(ValueError):
        block.forward(x, up(rand_map(1, 1, 4, 8, 2, 2, dtype=BF)))
