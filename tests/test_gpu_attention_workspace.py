"""What the attention's backward pass holds in its stream's workspace, and that
smaller batches of a captured step fit into what a larger one left."""
import pytest
import torch

from parity import say
from paper_2509_05512_amd import quan

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def rand_map(seed, n, c, h, w, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn((n, h, w, 4, c), generator=g, device="cuda").to(dtype).permute(0, 3, 4, 1, 2)


def bias(heads, radius, buckets):
    table = torch.randn((heads, 1, buckets), generator=torch.Generator().manual_seed(5)).cuda()
    return table, None, quan.quan_relpos_buckets(radius, buckets, "cuda")


def test_one_query_and_many_keys():
    """65536 keys: their 512 shares have sums by offset of their own keys, 0.5
    MB together, beside 8 MB of partial gradients (and torch's small blocks)."""
    say("workspace of one query against many keys")
    heads, dq, length = 1, 8, 65536
    q, do = (rand_map(s, 1, heads * dq, 1, 1, BF) for s in (1, 4))
    k, v = (rand_map(s, 1, heads * dq, 1, length, BF) for s in (2, 3))
    kw = dict(relpos=bias(heads, 128, 32), pos=torch.tensor([[0, length - 1]], dtype=torch.int32, device="cuda"))
    out, stats, rest = quan.quan_attention_forward(q, k, v, heads, save=True, **kw)
    dq_, dk, dv = (torch.empty_like(t) for t in (q, k, v))
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    before = torch.cuda.mem_get_info()[0]
    with torch.cuda.stream(st):
        quan.quan_attention_backward(q, k, v, out, stats, rest, do, heads, dq=dq_, dk=dk, dv=dv, **kw)
    torch.cuda.synchronize()
    held = before - torch.cuda.mem_get_info()[0]
    say(f"{held / 1e6:.1f} MB")
    assert held <= 32e6


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("hq,wq,hk,wk,heads", [(20, 21, 20, 21, 3), (1, 3, 1, 2000, 2), (1, 300, 40, 30, 1), (16, 16, 16, 16, 2)])
def test_captured_smaller_batches(hq, wq, hk, wk, heads, dtype):
    """Batches from 1 up, captured after the largest has run, whose keys are
    dealt out to other numbers of work-groups: every replay has an eager step's
    bits, beside eager steps of the other batches."""
    say(f"smaller batches {hq} {wq} {hk} {wk} {heads} {dtype}")
    most, dq = 7, 8
    q, do = (rand_map(s, most, heads * dq, hq, wq, dtype) for s in (1, 4))
    k, v = (rand_map(s, most, heads * dq, hk, wk, dtype) for s in (2, 3))
    by, bx = (quan.quan_relpos_buckets(max(a, b) - 1, 9, "cuda") for a, b in ((hq, hk), (wq, wk)))
    relpos = (torch.randn((heads, 9, 9), generator=torch.Generator().manual_seed(5)).cuda(), by, bx)

    def gradients(n, saved):
        out, stats, rest = saved
        return quan.quan_attention_backward(q[:n], k[:n], v[:n], out, stats, rest, do[:n], heads, relpos=relpos)

    saved = {n: quan.quan_attention_forward(q[:n], k[:n], v[:n], heads, relpos=relpos, save=True)
             for n in range(1, most + 1)}
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        gradients(most, saved[most])
    torch.cuda.synchronize()
    graphs = {}
    for n in (1, 2, 3, 5):
        graphs[n] = (torch.cuda.CUDAGraph(), None)
        with torch.cuda.graph(graphs[n][0], stream=st):
            graphs[n] = (graphs[n][0], gradients(n, saved[n]))
    for rep in range(2):
        for n, (graph, held) in graphs.items():
            do.copy_(rand_map(10 + rep, most, heads * dq, hq, wq, dtype))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            with torch.cuda.stream(st):
                gradients(most, saved[most])
                want = gradients(n, saved[n])
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(held, want)), n


def test_captured_smaller_batch_in_slices():
    """16 images whose sums go to their buckets directly, then 15, dealt out to
    twice the work-groups, whose sums go through slices of the images."""
    say("smaller batch in slices")
    most, n, heads, dq, h, w = 16, 15, 16, 8, 8, 16
    q, k, v, do = (rand_map(s, most, heads * dq, h, w, F32) for s in (1, 2, 3, 4))
    by, bx = (quan.quan_relpos_buckets(r - 1, 9, "cuda") for r in (h, w))
    relpos = (torch.randn((heads, 9, 9), generator=torch.Generator().manual_seed(5)).cuda(), by, bx)
    saved = [quan.quan_attention_forward(q[:m], k[:m], v[:m], heads, relpos=relpos, save=True) for m in (most, n)]

    def gradients(m, kept):
        return quan.quan_attention_backward(q[:m], k[:m], v[:m], *kept, do[:m], heads, relpos=relpos)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        gradients(most, saved[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        held = gradients(n, saved[1])
    for rep in range(3):
        do.copy_(rand_map(10 + rep, most, heads * dq, h, w, F32))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            gradients(most, saved[0])
            want = gradients(n, saved[1])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want))


def test_large_maps_in_turns():
    """96 heads of 160 x 160, whose sums by offset would take 3.9 GB: they are
    taken in turns, and the results are those of the images one by one."""
    say("sums by offset in turns")
    n, heads, h, w, dq = 3, 32, 160, 160, 8
    q, k, v, do = (rand_map(s, n, heads * dq, h, w, BF) for s in (1, 2, 3, 4))
    b = quan.quan_relpos_buckets(159, 16, "cuda")
    relpos = (torch.randn((heads, 16, 16), generator=torch.Generator().manual_seed(5)).cuda(), b, b)

    def step(i0, i1):
        q_, k_, v_, do_ = (t[i0:i1] for t in (q, k, v, do))
        out, stats, rest = quan.quan_attention_forward(q_, k_, v_, heads, relpos=relpos, save=True)
        grads = dict(zip(("dq", "dk", "dv"), (torch.empty_like(t) for t in (q_, k_, v_))))
        return lambda: quan.quan_attention_backward(q_, k_, v_, out, stats, rest, do_, heads, relpos=relpos, **grads)
    one = [step(i, i + 1)() for i in range(n)]
    call = step(0, n)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    before = torch.cuda.mem_get_info()[0]
    with torch.cuda.stream(st):
        got = call()
    torch.cuda.synchronize()
    held = before - torch.cuda.mem_get_info()[0]
    say(f"{held / 1e6:.1f} MB")
    # 2 GiB, 26 MB of sums, 25 of parts, 10 of rows, and a quarter of all; torch's small blocks
    assert held <= 2.85e9
    for i, each in enumerate(one):
        for name, a, e in zip(("dq", "dk", "dv"), got, each):
            assert torch.equal(a[i:i + 1], e), (name, i)
    parts = torch.stack([e[3] for e in one]).double()
    # (each rounded once to fp32, from sums that differ by fp64's rounding)
    off = (got[3].double() - parts.sum(0)).abs()
    assert bool((off <= 2.0 ** -23 * (parts.abs().sum(0) + got[3].double().abs())).all())
