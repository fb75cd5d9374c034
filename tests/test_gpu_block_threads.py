"""Two host threads on one stream, each with calls of the attention block that
hand data from one launch to the next through the stream's buffers (copies, sums
by offset, shared walks, sums by image): every result has the bits that one
thread gets."""
import threading

import pytest
import torch

from parity import say
from paper_2509_05512_amd import quan

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def rand_map(seed, n, c, h, w, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn((n, h, w, 4, c), generator=g, device="cuda").to(dtype).permute(0, 3, 4, 1, 2)


def attention(seed, n, h, w, heads, dq, dtype):
    q, k, v, do = (rand_map(seed + i, n, heads * dq, h, w, dtype) for i in range(4))
    by, bx = (quan.quan_relpos_buckets(r - 1, 8, "cuda") for r in (h, w))
    relpos = (torch.randn((heads, 8, 8), generator=torch.Generator().manual_seed(seed)).cuda(), by, bx)

    def call():
        out, stats, rest = quan.quan_attention_forward(q, k, v, heads, relpos=relpos, save=True)
        return (out, quan.quan_attention_forward(q[..., :1, :1], k, v, heads, relpos=relpos),
                *quan.quan_attention_backward(q, k, v, out, stats, rest, do, heads, relpos=relpos))
    return call


def residual(seed, n, h, w, c, dtype):
    y, do, o, dh = (rand_map(seed + i, n, c, h, w, dtype) for i in range(4))
    gamma, scale, following = (rand_map(seed + 4 + i, 1, c, 1, 1, F32)[0, :, :, 0, 0].contiguous() for i in range(3))
    gate = rand_map(seed + 7, n, c, 1, 1, dtype)
    rng = torch.tensor([seed, 1], dtype=torch.int64, device="cuda")

    def call():
        return tuple(quan.quan_residual_backward(y, do, gamma=gamma, gate=gate, scale=scale, next_gamma=following, out=o,
                                                 dh=dh, p=0.2, rng=rng))
    return call


def test_two_threads_on_one_stream():
    say("two threads on one stream")
    calls = [attention(1, 2, 16, 16, 2, 5, F32), residual(11, 3, 9, 11, 37, BF), attention(21, 1, 40, 31, 4, 16, BF),
             residual(31, 5, 30, 30, 64, BF), attention(41, 6, 20, 21, 3, 12, BF), residual(51, 2, 5, 5, 300, F32)]
    want = [call() for call in calls]
    torch.cuda.synchronize()
    got, failed = {0: [], 1: []}, []

    def run(tag):
        try:
            for _ in range(20):
                for i in (range(len(calls)) if tag == 0 else reversed(range(len(calls)))):
                    got[tag].append((i, calls[i]()))
        except Exception as e:  # noqa: BLE001
            failed.append(repr(e))

    threads = [threading.Thread(target=run, args=(t,)) for t in (0, 1)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed, failed
    for tag in got:
        assert len(got[tag]) == 20 * len(calls)
        for i, results in got[tag]:
            assert all(torch.equal(a, b) for a, b in zip(results, want[i])), f"thread {tag}, call {i}"
