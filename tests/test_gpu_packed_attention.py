"""Causal attention of packed sequences on the GPU, forward and backward."""
import numpy as np
import pytest
import torch

import sequence_reference as ref
from parity import say
from paper_2509_05512_amd import quan
from test_gpu_cache import BF, DEV, F32, ints, rand_map

pytestmark = pytest.mark.gpu


def rows(t, heads):
    return ref.rows_of(t.float().cpu().numpy().astype(np.float64), heads)


def step(q, k, v, do, first, heads, **kw):
    out, saved = quan.quan_packed_attention_forward(q, k, v, first, heads, save=True, **kw)
    grads = quan.quan_packed_attention_backward(q, k, v, out, saved, do, first, heads, **kw)
    return (out, saved.stats, *grads)


def compare(q, k, v, do, lq, lk, heads, got, what, causal=True, scale=None, q0=0, k0=0, score=0.0):
    """Against the reference; tokens of no sequence are not looked at.  score: the
    rounding of the scores where they are large."""
    dq = q.shape[2] // heads
    kvh = k.shape[2] // dq
    z, y = slice(q0, q0 + sum(lq)), slice(k0, k0 + sum(lk))
    want, err = ref.packed(rows(q, heads)[z], rows(k, kvh)[y], rows(v, kvh)[y], lq, lk, causal, scale, rows(do, heads)[z])
    err = {m: (a, b * (1.0 + 4.0 * score / ref.F32)) for m, (a, b) in err.items()}
    out, stats, dqs, dks, dvs = got
    bf = q.dtype == BF
    ref.check(rows(out, heads)[z], want["out"], err["out"], bf, what + " out")
    top, total = (stats[:, z, i].double().cpu().numpy().T for i in range(2))
    with np.errstate(divide="ignore"):
        lse = np.log(2) * top + np.log(total)
    there = np.isfinite(want["lse"])
    assert np.array_equal(np.isfinite(lse), there), what
    assert np.all(np.abs(lse[there] - want["lse"][there]) <= 1e-4 + score), what
    ref.check(rows(dqs, heads)[z], want["dq"], err["dq"], bf, what + " dq")
    ref.check(rows(dks, kvh)[y], want["dk"], err["dk"], bf, what + " dk")
    ref.check(rows(dvs, kvh)[y], want["dv"], err["dv"], bf, what + " dv")


LENS = {
    "mixed": ([0, 1, 2, 31, 0, 33, 64, 65, 127, 0], None),
    "long": ([300, 129, 128], None),
    "one": ([1], None),
    "past": ([3, 70, 1, 130, 0], [40, 200, 129, 131, 7]),
    "less": ([70, 5, 200, 3], [3, 0, 150, 3]),
}


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("dq,heads,kv_heads", [(16, 4, 2), (8, 3, 3), (32, 2, 1), (5, 2, 2), (12, 8, 1), (1, 1, 1)])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "all"])
def test_packed(dtype, lens, dq, heads, kv_heads, causal):
    say(f"packed {dtype} {lens} dq {dq} heads {heads}/{kv_heads} causal {causal}")
    lq, lk = LENS[lens]
    same = lk is None
    lk = lq if same else lk
    c, ckv = heads * dq, kv_heads * dq
    if same:  # slices of one map
        qkv = rand_map(1, 1, c + 2 * ckv, 1, sum(lq), dtype)
        q, k, v = qkv[:, :, :c], qkv[:, :, c:c + ckv], qkv[:, :, c + ckv:]
    else:
        q = rand_map(1, 1, c, 1, sum(lq), dtype)
        k, v = (rand_map(s, 1, ckv, 1, max(1, sum(lk)), dtype) for s in (2, 3))
    do = rand_map(4, 1, c, 1, sum(lq), dtype)
    kw = dict(k_first=None if same else ints(ref.starts(lk).tolist()), causal=causal)
    got = step(q, k, v, do, ints(ref.starts(lq).tolist()), heads, **kw)
    compare(q, k, v, do, lq, lk, heads, got, lens, causal)
    again = step(q, k, v, do, ints(ref.starts(lq).tolist()), heads, **kw)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
def test_images(dtype):
    """A sequence per image, pixels in row order; a scale of the caller's."""
    say(f"packed images {dtype}")
    n, heads, dq = 3, 2, 16
    q, k, v, do = (rand_map(s, n, heads * dq, 9, 15, dtype) for s in range(4))
    got = step(q, k, v, do, None, heads, scale=0.2)
    compare(q, k, v, do, [135] * n, [135] * n, heads, got, "images", scale=0.2)
    q, do = (rand_map(s, n, heads * dq, 1, 10, dtype) for s in (5, 6))
    got = step(q, k, v, do, None, heads)
    compare(q, k, v, do, [10] * n, [135] * n, heads, got, "images, few queries")


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
def test_long_sequences(dtype):
    """Walks that work-groups share, beside short ones."""
    say(f"packed, long walks {dtype}")
    heads, dq = 2, 16
    for lq, lk in (([130, 3], [2000, 900]), ([1100, 40], [1100, 40])):
        q, do = (rand_map(s, 1, heads * dq, 1, sum(lq), dtype) for s in (1, 2))
        k, v = (rand_map(s, 1, dq, 1, sum(lk), dtype) for s in (3, 4))
        first, k_first = (ints(ref.starts(t).tolist()) for t in (lq, lk))
        compare(q, k, v, do, lq, lk, heads, step(q, k, v, do, first, heads, k_first=k_first), f"{lq} on {lk}")


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("dq", [16, 12])
def test_tokens_of_no_sequence(dtype, dq):
    """Before the first and behind the last sequence: NaN there is not read, and
    what is there in the results stays."""
    say(f"packed, tokens of no sequence {dtype} {dq}")
    heads, lens, before, behind = 2, [70, 0, 130], 5, 9
    total = before + sum(lens) + behind
    q, k, v, do = (rand_map(s, 1, heads * dq, 1, total, dtype) for s in range(4))
    for t in (q, k, v, do):
        t[..., :before] = float("nan")
        t[..., before + sum(lens):] = float("nan")
    first = ints((ref.starts(lens) + before).tolist())
    out, g = (torch.full_like(q, 3.0) for _ in range(2))
    grads = [torch.full_like(q, 3.0) for _ in range(3)]
    out, saved = quan.quan_packed_attention_forward(q, k, v, first, heads, out=out, save=True)
    quan.quan_packed_attention_backward(q, k, v, out, saved, do, first, heads, dq=grads[0], dk=grads[1], dv=grads[2])
    compare(q, k, v, do, lens, lens, heads, (out, saved.stats, *grads), "inside", q0=before, k0=before)
    for t in (out, *grads):
        assert bool((t[..., :before] == 3.0).all()) and bool((t[..., before + sum(lens):] == 3.0).all())


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_masked_infinities_and_nan(dtype, bad):
    """What a query does not see leaves its result and gradient within the bounds
    that they have without it, and so it is with a key's gradients and queries that do
    not see it; other sequences keep every bit.  (Tiles that hold such a number at a
    walk's edge are taken row by row, where nothing is rounded to bf16 between the
    products: the same terms with fewer roundings than the bounds count.)"""
    say(f"packed, masked {bad} {dtype}")
    heads, dq, lens, at = 2, 16, [200, 40], 77
    q, k, v, do = (rand_map(s, 1, heads * dq, 1, sum(lens), dtype) for s in range(4))
    first = ints(ref.starts(lens).tolist())
    clean = step(q, k, v, do, first, heads)
    want, err = ref.packed(*(rows(t, heads) for t in (q, k, v)), lens, lens, dout=rows(do, heads))
    names = {0: "out", 2: "dq", 3: "dk", 4: "dv"}

    def within(got, i, z, what):
        name = names[i]
        ref.check(rows(got[i], heads)[z], want[name][z], (err[name][0][z], err[name][1]), dtype == BF, f"{what} {name}")
    for which in range(4):
        maps = [t.clone(memory_format=torch.preserve_format) for t in (q, k, v, do)]
        maps[which][0, 1, 3, 0, at] = bad
        got = step(*maps, first, heads)
        before, behind = slice(0, at), slice(at + 1, 200)
        for i in (0, 2):
            within(got, i, before, f"before {which}")
            if which in (0, 3):  # a query or its gradient reaches its own row alone
                within(got, i, behind, f"behind {which}")
        if which in (0, 3):  # and the keys before it
            for i in (3, 4):
                within(got, i, behind, f"behind {which}")
        if which == 2:
            assert not bool(torch.isfinite(got[0][0, 1, 3, 0, at:200]).any())
        for i in names:
            assert torch.equal(got[i][..., 200:], clean[i][..., 200:]), (which, i)


def test_sequences_out_of_order():
    """Values that descend or lie beyond the map reach no other memory."""
    say("packed, sequences out of order")
    heads, dq, total = 2, 8, 300
    room = torch.full((5, 3 * total, 4, heads * dq), 3.0, dtype=BF, device=DEV)
    q, k, v, do = (rand_map(s, 1, heads * dq, 1, total, BF) for s in range(4))
    out, a, b, c = (room[i, total:2 * total][None, None].permute(0, 3, 4, 1, 2) for i in range(4))
    for first in ([200, 100, 300, 0], [-7, 1000, 3, 2147483647], [-2147483648, 128, 128, 300], [301, 302, 400, 500]):
        out, saved = quan.quan_packed_attention_forward(q, k, v, ints(first), heads, out=out, save=True)
        saved.stats.zero_()
        quan.quan_packed_attention_backward(q, k, v, out, saved, do, ints(first), heads, k_first=ints(first[::-1]),
                                            dq=a, dk=b, dv=c)
    torch.cuda.synchronize()
    assert bool((room[:, :total] == 3.0).all()) and bool((room[:, 2 * total:] == 3.0).all())


@pytest.mark.parametrize("count", [3, 64, 65, 256, 257, 1000])
def test_many_sequences(count):
    say(f"packed, {count} sequences")
    rng = np.random.default_rng(count)
    lens = rng.integers(0, 9, count).tolist()
    lens[count // 2] = 140
    heads, dq = 1, 8
    q, k, v, do = (rand_map(s, 1, heads * dq, 1, sum(lens), BF) for s in range(4))
    compare(q, k, v, do, lens, lens, heads, step(q, k, v, do, ints(ref.starts(lens).tolist()), heads), "many")


def test_gradients_against_differences():
    """In fp32, along random directions: central differences of the sum of dout out
    are off by the third derivative's h^2 / 6 (1e-6 for h = 2^-6, terms of order 1)
    and by fp32's rounding of the sums, 2^-24 sqrt(terms) / h: 1e-3 of the sums of
    a hundred products leaves room for both."""
    say("packed, differences")
    heads, dq, lens = 2, 5, [9, 21]
    maps = [rand_map(s, 1, heads * dq, 1, sum(lens), F32) for s in range(4)]
    first = ints(ref.starts(lens).tolist())
    grads = step(*maps, first, heads)[2:]
    h = 2.0 ** -6
    for i in range(3):
        way = rand_map(10 + i, 1, heads * dq, 1, sum(lens), F32)

        def at(s):
            moved = [t + s * h * way if j == i else t for j, t in enumerate(maps[:3])]
            return (quan.quan_packed_attention_forward(*moved, first, heads).double() * maps[3].double()).sum()
        slope = float((at(1) - at(-1)) / (2 * h))
        want = float((grads[i].double() * way.double()).sum())
        size = float((grads[i].double() * way.double()).abs().sum())
        assert abs(slope - want) <= 1e-3 * size, (i, slope, want)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("scale", [0.0, -0.3, 4.0])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_scores_of_any_size(dtype, scale, sign):
    """Scores far above and far below zero (all of a row's by hundreds), scales of
    either sign and none.  A score is a sum of d products, off by d 2^-24 of the sum
    of their absolute values S at most; a probability, the quotient of two powers, by
    twice that relatively, and so is delta: 4 d 2^-24 S of the sums of terms."""
    say(f"packed, scores of any size {dtype} {scale} {sign}")
    heads, dq, lens = 2, 16, [150, 33]
    q, k, v, do = (rand_map(s, 1, heads * dq, 1, sum(lens), dtype) for s in range(4))
    q, k = sign * (q.abs() + 1), k.abs() + 1
    got = step(q, k, v, do, ints(ref.starts(lens).tolist()), heads, scale=scale)
    most = max(float((rows(q, heads)[:, h] @ rows(k, heads)[:, h].T * scale).__abs__().max()) for h in range(heads))
    compare(q, k, v, do, lens, lens, heads, got, "scores", scale=scale, score=4 * dq * 2.0 ** -24 * most)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("dq", [16, 5])
def test_inference_and_no_rest(dtype, dq):
    """Without save the bound of one bf16 number per probability; gradients without
    the rounding's rest have delta off by 2^-8 of the sums of |dout out| more."""
    say(f"packed, inference {dtype} {dq}")
    heads, lens = 2, [5, 300, 64]
    q, k, v, do = (rand_map(s, 1, heads * dq, 1, sum(lens), dtype) for s in range(4))
    first = ints(ref.starts(lens).tolist())
    out = quan.quan_packed_attention_forward(q, k, v, first, heads)
    want, err = ref.packed(*(rows(t, heads) for t in (q, k, v)), lens, lens)
    ref.check(rows(out, heads), want["out"], err["out"], dtype == BF, "inference")
    out, saved = quan.quan_packed_attention_forward(q, k, v, first, heads, save=True)
    grads = quan.quan_packed_attention_backward(q, k, v, out, saved._replace(rest=None), do, first, heads)
    again = quan.quan_packed_attention_backward(q, k, v, out, saved, do, first, heads)
    assert torch.equal(grads[2], again[2])  # (dv knows nothing of delta)
    if dtype == F32:
        assert all(torch.equal(a, b) for a, b in zip(grads, again))
        return
    # dq's change is scale sum_j P_ij k_j times delta's, |delta's| <= 2^-8 sum |dout out|,
    # and the two roundings of dS and of dq beside it
    off = (np.abs(rows(do, heads)) * np.abs(want["out"])).sum(2, keepdims=True) * ref.U
    res, bound = ref.packed(*(rows(t, heads) for t in (q, k, v)), lens, lens, dout=rows(do, heads))
    most = off * np.abs(rows(k, heads)).max() / np.sqrt(4 * dq)
    assert np.all(np.abs(rows(grads[0], heads) - res["dq"]) <= 1.01 * bound["dq"][0] + bound["dq"][1] + most)


@pytest.mark.parametrize("dq", [16, 12, 8])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "all"])
def test_many_heads(dq, causal):
    """Enough blocks for 64 queries to a wave, long ones and odd ones among them, with
    and without what a backward pass needs; a NaN key of the last sequence's middle
    reaches the queries behind it and no other."""
    say(f"packed, many heads {dq} causal {causal}")
    heads, kvh, lens = 56, 8, [600, 0, 1, 257, 700, 33]
    total = sum(lens)
    q, do = (rand_map(s, 1, heads * dq, 1, total, BF) for s in (1, 2))
    k, v = (rand_map(s, 1, kvh * dq, 1, total, BF) for s in (3, 4))
    first = ints(ref.starts(lens).tolist())
    got = step(q, k, v, do, first, heads, causal=causal)
    compare(q, k, v, do, lens, lens, heads, got, "many heads", causal)
    out = quan.quan_packed_attention_forward(q, k, v, first, heads, causal=causal)
    want, err = ref.packed(rows(q, heads), rows(k, kvh), rows(v, kvh), lens, lens, causal)
    ref.check(rows(out, heads), want["out"], err["out"], True, "many heads, inference")
    k = k.clone(memory_format=torch.preserve_format)
    k[0, :, :, 0, total - 17] = float("nan")
    hit = slice(total - 17, total) if causal else slice(total - 33, total)
    for t in (quan.quan_packed_attention_forward(q, k, v, first, heads, causal=causal),
              step(q, k, v, do, first, heads, causal=causal)[0]):
        assert not bool(torch.isfinite(t[..., hit]).any())
        assert bool(torch.isfinite(t[..., :hit.start]).all())
        ref.check(rows(t, heads)[:hit.start], want["out"][:hit.start], (err["out"][0][:hit.start], err["out"][1]), True, "rest")


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("dq,heads,kv_heads", [(16, 6, 2), (16, 12, 12), (8, 24, 8), (32, 6, 6), (16, 7, 7)])
def test_heads_in_cache_lines(dtype, dq, heads, kv_heads):
    """Heads that share lines of 128 bytes by twos, fours and eights, in three such sets
    or none: every head and block is there once, with walks shared and whole."""
    say(f"packed, heads in lines {dtype} {dq} {heads}/{kv_heads}")
    lens = [400, 129, 0, 33]
    q, do = (rand_map(s, 1, heads * dq, 1, sum(lens), dtype) for s in (1, 2))
    k, v = (rand_map(s, 1, kv_heads * dq, 1, sum(lens), dtype) for s in (3, 4))
    compare(q, k, v, do, lens, lens, heads, step(q, k, v, do, ints(ref.starts(lens).tolist()), heads), "lines")


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("dq", [16, 32])
@pytest.mark.parametrize("q_tokens,k_tokens,first,lq,lk", [
    (300, 200, [0, 300], [300], [200]), (200, 300, [0, 300], [200], [300]),
    (300, 200, [0, 130, 260, 300], [130, 130, 40], [130, 70, 0]), (200, 2100, [0, 90, 2100], [90, 110], [90, 2010]),
    (2100, 200, [0, 90, 2100], [90, 2010], [90, 110])])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "all"])
def test_one_array_for_maps_of_two_sizes(dtype, dq, q_tokens, k_tokens, first, lq, lk, causal):
    """Offsets beyond the smaller map, given for both as one tensor: its sequences end
    with it, as they do with an array of their own; NaN behind the keys is not read,
    and what lies around the results stays."""
    say(f"packed, one array {dtype} dq {dq} {q_tokens} on {k_tokens} of {first} causal {causal}")
    heads, spare = 2, 400

    def room(value, tokens):
        all_of = torch.full((spare + tokens + spare, 4, heads * dq), value, dtype=dtype, device=DEV)
        return all_of, all_of[spare:spare + tokens][None, None].permute(0, 3, 4, 1, 2)
    q, do = (rand_map(s, 1, heads * dq, 1, q_tokens, dtype) for s in (1, 2))
    k, v = (room(float("nan"), k_tokens)[1].copy_(rand_map(s, 1, heads * dq, 1, k_tokens, dtype)) for s in (3, 4))
    first = ints(first)

    def run(k_first):
        rooms = [room(3.0, t) for t in (q_tokens, q_tokens, k_tokens, k_tokens)]
        out, dqs, dks, dvs = (view for _, view in rooms)
        _, saved = quan.quan_packed_attention_forward(q, k, v, first, heads, k_first=k_first, causal=causal, out=out, save=True)
        quan.quan_packed_attention_backward(q, k, v, out, saved, do, first, heads, k_first=k_first, causal=causal, dq=dqs,
                                            dk=dks, dv=dvs)
        for all_of, _ in rooms:
            assert bool((all_of[:spare] == 3.0).all()) and bool((all_of[-spare:] == 3.0).all())
        return out, saved.stats, dqs, dks, dvs
    got = run(first)
    compare(q, k, v, do, lq, lk, heads, got, "one array", causal)
    assert all(torch.equal(a, b) for a, b in zip(got, run(first.clone())))


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("save", [False, True], ids=["inference", "training"])
@pytest.mark.parametrize("heads,kv_heads,dq,lq,lk", [
    (2, 1, 16, [300, 40], None), (2, 2, 32, [300, 40], None), (2, 2, 5, [70], [200]), (1, 1, 16, [130], [2000]),
    (56, 8, 16, [600, 300], None)])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "all"])
def test_infinite_values(dtype, save, heads, kv_heads, dq, lq, lk, causal):
    """An infinity in v that a query sees is its result's, both signs in one place are
    NaN, as is a NaN: in the walk and at its edge, at inference and in training.  The
    other reals keep their bounds."""
    say(f"packed, infinite values {dtype} save {save} heads {heads}/{kv_heads} dq {dq} {lq} {lk} causal {causal}")
    lk = lk or lq
    q = rand_map(1, 1, heads * dq, 1, sum(lq), dtype)
    k, v = (rand_map(s, 1, kv_heads * dq, 1, sum(lk), dtype) for s in (2, 3))
    first, k_first = (ints(ref.starts(t).tolist()) for t in (lq, lk))
    # (component, channel, token, value) of the first head of keys in the first sequence
    odd = [(0, 0, 3, np.inf), (1, 2, 3, -np.inf), (1, 3, 65, np.inf), (2, 1, 10, np.inf), (2, 1, lk[0] - 2, -np.inf),
           (3, 4, 69, np.nan), (3, 0, 20, np.inf), (3, 0, 66, np.nan), (3, 0, 67, np.inf)]
    zeros = v.clone(memory_format=torch.preserve_format)
    for comp, ch, token, value in odd:
        v[0, comp, ch, 0, token] = value
        zeros[0, comp, ch, 0, token] = 0.0
    got = quan.quan_packed_attention_forward(q, k, v, first, heads, k_first=k_first, causal=causal, save=save)
    got = rows(got[0] if save else got, heads)
    # (with dout the bounds are those of a training step)
    want, err = ref.packed(rows(q, heads), rows(k, kv_heads), rows(zeros, kv_heads), lq, lk, causal,
                           dout=np.zeros_like(got) if save else None)
    want, bound = want["out"], err["out"]
    extra = np.zeros_like(want)
    for comp, ch, token, value in odd:
        sees = np.arange(lq[0]) >= (token - (lk[0] - lq[0]) if causal else 0)
        with np.errstate(invalid="ignore"):
            extra[:lq[0], :heads // kv_heads, comp * dq + ch] += np.where(sees, value, 0.0)[:, None]
    hit = ~np.isfinite(extra)
    assert hit.any() and np.array_equal(got[hit], extra[hit], equal_nan=True)
    fixed = np.where(hit, want, got)
    ref.check(fixed, want, (bound[0], bound[1]), dtype == BF, "the others")


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("count", [65, 100, 200])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "all"])
def test_many_sequences_with_shared_walks(dtype, count, causal):
    """Sequences in several sets of 64, the long ones behind the first set with walks
    that work-groups share (one head leaves fewer blocks than are wanted)."""
    say(f"packed, {count} sequences with shared walks {dtype} causal {causal}")
    lens = np.random.default_rng(count).integers(0, 9, count).tolist()
    lens[0], lens[64], lens[count - 1] = 0, 700, 2000
    heads, dq = 1, 8
    q, k, v, do = (rand_map(s, 1, heads * dq, 1, sum(lens), dtype) for s in range(4))
    first = ints(ref.starts(lens).tolist())
    got = step(q, k, v, do, first, heads, causal=causal)
    compare(q, k, v, do, lens, lens, heads, got, "many", causal)
    assert all(torch.equal(a, b) for a, b in zip(got, step(q, k, v, do, first, heads, causal=causal)))


@pytest.mark.parametrize("count", [4096, 4097, 5000])
def test_thousands_of_sequences(count):
    """More sets of 64 sequences than a wave has lanes, longer ones in the last of them."""
    say(f"packed, {count} sequences")
    lens = np.random.default_rng(count).integers(0, 4, count).tolist()
    lens[0], lens[70], lens[count - 3], lens[count - 1] = 0, 300, 200, 129
    heads, dq = 1, 8
    q, k, v, do = (rand_map(s, 1, heads * dq, 1, sum(lens), BF) for s in range(4))
    compare(q, k, v, do, lens, lens, heads, step(q, k, v, do, ints(ref.starts(lens).tolist()), heads), "thousands")
