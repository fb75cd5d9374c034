"""The attention block's entry points refuse what they cannot take, on the
host; bucket maps."""
import ctypes
import math
import os

import numpy as np
import pytest
import torch

from paper_2509_05512_amd import quan

E_NULL, E_SHAPE, E_DTYPE, E_ALIGN, E_ALIAS, E_UNSUP, E_LAYOUT = -1, -2, -3, -4, -5, -6, -9


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(quan.LIB_PATH):
        pytest.skip("libquan.so not built")
    return quan.load_library()


def addr(i):
    """Disjoint made-up addresses, never read."""
    return 0x100000000 * (i + 1)


def desc(data, n=2, c=16, h=4, w=6, dtype=1, strides=None, ndim=5, comp=4, c_all=None):
    c_all = c_all or c
    s = strides or (h * w * 4 * c_all, c_all, 1, w * 4 * c_all, 4 * c_all)
    return quan.QuanTensor(data, dtype, ndim, (ctypes.c_int64 * 5)(n, comp, c, h, w), (ctypes.c_int64 * 5)(*s))


class QuanRelpos(ctypes.Structure):
    """struct quan_relpos"""
    _fields_ = [(m, ctypes.c_void_p) for m in ("table", "bucket_y", "bucket_x")] \
        + [(m, ctypes.c_int32) for m in ("buckets_y", "buckets_x", "radius_y", "radius_x")]


def relpos(**kw):
    a = dict(table=addr(20), bucket_y=addr(21), bucket_x=addr(22), buckets_y=4, buckets_x=5, radius_y=3, radius_x=5)
    a.update(kw)
    return QuanRelpos(*a.values())


def attention(lib, back=False, **kw):
    a = dict(q=desc(addr(0)), k=desc(addr(1)), v=desc(addr(2)), relpos=relpos(), kv_len=addr(23), pos=addr(24),
             scale=0.125, heads=2, out=desc(addr(3)), rest=addr(4), stats=addr(5), dout=desc(addr(6)), dq=desc(addr(7)),
             dk=desc(addr(8)), dv=desc(addr(9)), dtable=addr(10))
    a.update(kw)

    def ref(d):
        return None if d is None else ctypes.byref(d)
    first = [ref(a["q"]), ref(a["k"]), ref(a["v"]), ref(a["relpos"]), a["kv_len"], a["pos"], a["scale"], a["heads"],
             ref(a["out"]), a["rest"], a["stats"]]
    if back:
        rc = lib.quan_attention_backward(*first, ref(a["dout"]), ref(a["dq"]), ref(a["dk"]), ref(a["dv"]), a["dtable"], None)
    else:
        rc = lib.quan_attention_forward(*first, None)
    return rc, lib.quan_last_error().decode()


BOTH = [
    ("q null", dict(q=None), E_NULL), ("k null", dict(k=None), E_NULL), ("v null", dict(v=None), E_NULL),
    ("q data null", dict(q=desc(None)), E_NULL), ("out null", dict(out=None), E_NULL),
    ("dtype", dict(q=desc(addr(0), dtype=2)), E_DTYPE), ("k's dtype", dict(k=desc(addr(1), dtype=0)), E_DTYPE),
    ("out's dtype", dict(out=desc(addr(3), dtype=0)), E_DTYPE),
    ("axes", dict(q=desc(addr(0), ndim=4)), E_SHAPE), ("components", dict(q=desc(addr(0), comp=3)), E_SHAPE),
    ("batch of k", dict(k=desc(addr(1), n=3)), E_SHAPE), ("v unlike k", dict(v=desc(addr(2), w=7)), E_SHAPE),
    ("out unlike q", dict(out=desc(addr(3), h=5)), E_SHAPE), ("empty", dict(q=desc(addr(0), h=0)), E_SHAPE),
    ("heads 0", dict(heads=0), E_SHAPE), ("heads do not divide", dict(heads=3), E_SHAPE),
    ("kv channels", dict(k=desc(addr(1), c=12), v=desc(addr(2), c=12)), E_SHAPE),
    ("kv heads do not divide", dict(heads=4, k=desc(addr(1), c=12), v=desc(addr(2), c=12)), E_SHAPE),
    ("wide heads", dict(heads=1, **{m: desc(addr(i), c=33) for i, m in ((0, "q"), (1, "k"), (2, "v"), (3, "out"))}),
     E_UNSUP),
    ("scale nan", dict(scale=math.nan), E_SHAPE), ("scale inf", dict(scale=math.inf), E_SHAPE),
    ("channel stride", dict(q=desc(addr(0), strides=(1536, 1, 4, 384, 64))), E_LAYOUT),
    ("planes", dict(q=desc(addr(0), strides=(1536, 384, 24, 6, 1))), E_LAYOUT),
    ("broadcast images", dict(k=desc(addr(1), strides=(0, 16, 1, 384, 64))), E_LAYOUT),
    ("rows apart", dict(k=desc(addr(1), strides=(4096, 16, 1, 512, 64))), E_LAYOUT),
    ("pixels overlap", dict(k=desc(addr(1), strides=(1536, 16, 1, 360, 60))), E_LAYOUT),
    ("negative", dict(k=desc(addr(1), strides=(-1536, 16, 1, 384, 64))), E_LAYOUT),
    ("element alignment", dict(q=desc(addr(0) + 1)), E_ALIGN), ("rest alignment", dict(rest=addr(4) + 2), E_ALIGN),
    ("stats alignment", dict(stats=addr(5) + 2), E_ALIGN), ("kv_len alignment", dict(kv_len=addr(23) + 1), E_ALIGN),
    ("pos alignment", dict(pos=addr(24) + 3), E_ALIGN),
    ("rest of fp32", dict(**{m: desc(addr(i), dtype=0) for i, m in
                             ((0, "q"), (1, "k"), (2, "v"), (3, "out"), (6, "dout"), (7, "dq"), (8, "dk"), (9, "dv"))}),
     E_DTYPE),
    ("table null", dict(relpos=relpos(table=None)), E_NULL), ("no buckets", dict(relpos=relpos(buckets_x=0)), E_SHAPE),
    ("radius", dict(relpos=relpos(radius_y=-1)), E_SHAPE), ("many buckets", dict(relpos=relpos(buckets_y=1025)), E_UNSUP),
    ("table alignment", dict(relpos=relpos(table=addr(20) + 2)), E_ALIGN),
    ("wide map", dict(**{m: desc(addr(i), w=1793) for i, m in
                         ((0, "q"), (1, "k"), (2, "v"), (3, "out"), (6, "dout"), (7, "dq"), (8, "dk"), (9, "dv"))}), E_UNSUP),
    ("many pixels", dict(k=desc(addr(1), h=5000, w=5000), v=desc(addr(2), h=5000, w=5000)), E_UNSUP),
]


@pytest.mark.parametrize("back", [False, True], ids=["forward", "backward"])
@pytest.mark.parametrize("what,kw,code", BOTH, ids=[b[0] for b in BOTH])
def test_attention_refuses(lib, what, kw, code, back):
    rc, msg = attention(lib, back, **kw)
    assert rc == code, (what, rc, msg)
    assert msg


FORWARD = [
    ("out on q", dict(out=desc(addr(0))), E_ALIAS), ("out on k", dict(out=desc(addr(1) + 64)), E_ALIAS),
    ("rest on v", dict(rest=addr(2)), E_ALIAS), ("stats on out", dict(stats=addr(3)), E_ALIAS),
    ("out on the table", dict(out=desc(addr(20))), E_ALIAS), ("rest on kv_len", dict(rest=addr(23)), E_ALIAS),
    ("slices that meet", dict(q=desc(addr(0), c_all=64), out=desc(addr(0) + 2 * 8, c_all=64)), E_ALIAS),
]
BACKWARD = [
    ("dout null", dict(dout=None), E_NULL), ("dq null", dict(dq=None), E_NULL), ("dk null", dict(dk=None), E_NULL),
    ("dv null", dict(dv=None), E_NULL), ("stats null", dict(stats=None), E_NULL),
    ("dtable without a bias", dict(relpos=None), E_NULL), ("dq unlike q", dict(dq=desc(addr(7), c=8)), E_SHAPE),
    ("dk unlike k", dict(dk=desc(addr(8), h=2)), E_SHAPE), ("dq on dout", dict(dq=desc(addr(6))), E_ALIAS),
    ("dk on dv", dict(dk=desc(addr(9))), E_ALIAS), ("dk on k", dict(dk=desc(addr(1))), E_ALIAS),
    ("dtable on dq", dict(dtable=addr(7)), E_ALIAS), ("dtable on stats", dict(dtable=addr(5)), E_ALIAS),
    ("dtable alignment", dict(dtable=addr(10) + 1), E_ALIGN),
]


@pytest.mark.parametrize("what,kw,code", FORWARD, ids=[b[0] for b in FORWARD])
def test_forward_refuses(lib, what, kw, code):
    rc, msg = attention(lib, False, **kw)
    assert rc == code and msg, (what, rc, msg)


@pytest.mark.parametrize("what,kw,code", BACKWARD, ids=[b[0] for b in BACKWARD])
def test_backward_refuses(lib, what, kw, code):
    rc, msg = attention(lib, True, **kw)
    assert rc == code and msg, (what, rc, msg)


MAP, ROW = 2 * 4 * 6 * 4 * 16 * 2, 4 * 16 * 4
X, Y, GATE, OUT, H, DOUT, DH, DX, DY, DGATE = (0x10000000 * (i + 1) for i in range(10))
GA, SC, NG, DGA, DSC, DNG, RNG = (0x100000000 + 0x100000 * i for i in range(7))


def rows(lib, fn, **kw):
    a = dict(x=X, y=Y, gate=GATE, gamma=GA, scale=SC, next_gamma=NG, p=0.1, rng=RNG, eps=1e-6, out=OUT, h_=H, dout=DOUT,
             dh=DH, dx=DX, dy=DY, dgate=DGATE, dgamma=DGA, dscale=DSC, dnext=DNG, dres=None, n=2, c=16, h=4, w=6, dtype=1)
    a.update(kw)
    size = [a[k] for k in ("n", "c", "h", "w", "dtype")] + [None]
    if fn == "residual_forward":
        args = [a[k] for k in ("x", "y", "gate", "gamma", "scale", "next_gamma", "p", "rng", "eps", "out", "h_")]
    elif fn == "residual_backward":
        args = [a[k] for k in ("y", "dout", "out", "dh", "gate", "gamma", "scale", "next_gamma", "p", "rng", "eps", "dx",
                               "dy", "dgate", "dgamma", "dscale", "dnext")]
    elif fn == "rmsnorm_forward":
        args = [a[k] for k in ("x", "gamma", "eps", "out")]
    elif fn == "rmsnorm_backward":
        args = [a[k] for k in ("x", "dout", "gamma", "dres", "eps", "dx", "dgamma")]
    else:
        args = [a[k] for k in ("x", "p", "rng", "out")]
    rc = getattr(lib, "quan_" + fn)(*args, *size)
    return rc, lib.quan_last_error().decode()


ALL = ["residual_forward", "residual_backward", "rmsnorm_forward", "rmsnorm_backward", "dropout"]
ROWS = [(fn, kw, code) for fn in ALL for kw, code in (
    (dict(n=0), E_SHAPE), (dict(c=-1), E_SHAPE), (dict(dtype=2), E_DTYPE), (dict(h=1 << 20, w=1 << 20), E_UNSUP))]
ROWS += [(fn, kw, code) for fn in ALL[:4] for kw, code in (
    (dict(eps=0.0), E_SHAPE), (dict(eps=math.nan), E_SHAPE), (dict(eps=math.inf), E_SHAPE), (dict(c=1025), E_UNSUP),
    (dict(gamma=GA + 1), E_ALIGN))]
ROWS += [(fn, kw, code) for fn in ("residual_forward", "residual_backward", "dropout") for kw, code in (
    (dict(p=-0.1), E_SHAPE), (dict(p=1.0), E_SHAPE), (dict(p=math.nan), E_SHAPE), (dict(rng=None), E_NULL),
    (dict(rng=RNG + 4), E_ALIGN))]
ROWS += [("residual_forward", kw, code) for kw, code in (
    (dict(x=None), E_NULL), (dict(y=None), E_NULL), (dict(out=None), E_NULL), (dict(h_=None), E_NULL),
    (dict(next_gamma=None), E_NULL), (dict(x=X + 8), E_ALIGN), (dict(gate=GATE + 8), E_ALIGN), (dict(h_=OUT), E_ALIAS),
    (dict(h_=X), E_ALIAS), (dict(out=X + 16), E_ALIAS), (dict(out=GATE - 16), E_ALIAS), (dict(scale=H), E_ALIAS))]
ROWS += [("residual_backward", kw, code) for kw, code in (
    (dict(y=None), E_NULL), (dict(dout=None), E_NULL), (dict(dx=None), E_NULL), (dict(dy=None), E_NULL),
    (dict(out=None), E_NULL), (dict(dh=None), E_NULL), (dict(dnext=None), E_NULL), (dict(dgate=None), E_NULL),
    (dict(gate=None), E_NULL), (dict(dgamma=None), E_NULL), (dict(scale=None), E_NULL), (dict(dx=DX + 8), E_ALIGN),
    (dict(dgate=DGATE + 4), E_ALIGN), (dict(dx=DY), E_ALIAS), (dict(dx=OUT), E_ALIAS), (dict(dy=DOUT), E_ALIAS),
    (dict(dx=Y), E_ALIAS), (dict(dgate=DX), E_ALIAS), (dict(dgamma=DSC), E_ALIAS), (dict(dnext=NG), E_ALIAS),
    (dict(dscale=DY), E_ALIAS))]
ROWS += [("rmsnorm_forward", kw, code) for kw, code in (
    (dict(x=None), E_NULL), (dict(gamma=None), E_NULL), (dict(out=None), E_NULL), (dict(out=X + 16), E_ALIAS))]
ROWS += [("rmsnorm_backward", kw, code) for kw, code in (
    (dict(x=None), E_NULL), (dict(dgamma=None), E_NULL), (dict(dx=X), E_ALIAS), (dict(dres=DX + 16), E_ALIAS),
    (dict(dres=DX + 8), E_ALIGN), (dict(dgamma=DX), E_ALIAS))]
ROWS += [("dropout", kw, code) for kw, code in ((dict(x=None), E_NULL), (dict(out=X + 32), E_ALIAS), (dict(out=RNG - 16), E_ALIAS))]


@pytest.mark.parametrize("fn,kw,code", ROWS, ids=[f"{r[0]}-{'-'.join(map(str, r[1]))}-{i}" for i, r in enumerate(ROWS)])
def test_rows_refuse(lib, fn, kw, code):
    rc, msg = rows(lib, fn, **kw)
    assert rc == code and msg, (fn, kw, rc, msg)


def test_binding_refuses():
    q = quan.empty_qmap(2, 16, 4, 6, torch.bfloat16, "cpu")
    table, b = torch.zeros(2, 3, 3), torch.zeros(3, dtype=torch.int32)
    for kw in (dict(relpos=(table.double(), b, b)), dict(relpos=(table, b.long(), b)), dict(relpos=(table[:1], b, b)),
               dict(relpos=(table, b[:2], b)), dict(relpos=(table[0], b, b)), dict(kv_len=torch.zeros(3, dtype=torch.int32)),
               dict(kv_len=torch.zeros(2)), dict(pos=torch.zeros(2, dtype=torch.int32))):
        with pytest.raises(ValueError):
            quan.quan_attention_forward(q, q, q, 2, **kw)
    g = torch.ones(4, 16)
    for kw in (dict(gamma=g.double()), dict(gamma=g[:, :8]), dict(gate=q), dict(p=0.1), dict(h=q),
               dict(p=0.1, rng=torch.zeros(2)), dict(out=q.contiguous())):
        with pytest.raises(ValueError):
            quan.quan_residual_forward(q, q, **kw)
    with pytest.raises(ValueError):
        quan.quan_residual_backward(q, q, next_gamma=g)
    with pytest.raises(ValueError):
        quan.quan_rmsnorm_forward(q.contiguous(), g)
    with pytest.raises(TypeError):
        quan.quan_attention_forward(q.half(), q.half(), q.half(), 2)


def test_bucket_maps():
    """One bucket per offset where there are enough; else signs apart, near
    distances one each, then ever wider, all within range."""
    assert quan.quan_relpos_buckets(0, 1).tolist() == [0]
    assert quan.quan_relpos_buckets(3, 7).tolist() == list(range(7))
    assert quan.quan_relpos_buckets(3, 1).tolist() == [0] * 7
    for radius, buckets in ((64, 16), (100, 31), (13, 8), (1000, 32), (5, 3)):
        m = np.array(quan.quan_relpos_buckets(radius, buckets).tolist())
        half = buckets // 2
        left, right = m[:radius + 1][::-1], m[radius + 1:]
        assert m.min() >= 0 and m.max() < 2 * half
        assert np.all(np.diff(left) >= 0) and np.all(left < half)
        assert np.array_equal(right, left[1:] + half)
        near = max(1, half // 2)
        assert np.array_equal(left[:near], np.arange(near)) and left[-1] == half - 1
    for args, code in (((-1, 4), E_SHAPE), ((4, 0), E_SHAPE), ((4, 5000), E_UNSUP)):
        with pytest.raises(quan.QuanError) as e:
            quan.quan_relpos_buckets(*args)
        assert e.value.code == code
