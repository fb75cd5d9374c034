"""The entry points of sequences of pixels refuse what they cannot take, on the
host; the reference's pins."""
import ctypes
import math
import os

import numpy as np
import pytest
import torch

import sequence_reference as ref
from paper_2509_05512_amd import quan
from paper_2509_05512_amd.attention_block import AttentionBlock
from test_block_cpu import QuanRelpos, addr, desc, relpos

E_NULL, E_SHAPE, E_DTYPE, E_ALIGN, E_ALIAS, E_UNSUP, E_LAYOUT = -1, -2, -3, -4, -5, -6, -9


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(quan.LIB_PATH):
        pytest.skip("libquan.so not built")
    return quan.load_library()


class QuanCache(ctypes.Structure):
    """struct quan_cache"""
    _fields_ = [(m, ctypes.c_void_p) for m in ("keys", "values", "key_exp", "value_exp", "table")] \
        + [(m, ctypes.c_int32) for m in ("format", "pages", "page_tokens", "heads", "dq", "sequences", "table_pages")]


def cache(**kw):
    a = dict(keys=addr(30), values=addr(31), key_exp=addr(32), value_exp=addr(33), table=addr(34), format=2, pages=9,
             page_tokens=16, heads=2, dq=8, sequences=2, table_pages=4)
    a.update(kw)
    return QuanCache(*a.values())


def ref_of(d):
    return None if d is None else ctypes.byref(d)


def copy(lib, write, **kw):
    a = dict(k=desc(addr(0)), v=desc(addr(1)), first=None, start=addr(23), kv_len=addr(24), cache=cache())
    a.update(kw)
    maps = [ref_of(a["k"]), ref_of(a["v"])]
    ints = [a["first"], a["start"], a["kv_len"]]
    if write:
        rc = lib.quan_cache_write(*maps, *ints, ref_of(a["cache"]), None)
    else:
        rc = lib.quan_cache_read(ref_of(a["cache"]), *ints, *maps, None)
    return rc, lib.quan_last_error().decode()


CACHE = [
    (dict(cache=None), E_NULL), (dict(cache=cache(keys=None)), E_NULL), (dict(cache=cache(values=None)), E_NULL),
    (dict(cache=cache(table=None)), E_NULL), (dict(cache=cache(key_exp=None)), E_NULL),
    (dict(cache=cache(value_exp=None)), E_NULL), (dict(cache=cache(format=3)), E_DTYPE),
    (dict(cache=cache(format=-1)), E_DTYPE), (dict(cache=cache(format=0)), E_DTYPE), (dict(cache=cache(pages=0)), E_SHAPE),
    (dict(cache=cache(page_tokens=0)), E_SHAPE), (dict(cache=cache(heads=0)), E_SHAPE), (dict(cache=cache(dq=0)), E_SHAPE),
    (dict(cache=cache(sequences=0)), E_SHAPE), (dict(cache=cache(table_pages=0)), E_SHAPE),
    (dict(cache=cache(dq=33)), E_UNSUP), (dict(cache=cache(heads=65536)), E_UNSUP),
    (dict(cache=cache(page_tokens=(1 << 24) + 1)), E_UNSUP), (dict(cache=cache(pages=1 << 27)), E_UNSUP),
    (dict(cache=cache(table_pages=1 << 27)), E_UNSUP), (dict(cache=cache(table_pages=(1 << 26) + 1)), E_UNSUP), (dict(cache=cache(heads=65535, page_tokens=1 << 24)), E_UNSUP),
    (dict(cache=cache(sequences=1 << 16, table_pages=1 << 15)), E_UNSUP),
    (dict(cache=cache(keys=addr(30) + 8)), E_ALIGN), (dict(cache=cache(values=addr(31) + 4)), E_ALIGN),
    (dict(cache=cache(table=addr(34) + 2)), E_ALIGN),
]
COPY = CACHE + [
    (dict(k=None), E_NULL), (dict(v=None), E_NULL), (dict(k=desc(None)), E_NULL), (dict(k=desc(addr(0), dtype=2)), E_DTYPE),
    (dict(v=desc(addr(1), dtype=0)), E_DTYPE), (dict(k=desc(addr(0), c=24)), E_SHAPE), (dict(v=desc(addr(1), w=7)), E_SHAPE),
    (dict(k=desc(addr(0), n=3), v=desc(addr(1), n=3)), E_SHAPE), (dict(first=addr(25)), E_SHAPE),
    (dict(k=desc(addr(0), strides=(1536, 1, 4, 384, 64))), E_LAYOUT), (dict(k=desc(addr(0) + 1)), E_ALIGN),
    (dict(start=addr(23) + 1), E_ALIGN), (dict(kv_len=addr(24) + 2), E_ALIGN),
    (dict(first=addr(25) + 2, k=desc(addr(0), n=1), v=desc(addr(1), n=1)), E_ALIGN),
]


@pytest.mark.parametrize("write", [True, False], ids=["write", "read"])
@pytest.mark.parametrize("kw,code", COPY, ids=[f"{'-'.join(c[0])}-{i}" for i, c in enumerate(COPY)])
def test_copies_refuse(lib, kw, code, write):
    rc, msg = copy(lib, write, **kw)
    assert rc == code and msg, (kw, rc, msg)


@pytest.mark.parametrize("write,kw", [
    (True, dict(cache=cache(keys=addr(0)))), (True, dict(cache=cache(value_exp=addr(1) + 64))),
    (True, dict(cache=cache(values=addr(30) + 1024))), (True, dict(cache=cache(key_exp=addr(34)))),
    (True, dict(cache=cache(key_exp=addr(33) + 16))), (True, dict(start=addr(30) + 16)),
    (False, dict(k=desc(addr(30)))), (False, dict(v=desc(addr(0)))), (False, dict(v=desc(addr(32)))),
    (False, dict(k=desc(addr(24)))),
    (False, dict(k=desc(addr(0), c_all=64), v=desc(addr(0) + 2 * 8, c_all=64)))])
def test_copies_refuse_overlaps(lib, write, kw):
    rc, msg = copy(lib, write, **kw)
    assert rc == E_ALIAS and msg, (kw, rc, msg)


def test_first_takes_one_image(lib):
    one = dict(k=desc(addr(0), n=1), v=desc(addr(1), n=1))
    assert copy(lib, True, **one)[0] == E_SHAPE                  # two sequences, one image
    rc, msg = copy(lib, True, first=addr(1), **one)              # (taken up to the overlap with v: that is read only)
    assert "images" not in msg
    assert copy(lib, False, first=addr(1), **one)[0] == E_ALIAS


def token(lib, **kw):
    a = dict(q=desc(addr(0), h=1, w=1, c=32), cache=cache(), relpos=relpos(), width=5, kv_len=addr(23), pos=addr(24), scale=0.125,
             heads=4, out=desc(addr(1), h=1, w=1, c=32))
    a.update(kw)
    rc = lib.quan_cache_attention(ref_of(a["q"]), ref_of(a["cache"]), ref_of(a["relpos"]), a["width"], a["kv_len"], a["pos"],
                                  a["scale"], a["heads"], ref_of(a["out"]), None)
    return rc, lib.quan_last_error().decode()


def row(i, **kw):
    return desc(addr(i), **{**dict(h=1, w=1, c=32), **kw})


TOKEN = CACHE + [
    (dict(q=None), E_NULL), (dict(out=None), E_NULL), (dict(q=row(0, dtype=2)), E_DTYPE), (dict(out=row(1, dtype=0)), E_DTYPE),
    (dict(heads=0), E_SHAPE), (dict(heads=3), E_SHAPE), (dict(heads=2), E_SHAPE), (dict(heads=65536), E_UNSUP),
    (dict(q=row(0, w=2)), E_SHAPE), (dict(q=row(0, n=3)), E_SHAPE), (dict(q=row(0, c=16)), E_SHAPE),
    (dict(out=row(1, c=16)), E_SHAPE), (dict(scale=math.nan), E_SHAPE), (dict(scale=math.inf), E_SHAPE),
    (dict(width=0), E_SHAPE), (dict(relpos=relpos(table=None)), E_NULL), (dict(relpos=relpos(buckets_x=0)), E_SHAPE),
    (dict(relpos=relpos(buckets_y=1025)), E_UNSUP), (dict(relpos=relpos(bucket_x=addr(22) + 2)), E_ALIGN),
    (dict(kv_len=addr(23) + 1), E_ALIGN), (dict(pos=addr(24) + 2), E_ALIGN), (dict(q=desc(addr(0) + 1, h=1, w=1, c=32)), E_ALIGN),
    (dict(out=row(0)), E_ALIAS), (dict(out=row(30)), E_ALIAS), (dict(out=row(33)), E_ALIAS), (dict(out=row(34)), E_ALIAS),
    (dict(out=row(20)), E_ALIAS), (dict(out=row(23)), E_ALIAS),
]


@pytest.mark.parametrize("kw,code", TOKEN, ids=[f"{'-'.join(c[0])}-{i}" for i, c in enumerate(TOKEN)])
def test_cache_attention_refuses(lib, kw, code):
    rc, msg = token(lib, **kw)
    assert rc == code and msg, (kw, rc, msg)


def packed(lib, back=False, **kw):
    a = dict(q=desc(addr(0)), k=desc(addr(1)), v=desc(addr(2)), q_first=None, k_first=None, sequences=2, causal=1, scale=0.125,
             heads=2, out=desc(addr(3)), rest=addr(4), stats=addr(5), dout=desc(addr(6)), dq=desc(addr(7)), dk=desc(addr(8)), dv=desc(addr(9)))
    a.update(kw)
    first = [ref_of(a["q"]), ref_of(a["k"]), ref_of(a["v"]), a["q_first"], a["k_first"], a["sequences"], a["causal"], a["scale"],
             a["heads"], ref_of(a["out"]), a["rest"], a["stats"]]
    if back:
        rc = lib.quan_packed_attention_backward(*first, *(ref_of(a[m]) for m in ("dout", "dq", "dk", "dv")), None)
    else:
        rc = lib.quan_packed_attention_forward(*first, None)
    return rc, lib.quan_last_error().decode()


def one(**kw):
    """Maps of one image of 24 pixels."""
    return {m: desc(addr(i), n=1) for i, m in ((0, "q"), (1, "k"), (2, "v"), (3, "out"), (6, "dout"), (7, "dq"), (8, "dk"),
                                               (9, "dv"))} | dict(q_first=addr(23), **kw)


PACKED = [
    (dict(q=None), E_NULL), (dict(k=None), E_NULL), (dict(v=None), E_NULL), (dict(out=None), E_NULL),
    (dict(q=desc(addr(0), dtype=3)), E_DTYPE), (dict(k=desc(addr(1), dtype=0)), E_DTYPE), (dict(q=desc(addr(0), ndim=4)), E_SHAPE),
    (dict(k=desc(addr(1), n=3)), E_SHAPE), (dict(v=desc(addr(2), w=7)), E_SHAPE), (dict(out=desc(addr(3), h=5)), E_SHAPE),
    (dict(heads=0), E_SHAPE), (dict(heads=3), E_SHAPE), (dict(k=desc(addr(1), c=12), v=desc(addr(2), c=12)), E_SHAPE),
    (dict(heads=1, **{m: desc(addr(i), c=33) for i, m in ((0, "q"), (1, "k"), (2, "v"), (3, "out"))}), E_UNSUP),
    (dict(scale=math.nan), E_SHAPE), (dict(causal=2), E_SHAPE), (dict(causal=-1), E_SHAPE), (dict(sequences=0), E_SHAPE),
    (dict(sequences=3), E_SHAPE), (dict(q_first=addr(23)), E_SHAPE), (dict(k_first=addr(23)), E_NULL),
    (one(k=desc(addr(1), n=1, w=7), v=desc(addr(2), n=1, w=7)), E_SHAPE), (one() | dict(q_first=addr(23) + 2), E_ALIGN),
    (one(k_first=addr(24) + 1), E_ALIGN), (one(sequences=1 << 25), E_UNSUP), (one(sequences=1 << 22), E_UNSUP),
    (dict(q=desc(addr(0), strides=(1536, 384, 24, 6, 1))), E_LAYOUT), (dict(q=desc(addr(0) + 1)), E_ALIGN),
    (dict(stats=addr(5) + 2), E_ALIGN), (dict(rest=addr(4) + 8), E_ALIGN),
    ({m: desc(addr(i), dtype=0) for i, m in ((0, "q"), (1, "k"), (2, "v"), (3, "out"), (6, "dout"), (7, "dq"), (8, "dk"),
                                             (9, "dv"))}, E_DTYPE),
]


@pytest.mark.parametrize("back", [False, True], ids=["forward", "backward"])
@pytest.mark.parametrize("kw,code", PACKED, ids=[f"{'-'.join(c[0])[:24]}-{i}" for i, c in enumerate(PACKED)])
def test_packed_attention_refuses(lib, kw, code, back):
    rc, msg = packed(lib, back, **kw)
    assert rc == code and msg, (kw, rc, msg)


@pytest.mark.parametrize("back,kw,code", [
    (False, dict(out=desc(addr(0))), E_ALIAS), (False, dict(out=desc(addr(2) + 64)), E_ALIAS), (False, dict(stats=addr(3)), E_ALIAS),
    (False, dict(rest=addr(1)), E_ALIAS), (False, dict(rest=addr(3)), E_ALIAS), (True, dict(dk=desc(addr(4))), E_ALIAS),
    (False, one() | dict(out=desc(addr(23), n=1)), E_ALIAS),
    (False, dict(q=desc(addr(0), c_all=64), out=desc(addr(0) + 2 * 8, c_all=64)), E_ALIAS),
    (True, dict(dout=None), E_NULL), (True, dict(dq=None), E_NULL), (True, dict(dk=None), E_NULL), (True, dict(dv=None), E_NULL),
    (True, dict(stats=None), E_NULL), (True, dict(dq=desc(addr(7), c=8)), E_SHAPE), (True, dict(dk=desc(addr(8), h=2)), E_SHAPE),
    (True, dict(dq=desc(addr(6))), E_ALIAS), (True, dict(dk=desc(addr(9))), E_ALIAS), (True, dict(dv=desc(addr(2))), E_ALIAS),
    (True, dict(dq=desc(addr(5))), E_ALIAS), (True, dict(dq=desc(addr(3))), E_ALIAS)])
def test_packed_attention_refuses_more(lib, back, kw, code):
    rc, msg = packed(lib, back, **kw)
    assert rc == code and msg, (kw, rc, msg)


def test_row_bytes(lib):
    for dq in range(1, 33):
        for form, size in ((0, 4), (1, 2), (2, 1)):
            assert lib.quan_cache_row_bytes(dq, form) == -(-4 * dq * size // 16) * 16
    assert lib.quan_cache_row_bytes(0, 2) == E_SHAPE and lib.quan_cache_row_bytes(33, 2) == E_UNSUP
    assert lib.quan_cache_row_bytes(8, 3) == E_DTYPE


def test_binding_refuses():
    table = torch.zeros((2, 3), dtype=torch.int32)
    c = quan.empty_cache(4, 8, 2, 5, table)
    assert c.keys.shape == (4, 2, 8, 32) and c.heads == 2 and c.page_tokens == 8
    k = quan.empty_qmap(2, 10, 1, 3, torch.bfloat16, "cpu")
    ints = torch.zeros(2, dtype=torch.int32)
    for bad in (c._replace(keys=c.keys[:, :, :, :16]), c._replace(values=c.values[:3]), c._replace(key_exp=None),
                c._replace(table=table.long()), c._replace(table=table[0]), c._replace(dq=9), c._replace(dq=0),
                c._replace(value_exp=c.value_exp.int()), c._replace(keys=c.keys.transpose(1, 2))):
        with pytest.raises(ValueError):
            quan.quan_cache_write(bad, k, k)
        with pytest.raises(ValueError):
            quan.quan_cache_read(bad, k, k)
        with pytest.raises(ValueError):
            quan.quan_cache_attention(k[..., :1], bad, ints, 2)
    with pytest.raises(TypeError):
        quan.quan_cache_write(c._replace(keys=c.keys.view(torch.uint8), values=c.values.view(torch.uint8)), k, k)
    for kw in (dict(start=ints.long()), dict(first=ints), dict(kv_len=ints[:1])):
        with pytest.raises(ValueError):
            quan.quan_cache_write(c, k, k, **kw)
    q = quan.empty_qmap(2, 10, 1, 1, torch.bfloat16, "cpu")
    rel = (torch.zeros(2, 3, 3), torch.zeros(3, dtype=torch.int32), torch.zeros(3, dtype=torch.int32))
    for kw in (dict(relpos=rel), dict(pos=ints), dict(out=q[0])):
        with pytest.raises(ValueError):
            quan.quan_cache_attention(q, c, ints, 2, **kw)
    for kw in (dict(first=ints.long()), dict(first=ints, k_first=ints[:1])):
        with pytest.raises(ValueError):
            quan.quan_packed_attention_forward(k, k, k, heads=2, **kw)
    with pytest.raises(ValueError):
        quan.quan_packed_attention_backward(k, k, k, k, quan.PackedSaved(torch.zeros(2, 5, 2), None), k, None, 2)


def test_reference_quantises():
    """Largest values, halves, the least exponent, against torch's 8-bit type."""
    x = np.array([[448.0, 1.0, 2.0 ** -9, 2.0 ** -10], [449.0, 3.0, 0, 0], [0.0, 0, 0, 0], [1.7, -1.8, 0.3, 2.0 ** -20],
                  [2.0 ** -149, 0, 0, 0], [np.inf, 1, 2, 3], [np.nan, 1, 2, 3], [3.4e38, 1e38, 0, 0]])
    v, e = ref.quantise(x)
    assert e.tolist() == [127, 128, 10, 119 + 1, 10, 255, 255, 247]
    assert np.isnan(v[5:7]).all() and v[0].tolist() == [448, 1, 2.0 ** -9, 0]
    rng = np.random.default_rng(1)
    x = rng.standard_normal((200, 64)).astype(np.float32) * np.exp2(rng.integers(-100, 120, (200, 1))).astype(np.float32)
    v, e = ref.quantise(x)
    y = torch.from_numpy(x) * torch.exp2(-(torch.from_numpy(e) - 127).float())[:, None]
    assert torch.equal(y.to(torch.float8_e4m3fn).double(), torch.from_numpy(v))
    assert np.abs(v).max() <= 448 and (np.abs(v).max(1) > 223).all()


def test_reference_attends():
    """Against torch in 64 bits, gradients by differentiation."""
    rng = np.random.default_rng(2)
    lq, lk = [3, 0, 5, 2], [3, 4, 7, 1]
    q, do = (rng.standard_normal((10, 4, 8)) for _ in range(2))
    k, v = (rng.standard_normal((15, 2, 8)) for _ in range(2))
    for causal in (True, False):
        res, _ = ref.packed(q, k, v, lq, lk, causal, dout=do)
        t = [torch.tensor(a, requires_grad=True) for a in (q, k, v)]
        outs = []
        for a, n, b, m in zip(ref.starts(lq), lq, ref.starts(lk), lk):
            s = torch.einsum("ihd,jhd->hij", t[0][a:a + n], t[1][b:b + m].repeat_interleave(2, 1)) / math.sqrt(8)
            if causal:
                s = s.masked_fill(torch.arange(m)[None, :] > torch.arange(n)[:, None] + m - n, -math.inf)
            outs.append(torch.einsum("hij,jhd->ihd", torch.nan_to_num(torch.softmax(s, -1)), t[2][b:b + m].repeat_interleave(2, 1)))
        out = torch.cat(outs)
        out.backward(torch.tensor(do))
        assert np.allclose(res["out"], out.detach().numpy(), atol=1e-12)
        for name, x in zip(("dq", "dk", "dv"), t):
            assert np.allclose(res[name], np.nan_to_num(x.grad.numpy()), atol=1e-12), name


def bare_block(c=8, heads=2):
    """A block without parameters: what its checks look at."""
    block = AttentionBlock.__new__(AttentionBlock)
    block.c, block.heads, block.kv, block.causal, block.dtype = c, heads, c, True, torch.bfloat16
    return block


@pytest.mark.parametrize("past", [[5], [5, 5, 5], [-1, 5], [5, 19], [18, 0], [1 << 31, 0]])
def test_extend_refuses(past):
    """Pixels behind what the cache has room for, or a number of lengths that is not the
    maps'; nothing has been computed by then."""
    block, table = bare_block(), torch.zeros((2, 3), dtype=torch.int32)
    cache = quan.empty_cache(4, 8, 2, 4, table)  # 24 positions
    x = quan.empty_qmap(2, 8, 2, 4, torch.bfloat16, "cpu")
    with pytest.raises(ValueError, match="past"):
        block.extend(cache, x, x, past)


@pytest.mark.parametrize("rows,row", [(3, 4), (7, 0), (1, 6), (1, -1)])
def test_write_refuses(rows, row):
    """Rows behind what a cache of pages has room for, or before its first; nothing has
    been computed by then."""
    block, table = bare_block(), torch.zeros((2, 3), dtype=torch.int32)
    cache = quan.empty_cache(4, 8, 2, 4, table)  # 24 positions, 6 rows of 4
    h = quan.empty_qmap(2, 8, rows, 4, torch.bfloat16, "cpu")
    with pytest.raises(ValueError, match="rows"):
        block.write(cache, h, row)
