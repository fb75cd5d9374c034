"""With a bias, calls whose offsets do not fit in a work-group's LDS are refused
on the host; every other one gets past that check.  (Made-up addresses: those
others are told from an output that lies on an input, which is looked at last,
so that nothing is launched.)"""
import ctypes
import os

import pytest

from paper_2509_05512_amd import quan

E_ALIAS, E_UNSUP = -5, -6
LDS = 160 * 1024
BF, F32 = 1, 0


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(quan.LIB_PATH):
        pytest.skip("libquan.so not built")
    return quan.load_library()


def addr(i):
    return 0x1000000000 * (i + 1)


def desc(i, c, hw, dtype, n=1):
    h, w = hw
    return quan.QuanTensor(addr(i), dtype, 5, (ctypes.c_int64 * 5)(n, 4, c, h, w),
                           (ctypes.c_int64 * 5)(h * w * 4 * c, c, 1, w * 4 * c, 4 * c))


class QuanRelpos(ctypes.Structure):
    """struct quan_relpos"""
    _fields_ = [(m, ctypes.c_void_p) for m in ("table", "bucket_y", "bucket_x")] \
        + [(m, ctypes.c_int32) for m in ("buckets_y", "buckets_x", "radius_y", "radius_x")]


def call(lib, q_hw, k_hw, dq, dtype, what, n=1, heads=1, buckets=4):
    """what: "forward", "save", "backward" (without dtable) or "dtable"; the
    outputs lie on q."""
    q, k, v, out, dout = (desc(i, heads * dq, hw, dtype, n) for i, hw in enumerate((q_hw, k_hw, k_hw, q_hw, q_hw)))
    rp = QuanRelpos(addr(20), addr(21), addr(22), buckets, 4, 8, 8)

    def ref(d):
        return ctypes.byref(d)
    first = [ref(q), ref(k), ref(v), ref(rp), None, None, 0.1, heads]
    if what in ("forward", "save"):
        return lib.quan_attention_forward(*first, ref(desc(0, heads * dq, q_hw, dtype, n)), None, addr(10) if what == "save" else None,
                                          None)
    grads = [ref(desc(0, heads * dq, q_hw, dtype, n)), ref(desc(11, heads * dq, k_hw, dtype, n)), ref(desc(12, heads * dq, k_hw, dtype, n))]
    return lib.quan_attention_backward(*first, ref(out), None, addr(10), ref(dout), *grads,
                                       addr(13) if what == "dtable" else None, None)


def places(hw, pitch):
    h, w = hw
    return [t // w * pitch + t % w for t in range(h * w)]


def widest(a, block):
    return max(a[min(i + block, len(a)) - 1] - a[i] for i in range(0, len(a), block))


def need(q_hw, k_hw, dq, dtype, what):
    """LDS bytes at least: the offsets of every block and tile that there are
    (their first's and last's places), and the tiles."""
    pitch = q_hw[1] + k_hw[1] - 1
    q, k = places(q_hw, pitch), places(k_hw, pitch)
    d = 4 * (8 if dq <= 8 else 16 if dq <= 16 else 32)
    tile, row = (64, 2 * d) if dtype == BF else (32, 4 * (d + 4))
    tiles = 4 * tile * row + 8 * tile
    by_q = widest(q, 128) + widest(k, tile) + 1
    by_k = widest(k, 128) + widest(q, tile) + 1
    needs = {"forward": tiles + 4 * by_q, "backward": max(tiles + 4 * by_q, tiles + 24 * tile + 4 * by_k),
             "dtable": max(tiles + 12 * by_q, tiles + 24 * tile + 4 * by_k)}
    needs["save"] = max(needs["forward"], needs["backward"])
    return needs[what]


WHAT = ["forward", "save", "backward", "dtable"]


@pytest.mark.parametrize("what", WHAT)
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("dq", [5, 16, 32])
def test_what_does_not_fit_is_refused(lib, dq, dtype, what):
    refused = taken = 0
    for q_hw in ((1, 2), (1, 500), (2, 1), (128, 1), (64, 4), (16, 4), (8, 8), (16, 8), (16, 16), (3, 300), (2, 1792)):
        for k_hw in ((1, 1), (1, 1000), (300, 1), (128, 2), (7, 33), (16, 128), (8, 256), (5, 512), (16, 1024), (4, 1792)):
            for a, b in ((q_hw, k_hw), (k_hw, q_hw)):
                if a == (1, 1) and what == "forward":  # one query: a form without tiles
                    continue
                rc = call(lib, a, b, dq, dtype, what)
                bytes_ = need(a, b, dq, dtype, what)
                assert rc in (E_ALIAS, E_UNSUP), (a, b, rc, lib.quan_last_error())
                if rc == E_UNSUP:
                    refused += 1
                    assert b"fit" in lib.quan_last_error()
                    # (a block's rows may end one sooner than the rule takes it to)
                    assert 2 * bytes_ > LDS, (a, b, bytes_)
                else:
                    taken += 1
                    assert bytes_ <= LDS, (a, b, bytes_)
    assert refused and taken


@pytest.mark.parametrize("what", WHAT)
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("dq", [8, 32])
def test_maps_of_one_width_are_taken(lib, dq, dtype, what):
    for h, w in ((1, 1), (1, 100000), (2, 1792), (50, 1792), (2000, 1), (64, 64), (130, 129), (1000, 3)):
        for hk in (1, h, 3 * h):
            assert call(lib, (h, w), (hk, w), dq, dtype, what) == E_ALIAS or w > 1792, (h, w, hk, lib.quan_last_error())


@pytest.mark.parametrize("q_hw,k_hw,dq,what", [
    ((16, 8), (256, 512), 32, "dtable"), ((16, 16), (16, 1024), 16, "dtable"), ((64, 4), (8, 512), 32, "forward"),
    ((16, 4), (16, 1024), 16, "dtable"), ((128, 1), (128, 128), 8, "dtable"), ((128, 1), (128, 256), 16, "forward")])
def test_examples(lib, q_hw, k_hw, dq, what):
    """Calls that asked for more than 160 KiB; taken where the offsets alone,
    not rounded up to a power of two, fit."""
    rc = call(lib, q_hw, k_hw, dq, BF, what)
    assert rc == (E_UNSUP if need(q_hw, k_hw, dq, BF, what) + 3000 > LDS else E_ALIAS), need(q_hw, k_hw, dq, BF, what)
    assert call(lib, (8, 8), (64, 512), 32, BF, "dtable") == E_ALIAS
    assert call(lib, (16, 4), (16, 1024), 16, BF, "dtable") == E_UNSUP


# (n, heads, queries, keys, buckets): a launch's axis has less than 2^32 lanes, 256
# to a work-group of 128 queries or keys of a head and image
@pytest.mark.parametrize("what", WHAT)
@pytest.mark.parametrize("n,heads,q_hw,k_hw,buckets,limited", [
    (16777208, 1, (1, 1), (1, 1), 4, ()), (16777209, 1, (1, 1), (1, 1), 4, WHAT),
    (2097151, 8, (1, 128), (1, 128), 4, ()), (2097151, 8, (1, 129), (1, 129), 4, WHAT),
    (2097151, 8, (1, 1), (1, 129), 4, ("backward", "dtable")),
    (1, 1, (1, 1), (1, 16777216), 4, ()),
    (1, 8191, (1, 2), (1, 2), 1024, ()), (1, 8192, (1, 2), (1, 2), 1024, ("dtable",))])
def test_launches_of_too_many_work_groups(lib, n, heads, q_hw, k_hw, buckets, limited, what):
    rc = call(lib, q_hw, k_hw, 2, BF, what, n, heads, buckets)
    assert rc == (E_UNSUP if what in limited else E_ALIAS), lib.quan_last_error()


@pytest.mark.parametrize("what", ["forward", "dtable"])
@pytest.mark.parametrize("shape,strides", [
    ((1, 4, 8, 1, 1 << 24), (1 << 60, 8, 1, 1 << 60, 1 << 40)),     # pixels of an image: 2^64 elements
    ((1 << 15, 4, 8, 1, 1 << 12), (1 << 40, 8, 1, 1 << 30, 32)),    # images: 2^55
    ((1, 4, 8, 1 << 12, 1 << 12), (1 << 60, 8, 1, 1 << 40, 1 << 28)),
    ((1, 4, 8, 1, 1 << 20), (1 << 60, 1 << 38, 1, 1 << 60, 1 << 40))])
def test_strides_beyond_any_memory(lib, shape, strides, what):
    """What they span does not fit in 64 bits, or in any memory: refused, with
    nothing computed from it."""
    n, _, c, h, w = shape
    dense = (h * w * 4 * c, c, 1, w * 4 * c, 4 * c)

    def t(i, s):
        return quan.QuanTensor(addr(i) * 1000, BF, 5, (ctypes.c_int64 * 5)(*shape), (ctypes.c_int64 * 5)(*s))
    for wide in ("q", "k", "out"):
        q, k, v, out, dout, dq, dk, dv = (t(i, strides if name == wide else dense) for i, name in
                                          enumerate(("q", "k", "v", "out", "dout", "dq", "dk", "dv")))
        first = [ctypes.byref(q), ctypes.byref(k), ctypes.byref(v), None, None, None, 0.1, 1]
        if what == "forward":
            rc = lib.quan_attention_forward(*first, ctypes.byref(out), None, 2, None)
        else:
            rc = lib.quan_attention_backward(*first, ctypes.byref(out), None, 2, ctypes.byref(dout), ctypes.byref(dq),
                                             ctypes.byref(dk), ctypes.byref(dv), None, None)
        assert rc == E_UNSUP and b"2^48" in lib.quan_last_error(), (wide, rc, lib.quan_last_error())
