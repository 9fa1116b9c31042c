"""The cache's entry points without a GPU: what they refuse, before any launch, and the oracle's own rules."""
import ctypes
import math

import numpy as np
import pytest

import cache_oracle as co
import paper_2607_07724_amd as ugbs
from test_abi_cpu import _enum

FAKE = ctypes.c_void_p(0x100000)        # never dereferenced: validation fails first


def good(**kw):
    c = ugbs.Cache.make(3, 8, 2, 128, 40, 10, rows=4)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def fake(i):
    return ctypes.c_void_p(0x100000 * (i + 1))


def call(name, c, null=None, off=None, ws=1 << 40, width=4):
    """One call with distinct fake pointers; pointer `null` NULL, pointer `off` moved by off[1] bytes."""
    n = {"plan": 9, "store": 5, "load": 7, "attend": 8}[name]
    p = [fake(i) for i in range(n)]
    if null is not None:
        p[null] = None
    if off is not None:
        p[off[0]] = ctypes.c_void_p(p[off[0]].value + off[1])
    L = ugbs.lib()
    ref = ctypes.byref(c) if c is not None else None
    if name == "plan":
        return L.ugbs_cache_plan(ref, *p, None)
    if name == "store":
        return L.ugbs_cache_store(ref, *p, None)
    if name == "load":
        return L.ugbs_cache_load(ref, *p[:5], width, *p[5:], None)
    return L.ugbs_cache_attend(ref, *p, ws, None)


BAD = [
    (dict(batch=0), "UGBS_ERR_SHAPE"),
    (dict(batch=4097), "UGBS_ERR_SHAPE"),
    (dict(n_heads=7), "UGBS_ERR_SHAPE"),
    (dict(n_kv_heads=0), "UGBS_ERR_SHAPE"),
    (dict(head_dim=96), "UGBS_ERR_SHAPE"),
    (dict(n_pages=0), "UGBS_ERR_SHAPE"),
    (dict(n_pages=(1 << 24) + 1), "UGBS_ERR_SHAPE"),
    (dict(max_pages=0), "UGBS_ERR_SHAPE"),
    (dict(max_pages=4097), "UGBS_ERR_SHAPE"),
    (dict(rows=0), "UGBS_ERR_SHAPE"),
    (dict(rows=641), "UGBS_ERR_SHAPE"),
    (dict(batch=4096, max_pages=4096, rows=262144), "UGBS_ERR_SHAPE"),
    (dict(batch=4096, n_heads=2048, n_kv_heads=2048), "UGBS_ERR_SHAPE"),
    (dict(dtype=2), "UGBS_ERR_DTYPE"),
    (dict(dtype=-1), "UGBS_ERR_DTYPE"),
    (dict(softmax_scale=-1.0), "UGBS_ERR_SCALE"),
    (dict(softmax_scale=math.nan), "UGBS_ERR_SCALE"),
]


@pytest.mark.parametrize("kw,code", BAD, ids=[str(b[0]) for b in BAD])
def test_invalid_caches_are_refused_by_every_entry_point(kw, code):
    c = good(**kw)
    for name in ("plan", "store", "load", "attend"):
        assert call(name, c) == _enum(code), name
    assert ugbs.ugbs_cache_workspace_bytes(c) == 0


def test_missing_misaligned_and_shared_arrays_are_refused():
    c = good()
    for name, n in (("plan", 9), ("store", 5), ("load", 7), ("attend", 7)):
        assert call(name, None) == _enum("UGBS_ERR_NULL")
        for i in range(n):
            assert call(name, c, null=i) == _enum("UGBS_ERR_NULL"), (name, i)
            assert call(name, c, off=(i, 2)) == _enum("UGBS_ERR_ALIGN"), (name, i)
    for name, which in (("store", (0, 1, 3)), ("load", (0, 5, 6)), ("attend", (0, 1, 6))):
        for i in which:
            assert call(name, c, off=(i, 8)) == _enum("UGBS_ERR_ALIGN"), (name, i)
    for name, i in (("store", 4), ("load", 1), ("attend", 2)):
        assert call(name, c, off=(i, 4)) == _enum("UGBS_ERR_ALIGN"), (name, i)
    L = ugbs.lib()
    for out in (5, 6, 7, 8):
        for other in range(out):
            p = [fake(i) for i in range(9)]
            p[out] = p[other]
            assert L.ugbs_cache_plan(ctypes.byref(c), *p, None) == _enum("UGBS_ERR_ALIAS"), (out, other)
    for width in (0, -1, (1 << 20) + 1):
        assert call("load", c, width=width) == _enum("UGBS_ERR_SHAPE")


def test_workspace_is_asked_for_where_parts_are_possible():
    c = good(max_pages=4096, n_pages=5000)
    need = ugbs.ugbs_cache_workspace_bytes(c)
    assert need > 0
    assert call("attend", c, ws=need - 1) == _enum("UGBS_ERR_WORKSPACE")
    assert call("attend", c, null=7) == _enum("UGBS_ERR_WORKSPACE")
    assert call("attend", c, off=(7, 128)) == _enum("UGBS_ERR_ALIGN")
    assert ugbs.ugbs_cache_workspace_bytes(good(max_pages=1)) == 0


def test_struct_and_statuses():
    assert ctypes.sizeof(ugbs.Cache) == 36 and ugbs.Cache.softmax_scale.offset == 32
    for st in (11, 12):
        assert ugbs.ugbs_status_string(st) not in ("", "unknown status")
    assert (ugbs.E4M3, ugbs.INT8) == (_enum("UGBS_E4M3"), _enum("UGBS_INT8"))


def test_binding_checks_tensors():
    """Host tensors, wrong shapes and wrong types raise before the library is called."""
    torch = pytest.importorskip("torch")
    c = good()
    z = lambda *s, dtype=torch.int32: torch.zeros(s, dtype=dtype)
    kv = z(3, 2, 4, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        ugbs.ugbs_cache_store(c, kv, kv, z(3, 4), z(40, 2, 2, 8192, dtype=torch.uint8), z(40, 2, 2, dtype=torch.float32))
    with pytest.raises(ValueError):
        ugbs.ugbs_cache_plan(c, z(4), z(3), z(40), z(1), z(3, 10), z(3), z(3), z(3, 4), z(1))
    with pytest.raises(ValueError):
        ugbs.ugbs_cache_load(c, z(40, 2, 2, 8192, dtype=torch.uint8), z(40, 2, 2, dtype=torch.float32), z(3, 10), z(3), z(3),
                             kv[0], kv[0])
    with pytest.raises(ValueError):
        ugbs.ugbs_cache_attend(c, z(3, 8, 4, 128, dtype=torch.float16), z(40, 2, 2, 8192, dtype=torch.uint8),
                               z(40, 2, 2, dtype=torch.float32), z(3, 10), z(3), z(3), z(3, 8, 4, 128, dtype=torch.bfloat16))


# ---------------------------------------------------------------- the oracle itself

def test_orders_are_permutations():
    for d in (64, 128, 256):
        for at in (co.key_at(d), co.value_at(d)):
            assert np.array_equal(np.sort(at.ravel()), np.arange(64 * d))


def test_nearest_is_nearest():
    """Against a search over all numbers of the type; ties go to the even byte."""
    g = np.random.default_rng(1)
    x = np.concatenate([g.normal(0, 100, 4000), g.normal(0, 0.01, 2000), np.ldexp(g.integers(-255, 256, 4000).astype(float), g.integers(-14, 1, 4000))])
    x = np.clip(x, -448, 448)
    for dtype in (0, 1):
        pos = np.unique(np.abs(co.NUMBERS[dtype][np.isfinite(co.NUMBERS[dtype])]))
        if dtype == 1:
            pos = pos[:128]
        y = np.clip(x, -co.TOP[dtype], co.TOP[dtype])
        i = np.clip(np.searchsorted(pos, np.abs(y)), 1, len(pos) - 1)
        lo, hi = pos[i - 1], pos[i]
        dl, dh = np.abs(y) - lo, hi - np.abs(y)
        want = np.where((dh < dl) | ((dh == dl) & (i % 2 == 0)), hi, lo) * np.sign(y)
        assert np.array_equal(co.nearest(x, dtype), want)


def test_encode_and_decode_are_inverse():
    g = np.random.default_rng(2)
    for dtype in (0, 1):
        k, v = (co.nearest(g.normal(0, 30, (2, 3, 64, 64)), dtype) for _ in range(2))
        raw = co.encode(k, v, dtype)
        sc = np.ones((2, 3, 2), np.float32)
        k2, v2 = co.decode(raw, sc, dtype, 64)
        assert np.array_equal(k, k2) and np.array_equal(v, v2)


def test_plan_small_by_hand():
    """Two pages given back by request 1 go to request 0 and 2; request 3 asks for more than is left."""
    table = np.full((4, 4), -1, np.int32)
    table[0, 0], table[1, :2], table[3, 0] = 7, (5, 6), 3
    stack, tb, kv, q, slots, left = co.plan([64, 70, 0, 10], [2, -1, 1, 118], np.array([9, 8, 0, 0, 0, 0, 0, 0, 0, 0]), 1, table, 118)
    assert list(stack[:3]) == [9, 5, 6] and left == 0
    assert tb[0].tolist() == [7, 6, -1, -1] and tb[2, 0] == 5 and tb[3].tolist() == [3, 9, -1, -1]
    assert kv.tolist() == [66, 0, 1, 128] and q.tolist() == [2, 0, 1, 118]
    assert slots[0, :3].tolist() == [384, 385, -1] and slots[3, :2].tolist() == [202, 203] and slots[3, 117] == 9 * 64 + 63
