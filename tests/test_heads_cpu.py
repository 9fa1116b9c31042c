"""From a projection's rows to heads, without a GPU: what the entry points refuse, before any launch."""
import ctypes
import math

import pytest
import torch

import paper_2607_07724_amd as ugbs
from test_abi_cpu import _enum


class Rows(ctypes.Structure):
    """Mirror of ugbs_rows."""
    _fields_ = [("at", ctypes.c_void_p), ("batch", ctypes.c_int64), ("token", ctypes.c_int64), ("head", ctypes.c_int64)]


def fake(i):
    return ctypes.c_void_p(0x100000 * (i + 1))        # never dereferenced: validation fails first


def good(**kw):
    h = ugbs.Heads.make(3, 8, 2, 128, rows=4, rot=64, axes=3)
    for k, v in kw.items():
        setattr(h, k, v)
    return h


def cache(**kw):
    c = ugbs.Cache.make(3, 8, 2, 128, 40, 10, rows=4)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


ARRAYS = ("q_norm", "k_norm", "freqs", "positions", "axis", "first", "lens", "Q")
OPTIONAL = ("q_norm", "k_norm", "positions", "axis", "first", "lens")


def call(store, h, c=None, null=None, off=None, stride=None, rows_null=None):
    """One call; array `null` is NULL, `off` moved by 2 bytes, rows `stride[0]` have stride[1] for field stride[2]."""
    more = ("slots", "cache", "scales") if store else ("K", "V")
    p = {n: fake(i) for i, n in enumerate(ARRAYS + more)}
    rows = {n: Rows(0x9000000 + 0x100000 * i, 4096, 1024, 128) for i, n in enumerate("qkv")}
    if null in rows:
        rows[null].at = None
    elif null:
        p[null] = None
    if off in rows:
        rows[off].at += 2
    elif off:
        p[off] = ctypes.c_void_p(p[off].value + 2)
    if stride:
        setattr(rows[stride[0]], stride[2], stride[1])
    L = ugbs.lib()
    r = [None if n == rows_null else ctypes.byref(x) for n, x in rows.items()]
    a = [p[n] for n in ARRAYS]
    hp = None if h is None else ctypes.byref(h)
    if store:
        return L.ugbs_heads_store(hp, None if c is None else ctypes.byref(c), *r, *a, p["slots"], p["cache"], p["scales"], None)
    return L.ugbs_heads_split(hp, *r, *a, p["K"], p["V"], None)


BAD = [
    (dict(batch=0), "UGBS_ERR_SHAPE"),
    (dict(batch=4097), "UGBS_ERR_SHAPE"),
    (dict(n_heads=7), "UGBS_ERR_SHAPE"),
    (dict(n_heads=0), "UGBS_ERR_SHAPE"),
    (dict(n_kv_heads=0), "UGBS_ERR_SHAPE"),
    (dict(n_heads=4096, n_kv_heads=1), "UGBS_ERR_SHAPE"),
    (dict(head_dim=96), "UGBS_ERR_SHAPE"),
    (dict(rows=0), "UGBS_ERR_SHAPE"),
    (dict(rows=(1 << 23) // 3 + 1), "UGBS_ERR_SHAPE"),
    (dict(rot_dim=-16), "UGBS_ERR_ROTARY"),
    (dict(rot_dim=144), "UGBS_ERR_ROTARY"),
    (dict(rot_dim=24), "UGBS_ERR_ROTARY"),
    (dict(pairs=2), "UGBS_ERR_ROTARY"),
    (dict(pairs=-1), "UGBS_ERR_ROTARY"),
    (dict(axes=0), "UGBS_ERR_ROTARY"),
    (dict(axes=5), "UGBS_ERR_ROTARY"),
    (dict(norm_eps=-1e-6), "UGBS_ERR_ROTARY"),
    (dict(norm_eps=math.nan), "UGBS_ERR_ROTARY"),
    (dict(norm_eps=math.inf), "UGBS_ERR_ROTARY"),
    (dict(rot_gain=math.nan), "UGBS_ERR_ROTARY"),
    (dict(rot_gain=math.inf), "UGBS_ERR_ROTARY"),
]


@pytest.mark.parametrize("kw,code", BAD, ids=[str(b[0]) for b in BAD])
def test_invalid_heads_are_refused_by_both_entry_points(kw, code):
    assert call(False, good(**kw)) == _enum(code)
    assert call(True, good(**kw), cache()) == _enum(code)


def test_missing_and_misaligned_arrays_are_refused():
    for store in (False, True):
        c = cache()
        assert call(store, None, c) == _enum("UGBS_ERR_NULL")
        for n in "qkv":
            assert call(store, good(), c, rows_null=n) == _enum("UGBS_ERR_NULL")
        names = tuple("qkv") + ARRAYS + (("slots", "cache", "scales") if store else ("K", "V"))
        for n in names:
            if n not in OPTIONAL:
                assert call(store, good(), c, null=n) == _enum("UGBS_ERR_NULL"), n
            assert call(store, good(), c, off=n) == _enum("UGBS_ERR_ALIGN"), n
    assert call(True, good(), None) == _enum("UGBS_ERR_NULL")


def test_strides_that_break_the_alignment_are_refused():
    for store in (False, True):
        for n in "qkv":
            for field in ("batch", "token", "head"):
                assert call(store, good(), cache(), stride=(n, 132, field)) == _enum("UGBS_ERR_STRIDE")


def test_a_cache_of_another_batch_is_refused():
    for kw in (dict(batch=2), dict(n_heads=4), dict(n_kv_heads=4), dict(head_dim=64), dict(rows=5)):
        assert call(True, good(), cache(**kw)) == _enum("UGBS_ERR_SHAPE"), kw
    assert call(True, good(), cache(dtype=7)) == _enum("UGBS_ERR_DTYPE")


def test_struct_layouts_match_the_header():
    assert ctypes.sizeof(ugbs.Heads) == 40 and ugbs.Heads.norm_eps.offset == 32
    assert ctypes.sizeof(ugbs._Views) == 3 * ctypes.sizeof(Rows) and Rows.head.offset == 24


def test_python_refuses_tensors_that_are_not_rows():
    h = ugbs.Heads.make(1, 2, 1, 64, rows=3)
    x = torch.zeros((1, 3, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device tensor"):
        ugbs.ugbs_heads_split(h, x, x, x, None, x, x, x)
    with pytest.raises(ValueError, match="device tensor"):
        ugbs.ugbs_heads_split(h, None, x, x, None, x, x, x)
    ugbs._get_torch()
    cpu = x.get_device()
    assert ugbs._rows_of("Xq", x, (1, 3, 2, 64), cpu) == (x.data_ptr(), 0, 128, 64)
    for bad, why in ((x.transpose(1, 2), "shape"), (x.float(), "dtype"), (x[..., ::1].transpose(2, 3).contiguous().transpose(2, 3), "channels")):
        with pytest.raises(ValueError, match=why):
            ugbs._rows_of("Xq", bad, (1, 3, 2, 64), cpu)
    with pytest.raises(ValueError, match="required"):
        ugbs._rows_of("Xq", None, (1, 3, 2, 64), cpu)
    with pytest.raises(ValueError, match="is on"):
        ugbs._rows_of("Xq", x, (1, 3, 2, 64), 0)
