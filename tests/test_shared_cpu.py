"""Attention over common first pages, without a GPU: what the entry points refuse, before any launch, and the sizes."""
import ctypes

import pytest

import paper_2607_07724_amd as ugbs
from test_abi_cpu import _enum
from test_cache_cpu import BAD, fake, good


def share(c, null=None, off=None, nbytes=1 << 40):
    p = [fake(i) for i in range(5)]
    if null is not None:
        p[null] = None
    if off is not None:
        p[off] = ctypes.c_void_p(p[off].value + 2)
    return ugbs.lib().ugbs_cache_share(None if c is None else ctypes.byref(c), *p, nbytes, None)


def attend(c, null=None, off=None, nbytes=1 << 40, ws=1 << 40):
    p = [fake(i) for i in range(9)]
    if null is not None:
        p[null] = None
    if off is not None:
        p[off] = ctypes.c_void_p(p[off].value + 2)
    return ugbs.lib().ugbs_cache_attend_shared(None if c is None else ctypes.byref(c), *p[:7], nbytes, *p[7:], ws, None)


@pytest.mark.parametrize("kw,code", BAD, ids=[str(b[0]) for b in BAD])
def test_invalid_caches_are_refused(kw, code):
    c = good(**kw)
    assert share(c) == _enum(code) and attend(c) == _enum(code)
    assert ugbs.ugbs_cache_share_bytes(c) == 0 and ugbs.ugbs_cache_shared_workspace_bytes(c) == 0


def test_missing_misaligned_and_short_arrays_are_refused():
    c = good()
    assert share(None) == _enum("UGBS_ERR_NULL") and attend(None) == _enum("UGBS_ERR_NULL")
    for i in range(4):
        assert share(c, null=i) == _enum("UGBS_ERR_NULL")
    for i in (0, 1, 2, 3, 4, 5, 7):
        assert attend(c, null=i) == _enum("UGBS_ERR_NULL"), i
    assert share(c, null=4) == _enum("UGBS_ERR_WORKSPACE")
    assert attend(c, null=6) == _enum("UGBS_ERR_WORKSPACE") and attend(c, null=8) == _enum("UGBS_ERR_WORKSPACE")
    for i in range(5):
        assert share(c, off=i) == _enum("UGBS_ERR_ALIGN"), i
    for i in range(9):
        assert attend(c, off=i) == _enum("UGBS_ERR_ALIGN"), i
    need, ws = ugbs.ugbs_cache_share_bytes(c), ugbs.ugbs_cache_shared_workspace_bytes(c)
    assert share(c, nbytes=need - 1) == _enum("UGBS_ERR_WORKSPACE")
    assert attend(c, nbytes=need - 1) == _enum("UGBS_ERR_WORKSPACE")
    assert attend(c, ws=ws - 1) == _enum("UGBS_ERR_WORKSPACE")


@pytest.mark.parametrize("B,H,Hkv,d,rows", [(2, 4, 1, 64, 1), (64, 32, 8, 128, 1), (40, 16, 2, 256, 4), (4096, 32, 8, 128, 1), (300, 8, 2, 64, 16)])
def test_sizes_hold_the_sums_of_every_row(B, H, Hkv, d, rows):
    """Every row of a group has sums of at least two parts."""
    c = ugbs.Cache.make(B, H, Hkv, d, 1000, 100, rows=rows)
    assert ugbs.ugbs_cache_share_bytes(c) % 256 == 0
    ws = ugbs.ugbs_cache_shared_workspace_bytes(c)
    assert ws >= 2 * B * H * rows * (4 * d + 8)
    assert ws <= (2 * B * H * rows + 512 * 64) * (4 * d + 8)
    # rows that fill tiles of their own: the plain call's workspace
    many = ugbs.Cache.make(B, H, Hkv, d, 1000, 100, rows=128 * Hkv // H + 1)
    assert ugbs.ugbs_cache_shared_workspace_bytes(many) == ugbs.ugbs_cache_workspace_bytes(many)
