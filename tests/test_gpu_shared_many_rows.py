"""Attention over common first pages where the rows of a group are more than 16 of a kv head, so that their parts are tiles of
many rows: far pages, replayed graphs, streams of their own, rows that see less than the prefix.  Each test reads from the
layout that pages were shared.  Tolerances: reference() of test_gpu_cache.py."""
import math

import numpy as np
import pytest
import torch

import paper_2607_07724_amd as ugbs
from gpu_helpers import bf16_to_f64, dev, dev_bf16, host_bits
from test_gpu_cache import I32, PAGE, bf16, reference
from test_gpu_shared import check, prefix_parts, run_shared, shared_contents

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need an MI355X (gfx950) visible to torch")
    ugbs.lib()


def check_against_64_bits(x, Qv, lens, q, d, O, some=None):
    """The requests `some` against 64 bits."""
    got = bf16_to_f64(host_bits(O))
    for b in some or range(len(lens)):
        want, tol = reference(x, b, Qv[b], lens[b], q[b], 1 / math.sqrt(d), True)
        assert (np.abs(got[b, :, :q[b]] - want[:, :q[b]]) <= tol[:, :q[b]]).all(), b


@pytest.mark.parametrize("d,dtype,rows", [(256, 0, 9), (256, 1, 9), (128, 0, 3), (64, 1, 2)])
def test_prefix_pages_behind_4_gib(d, dtype, rows):
    """The common pages, and the requests' own, are the last ones of a cache of 5.2e9 bytes."""
    Hkv, common = 8, 25
    n_pages = int(5.2e9) // (2 * PAGE * d * Hkv)
    g = np.random.default_rng(d + dtype)
    lens = [common * PAGE + n for n in [130, 50, 20] * 14]
    B = len(lens)
    small = shared_contents(g, lens, Hkv, d, dtype, [0] * B, {0: common})
    shift = n_pages - small.n_pages
    cache = torch.zeros((n_pages, Hkv, 2, PAGE * d), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((n_pages, Hkv, 2), dtype=torch.float32, device="cuda")
    cache[shift:], scales[shift:] = dev(small.raw), dev(small.scales)
    table = np.where(small.table >= 0, small.table + shift, -1).astype(I32)
    Qb, Qv = bf16(g.normal(0, 1, (B, 8, rows, d)))
    c = ugbs.Cache.make(B, 8, Hkv, d, n_pages, small.max_pages, rows=rows, dtype=dtype)
    O = run_shared(c, None, Qb, lens, [rows] * B, [0] * B, arrays=(cache, scales, dev(table)), shared=True)
    check_against_64_bits(small, Qv, lens, [rows] * B, d, O)


def test_more_new_tokens_than_the_common_pages_hold():
    """Requests of one page, all of it common, whose new tokens are some, all or more than its 64."""
    g = np.random.default_rng(62)
    check(g, [64] * 60, [5] * 60, 100, 24, 24, 128, 0, [0] * 60, {0: 1}, max_pages=2)
    check(g, [64] * 40, [64, 70] * 20, 80, 48, 48, 64, 1, [0] * 40, {0: 1}, max_pages=2)


@pytest.mark.parametrize("d,dtype", [(128, 0), (256, 1), (64, 0)])
def test_two_graphs_share_a_workspace_and_a_layout_as_lengths_grow(d, dtype):
    g = np.random.default_rng(46 + d)
    B, H, Hkv = 40, 16, 8
    group = [0, 1] * 20
    lens = [PAGE * (40 if n else 50) + int(g.integers(20, 900)) for n in group]
    x = shared_contents(g, [n + 40 for n in lens], Hkv, d, dtype, group, {0: 50, 1: 40}, max_pages=70)
    cache, scales, table = x.device()
    groups, kv = dev(np.array(group, I32)), dev(np.array(lens, I32))
    calls = []
    for rows in (1, 4):
        c = ugbs.Cache.make(B, H, Hkv, d, x.n_pages, 70, rows=rows, dtype=dtype)
        Qb, Qv = bf16(g.normal(0, 1, (B, H, rows, d)))
        calls.append((c, dev_bf16(Qb), dev(np.array([rows] * B, I32)), torch.zeros((B, H, rows, d), dtype=BF, device="cuda"), Qv))
    u8 = dict(dtype=torch.uint8, device="cuda")
    ws = torch.empty(max(ugbs.ugbs_cache_shared_workspace_bytes(y[0]) for y in calls), **u8)
    share = torch.empty(max(ugbs.ugbs_cache_share_bytes(y[0]) for y in calls), **u8)

    def one(c, Q, q, O, _):
        ugbs.ugbs_cache_share(c, groups, table, kv, q, share)
        ugbs.ugbs_cache_attend_shared(c, Q, cache, scales, table, kv, q, share, O, ws)
    graphs = []
    for call in calls:
        one(*call)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            one(*call)
        graphs.append(graph)
    for rep in range(5):
        kv.add_(7)                                 # (within the pages they hold)
        lens = [n + 7 for n in lens]
        for call in calls:
            call[3].fill_(3.0)
        ws.fill_(255 - rep)
        for k in (0, 1) if rep % 2 else (1, 0):
            graphs[k].replay()
            torch.cuda.synchronize()
            assert prefix_parts(calls[k][0], share[:ugbs.ugbs_cache_share_bytes(calls[k][0])]) > 0
        got = [call[3].clone() for call in calls]
        for call, w in zip(calls, got):
            one(*call)
            torch.cuda.synchronize()
            assert torch.equal(call[3].view(torch.int16), w.view(torch.int16)), rep
    for (c, _, _, _, Qv), w in zip(calls, got):
        check_against_64_bits(x, Qv, lens, [c.rows] * B, d, w, range(0, B, 7))


def test_many_rows_on_streams_of_their_own():
    g = np.random.default_rng(12)
    sides = []
    for k in range(2):
        B, H, Hkv, d, rows = 36 + 4 * k, 16, 16, 128, 2
        lens = [30 * PAGE + 100 * k + b + 2 for b in range(B)]
        x = shared_contents(g, lens, Hkv, d, k, [0] * B, {0: 30})
        Qb, Qv = bf16(g.normal(0, 1, (B, H, rows, d)))
        c = ugbs.Cache.make(B, H, Hkv, d, x.n_pages, x.max_pages, rows=rows, dtype=k)
        u8 = dict(dtype=torch.uint8, device="cuda")
        want = run_shared(c, x, Qb, lens, [rows] * B, [0] * B, shared=True)
        check_against_64_bits(x, Qv, lens, [rows] * B, d, want, range(0, B, 5))
        sides.append((c, x.device(), dev_bf16(Qb), dev(np.array(lens, I32)), dev(np.full(B, rows, I32)), dev(np.zeros(B, I32)),
                      torch.empty(ugbs.ugbs_cache_share_bytes(c), **u8), torch.empty(ugbs.ugbs_cache_shared_workspace_bytes(c), **u8),
                      want, torch.zeros((B, H, rows, d), dtype=BF, device="cuda"), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for c, (cache, scales, table), Q, kv, q, group, share, ws, _, O, stream in sides:
            with torch.cuda.stream(stream):
                O.zero_()
                ugbs.ugbs_cache_share(c, group, table, kv, q, share)
                ugbs.ugbs_cache_attend_shared(c, Q, cache, scales, table, kv, q, share, O, ws)
    torch.cuda.synchronize()
    for *_, want, O, _ in sides:
        assert torch.equal(want.view(torch.int16), O.view(torch.int16))
