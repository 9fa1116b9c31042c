"""Attention over common first pages on the GPU against the 64-bit oracle (cache_oracle.py); tolerances: reference() of
test_gpu_cache.py (the parts of a prefix are parts like others).  Whether pages were shared is read from the layout: few common
pages are not (up to 16 rows of a kv head in all, any are)."""
import math

import numpy as np
import pytest
import torch

import paper_2607_07724_amd as ugbs
from gpu_helpers import bf16_to_f64, dev, dev_bf16, host_bits
from test_gpu_cache import I32, PAGE, Contents, bf16, pages, reference
from test_gpu_shared_layout import OF_PREFIX, align

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need an MI355X (gfx950) visible to torch")
    ugbs.lib()


def shared_contents(g, lens, Hkv, d, dtype, group, common, max_pages=None):
    """Contents in which the first common[n] pages (as far as they are full) of every request of group n are those of its first one."""
    first, take = {}, []
    for b, n in enumerate(group):
        lead = first.setdefault(n, b) if n in common else b
        take.append(0 if lead == b else min(common[n], lens[b] // PAGE, lens[lead] // PAGE))
    x = Contents(g, [n - PAGE * t for n, t in zip(lens, take)], Hkv, d, dtype, max_pages=max(pages(n) for n in lens))
    for b, t in enumerate(take):
        if t:
            x.table[b] = np.concatenate([x.table[first[group[b]], :t], x.table[b, :x.max_pages - t]])
    if max_pages:
        x.table = np.concatenate([x.table, np.full((len(lens), max_pages - x.max_pages), -1, I32)], 1)
        x.max_pages = max_pages
    x.lens = list(lens)
    return x


def prefix_parts(c, share):
    """Parts of common pages in a layout (cache_attend.h, Share)."""
    B, G = c.batch, c.n_heads // c.n_kv_heads
    parts = share[2 * align(32 * B):len(share) - align(16 * B) - align(8 * B * c.rows * G)].view(torch.int32)
    parts = parts[:parts.numel() // 8 * 8].view(-1, 8)
    return int(((parts[:, 0] >= 0) & (parts[:, 0] < B) & (parts[:, 1] >= OF_PREFIX)).sum())


def run_shared(c, x, Qb, kv, q, group, fill=7.0, arrays=None, shared=None):
    cache, scales, table = arrays or x.device()
    u8 = dict(dtype=torch.uint8, device="cuda")
    O = torch.full(Qb.shape, fill, dtype=torch.bfloat16, device="cuda")
    ws = torch.full((max(256, ugbs.ugbs_cache_shared_workspace_bytes(c)),), 255, **u8)      # contents do not matter
    share = torch.full((ugbs.ugbs_cache_share_bytes(c),), 255, **u8)
    kv, q = dev(np.array(kv, I32)), dev(np.array(q, I32))
    ugbs.ugbs_cache_share(c, dev(np.array(group, I32)), table, kv, q, share)
    ugbs.ugbs_cache_attend_shared(c, dev_bf16(Qb), cache, scales, table, kv, q, share, O, ws)
    torch.cuda.synchronize()
    if shared is not None:
        assert (prefix_parts(c, share) > 0) == shared
    return O


def check(g, lens, q, rows, H, Hkv, d, dtype, group, common, max_pages=None, spoil=None, temper=1.0, shared=True):
    x = shared_contents(g, lens, Hkv, d, dtype, group, common, max_pages)
    if spoil:
        spoil(x)
    B = len(lens)
    Qb, Qv = bf16(g.normal(0, temper, (B, H, rows, d)))
    for b in range(B):
        Qb[b, :, q[b]:] = 0x7FC0                   # rows without a token are not read
    c = ugbs.Cache.make(B, H, Hkv, d, x.n_pages, x.max_pages, rows=rows, dtype=dtype)
    O = run_shared(c, x, Qb, lens, q, group, shared=shared)
    got = bf16_to_f64(host_bits(O))
    tiles = B * rows * H // Hkv > (32 if d < 256 else 16)
    for b in range(B):
        want, tol = reference(x, b, Qv[b], lens[b], q[b], 1 / math.sqrt(d), tiles)
        off = np.abs(got[b, :, :q[b]] - want[:, :q[b]])
        assert (off <= tol[:, :q[b]]).all(), (b, float((off - tol[:, :q[b]]).max()), np.argwhere(~(off <= tol[:, :q[b]]))[:3])
        assert (got[b, :, q[b]:] == 7.0).all(), b
    return O


KINDS = [(64, 0), (128, 0), (128, 1), (256, 0), (256, 1), (64, 1)]


@pytest.mark.parametrize("B,H,Hkv,common,d,dtype", [
    (*size, *kind) for size, kinds in (
        ((2, 1, 1, 5), KINDS), ((3, 4, 1, 5), KINDS), ((4, 8, 2, 5), KINDS),      # one tile of 16 rows
        ((64, 8, 8, 12), KINDS),                                                  # one of 64 (two of 32)
        ((20, 16, 16, 18), [(64, 0), (128, 1)]), ((33, 12, 12, 16), [(128, 0), (256, 1)]),      # one of 20 rows, of 33
        ((72, 8, 8, 12), [(64, 1), (128, 0), (256, 0)]),                          # 8 rows in the last one
        ((40, 32, 4, 50), [(128, 0)]), ((24, 56, 8, 42), [(64, 0), (128, 1)])) for kind in kinds])
def test_one_prefix_and_tails_of_every_length(B, H, Hkv, common, d, dtype):
    g = np.random.default_rng(B * d + dtype)
    tails = [1, 64, 63, 65, 2, 130, 31, 129, 300]
    lens = [common * PAGE + tails[b % 9] for b in range(B)]
    check(g, lens, [1] * B, 1, H, Hkv, d, dtype, [3] * B, {3: common})


@pytest.mark.parametrize("d,dtype,H,Hkv,rows", [(128, 0, 16, 8, 1), (64, 1, 16, 8, 3), (256, 1, 16, 8, 4), (128, 1, 28, 4, 2), (64, 0, 16, 16, 16),
                                                (128, 0, 16, 8, 16), (256, 0, 16, 8, 8), (64, 1, 32, 8, 16)])
def test_groups_among_each_other_and_requests_alone(d, dtype, H, Hkv, rows):
    g = np.random.default_rng(d + rows)
    B = 44
    group = g.integers(-1, 4, B)
    group[:3] = (9, 1, 1)                          # a group of one
    common = {int(n): int(g.integers(60, 110)) for n in set(group.tolist()) if n >= 0}
    common[3] = 130
    lens = [PAGE * common.get(int(n), 0) + rows + int(g.integers(0, 400)) for n in group]
    q = g.integers(max(1, rows // 2), rows + 1, B)
    q[1:3] = rows
    q[5::7] = 0
    check(g, lens, q.tolist(), rows, H, Hkv, d, dtype, group.tolist(), common)


@pytest.mark.parametrize("B,H,Hkv,d,dtype,prefix,tail", [
    (3, 4, 1, 128, 0, 9000, 100), (16, 8, 8, 128, 0, 5000, 3000), (40, 8, 2, 64, 1, 6000, 50), (7, 16, 8, 256, 1, 8000, 700),
    (24, 28, 4, 128, 0, 5000, 200), (2, 2, 2, 64, 0, 20000, 5), (4, 16, 4, 64, 1, 90000, 300)])
def test_long_prefixes_are_split_and_joined(B, H, Hkv, d, dtype, prefix, tail):
    g = np.random.default_rng(prefix)
    n = prefix // PAGE
    lens = [n * PAGE + 1 + int(g.integers(0, tail)) for _ in range(B)]
    check(g, lens, [1] * B, 1, H, Hkv, d, dtype, [0] * B, {0: n}, temper=2.0)


@pytest.mark.parametrize("B,d,dtype", [(300, 64, 0), (1030, 64, 1), (4096, 64, 0)])
def test_large_batches(B, d, dtype):
    """More requests than a wave, than the plan's threads, and the most there may be; groups of two to many, far apart."""
    g = np.random.default_rng(B)
    Hkv = 12 if B == 300 else 4 if B == 1030 else 1
    group = g.integers(-1, 40, B)
    group[-1] = group[0] = 77
    common = {n: int(g.integers(1, 4)) for n in range(40)} | {77: 30}
    lens = [PAGE * common.get(int(n), 0) + 1 + int(g.integers(0, 60)) for n in group]
    check(g, lens, [1] * B, 1, Hkv, Hkv, d, dtype, group.tolist(), common)


def test_what_is_shared_goes_by_the_tables_alone():
    """Groups whose tables have nothing, less than their pages, or all in common; numbers of groups of any size."""
    g = np.random.default_rng(5)
    big = 2 ** 31 - 1
    check(g, [300, 400, 500], [1] * 3, 1, 8, 2, 128, 0, [big] * 3, {}, shared=False)
    check(g, [600, 700, 601, 900], [1] * 4, 1, 8, 2, 128, 0, [0, 0, big, big], {0: 3, big: 9})
    # equal tables to the last entry: the pages that are not full for all are each request's own
    check(g, [640, 640, 640], [1] * 3, 1, 8, 2, 128, 0, [0] * 3, {0: 10})
    check(g, [640, 320, 641], [1, 1, 1], 1, 8, 2, 128, 0, [0] * 3, {0: 5})
    # few common pages among many rows: laid out alone
    check(g, [500] * 20, [1] * 20, 1, 8, 2, 128, 0, [0] * 20, {0: 2}, shared=False)


@pytest.mark.parametrize("d,H,Hkv,rows,B", [(64, 1, 1, 4, 3), (64, 16, 16, 5, 40), (128, 20, 20, 16, 44), (256, 16, 16, 7, 44)])
def test_new_tokens_within_the_common_pages(d, H, Hkv, rows, B):
    """Rows that do not see all of the prefix: requests of one prompt whose drafts reach into it."""
    g = np.random.default_rng(6)
    lens = [14 * PAGE, 14 * PAGE, 14 * PAGE + 3] * (B // 3) + [3] * (B - B // 3 * 3)
    q = [rows, 1, rows] * (B // 3) + [rows] * (B - B // 3 * 3)
    check(g, lens, q, rows, H, Hkv, d, 0, [0] * (B // 3 * 3) + [-1] * (B - B // 3 * 3), {0: 14})


def test_more_new_tokens_than_cached_ones():
    g = np.random.default_rng(61)
    check(g, [64, 64, 64], [5, 5, 5], 5, 1, 1, 128, 0, [0] * 3, {0: 1})
    check(g, [64] * 60, [5] * 60, 100, 1, 1, 128, 0, [0] * 60, {0: 1}, max_pages=2, shared=None)
    check(g, [64] * 40, [64, 70] * 20, 80, 1, 1, 64, 1, [0] * 40, {0: 1}, max_pages=2, shared=None)


@pytest.mark.parametrize("B,H,Hkv", [(4, 8, 2), (48, 16, 16)])
def test_entries_that_are_no_page_are_left_out(B, H, Hkv):
    g = np.random.default_rng(7)

    def spoil(x):
        x.table[:, 2] = -1
        x.table[:, 3] = x.n_pages
        x.table[1, 11] = -5
    check(g, [900] * B, [1] * B, 1, H, Hkv, 128, 0, [0] * B, {0: 11}, spoil=spoil)

    def all_gone(x):
        x.table[:] = -1
    check(g, [900] * B, [1] * B, 1, H, Hkv, 128, 1, [0] * B, {}, spoil=all_gone)


@pytest.mark.parametrize("n,H,Hkv", [(1, 2, 2), (12, 16, 16)])
def test_requests_without_new_tokens_are_left_as_they_are(n, H, Hkv):
    g = np.random.default_rng(8)
    check(g, [500, 0, 700, 600, 64 * 14] * n, [1, 0, 0, 1, 1] * n, 1, H, Hkv, 128, 0, [0] * 5 * n, {0: 0}, max_pages=15, shared=False)
    check(g, [900] * 5 * n, [0] * 5 * n, 1, H, Hkv, 128, 0, [0] * 5 * n, {0: 14}, shared=False)
    # the leader is the first request that has any
    check(g, [900] * 5 * n, [0, 0, 2, 1, 2] * n, 2, H, Hkv, 128, 0, [4] * 5 * n, {4: 14})


@pytest.mark.parametrize("B,rows,H,Hkv,d", [(1, 1, 8, 2, 128), (3, 70, 4, 1, 128), (2, 65, 2, 1, 64), (2, 90, 16, 2, 256)])
def test_where_nothing_is_shared_the_call_is_the_plain_one(B, rows, H, Hkv, d):
    g = np.random.default_rng(rows)
    lens = [500] * B
    x = shared_contents(g, lens, Hkv, d, 0, [0] * B, {0: 4})
    Qb, _ = bf16(g.normal(0, 1, (B, H, rows, d)))
    c = ugbs.Cache.make(B, H, Hkv, d, x.n_pages, x.max_pages, rows=rows)
    O = run_shared(c, x, Qb, lens, [rows] * B, [0] * B)
    cache, scales, table = x.device()
    want = torch.zeros_like(O)
    ugbs.ugbs_cache_attend(c, dev_bf16(Qb), cache, scales, table, dev(np.array(lens, I32)), dev(np.array([rows] * B, I32)), want,
                           torch.empty(max(256, ugbs.ugbs_cache_workspace_bytes(c)), dtype=torch.uint8, device="cuda"))
    assert torch.equal(O.view(torch.int16), want.view(torch.int16))


@pytest.mark.parametrize("rows,H,Hkv,d,dtype", [(20, 8, 2, 128, 0), (32, 8, 2, 64, 1), (17, 4, 1, 256, 0), (33, 3, 1, 128, 1)])
def test_requests_of_several_tiles(rows, H, Hkv, d, dtype):
    """66 to 128 rows of a kv head: a request's own pages are read by several tiles."""
    g = np.random.default_rng(rows + d)
    lens = [160 * PAGE + int(n) for n in g.integers(rows, 300, 14)]
    check(g, lens, [rows] * 11 + [1, rows - 1, 0], rows, H, Hkv, d, dtype, [0] * 13 + [-1], {0: 160})


@pytest.mark.parametrize("B,H,Hkv,rows,d,shared", [(4, 4, 1, 1, 64, True), (20, 16, 16, 1, 128, True), (70, 8, 8, 1, 128, True), (24, 28, 4, 2, 64, False),
                                                   (72, 8, 8, 1, 64, True), (40, 16, 8, 4, 256, True)])
def test_a_request_whose_queries_are_not_finite_leaves_its_group_alone(B, H, Hkv, rows, d, shared):
    g = np.random.default_rng(B)
    lens = [40 * PAGE + rows + int(g.integers(0, 200)) for _ in range(B)]
    x = shared_contents(g, lens, Hkv, d, 0, [0] * B, {0: 40})
    Qb, Qv = bf16(g.normal(0, 1, (B, H, rows, d)))
    Qb[1], Qb[B // 2] = 0x7FC0, 0x7F80
    c = ugbs.Cache.make(B, H, Hkv, d, x.n_pages, x.max_pages, rows=rows)
    got = bf16_to_f64(host_bits(run_shared(c, x, Qb, lens, [rows] * B, [0] * B, shared=shared)))
    for b in sorted(set(range(B)) - {1, B // 2}):
        want, tol = reference(x, b, Qv[b], lens[b], rows, 1 / math.sqrt(d), B * rows * H // Hkv > (32 if d < 256 else 16))
        assert (np.abs(got[b] - want) <= tol).all(), b


def test_lengths_outside_their_range_are_clamped():
    g = np.random.default_rng(9)
    x = shared_contents(g, [640, 640, 640], 2, 64, 0, [0] * 3, {0: 8})
    Qb, Qv = bf16(g.normal(0, 1, (3, 4, 2, 64)))
    c = ugbs.Cache.make(3, 4, 2, 64, x.n_pages, 10, rows=2)
    O = run_shared(c, x, Qb, [2 ** 31 - 1, 640, -7], [5, -3, 2], [0] * 3)
    got = bf16_to_f64(host_bits(O))
    want, tol = reference(x, 0, Qv[0], 640, 2, 1 / 8)
    assert (np.abs(got[0] - want) <= tol).all() and (got[1] == 7.0).all() and (got[2] == 0).all()


def test_two_calls_give_the_same_bits():
    g = np.random.default_rng(10)
    lens = [3000 + int(n) for n in g.integers(1, 900, 40)]
    group = [0, 1] * 20
    x = shared_contents(g, lens, 8, 128, 0, group, {0: 46, 1: 30})
    Qb, _ = bf16(g.normal(0, 1, (40, 16, 2, 128)))
    c = ugbs.Cache.make(40, 16, 8, 128, x.n_pages, x.max_pages, rows=2)
    a, b = (run_shared(c, x, Qb, lens, [2] * 40, group, shared=True) for _ in range(2))
    assert torch.equal(a.view(torch.int16), b.view(torch.int16))


def test_offsets_pass_32_bits():
    """A cache of more than 4 GiB, its last pages used."""
    d, Hkv, n_pages = 256, 8, 20000                # 5.2e9 bytes
    g = np.random.default_rng(14)
    lens = [450, 370, 340] * 14
    B = len(lens)
    small = shared_contents(g, lens, Hkv, d, 0, [0] * B, {0: 5})
    shift = n_pages - small.n_pages
    cache = torch.zeros((n_pages, Hkv, 2, PAGE * d), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((n_pages, Hkv, 2), dtype=torch.float32, device="cuda")
    cache[shift:] = dev(small.raw)
    scales[shift:] = dev(small.scales)
    table = np.where(small.table >= 0, small.table + shift, -1).astype(I32)
    for n, rows, group in ((3, 1, [0] * 3), (B, 9, [0] * B)):
        Qb, Qv = bf16(g.normal(0, 1, (n, 8, rows, d)))
        c = ugbs.Cache.make(n, 8, Hkv, d, n_pages, small.max_pages, rows=rows)
        O = run_shared(c, None, Qb, lens[:n], [rows] * n, group, arrays=(cache, scales, dev(table[:n])), shared=n == 3 or None)
        for b in range(n):
            want, tol = reference(small, b, Qv[b], lens[b], rows, 1 / 16, rows > 1)
            assert (np.abs(bf16_to_f64(host_bits(O[b])) - want) <= tol).all()


def test_two_graphs_share_a_workspace_and_a_layout_is_made_in_each():
    g = np.random.default_rng(45)
    lens = [2000, 1990, 1500, 1400]
    x = shared_contents(g, lens, 2, 128, 0, [0, 0, 1, 1], {0: 30, 1: 20}, max_pages=40)
    cache, scales, table = x.device()
    group, kv = dev(np.array([0, 0, 1, 1], I32)), dev(np.array(lens, I32))
    calls = []
    for rows in (1, 3):
        c = ugbs.Cache.make(4, 8, 2, 128, x.n_pages, 40, rows=rows)
        Qb, Qv = bf16(g.normal(0, 1, (4, 8, rows, 128)))
        calls.append((c, dev_bf16(Qb), dev(np.array([rows] * 4, I32)), torch.zeros((4, 8, rows, 128), dtype=torch.bfloat16, device="cuda")))
    u8 = dict(dtype=torch.uint8, device="cuda")
    ws = torch.empty(max(ugbs.ugbs_cache_shared_workspace_bytes(y[0]) for y in calls), **u8)
    share = torch.empty(max(ugbs.ugbs_cache_share_bytes(y[0]) for y in calls), **u8)

    def one(c, Q, q, O):
        ugbs.ugbs_cache_share(c, group, table, kv, q, share)
        ugbs.ugbs_cache_attend_shared(c, Q, cache, scales, table, kv, q, share, O, ws)
    graphs = []
    for call in calls:
        one(*call)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            one(*call)
        graphs.append(graph)
    for rep in range(4):
        kv.add_(7)                                 # lengths grow between the replays (within the pages they hold)
        for _, _, _, O in calls:
            O.fill_(3.0)
        ws.fill_(rep)
        for graph in graphs if rep % 2 else graphs[::-1]:
            graph.replay()
        torch.cuda.synchronize()
        got = [O.clone() for *_, O in calls]
        for call, w in zip(calls, got):
            one(*call)
            torch.cuda.synchronize()
            assert torch.equal(call[3].view(torch.int16), w.view(torch.int16)), rep


def test_on_streams_of_their_own():
    g = np.random.default_rng(11)
    sides = []
    for k in range(2):
        lens = [900 + 100 * k + b for b in range(4)]
        x = shared_contents(g, lens, 2, 128, k, [0] * 4, {0: 12})
        Qb, _ = bf16(g.normal(0, 1, (4, 8, 1, 128)))
        c = ugbs.Cache.make(4, 8, 2, 128, x.n_pages, x.max_pages, dtype=k)
        u8 = dict(dtype=torch.uint8, device="cuda")
        sides.append((c, x.device(), dev_bf16(Qb), dev(np.array(lens, I32)), dev(np.ones(4, I32)), dev(np.zeros(4, I32)),
                      torch.empty(ugbs.ugbs_cache_share_bytes(c), **u8), torch.empty(ugbs.ugbs_cache_shared_workspace_bytes(c), **u8),
                      run_shared(c, x, Qb, lens, [1] * 4, [0] * 4, shared=True), torch.zeros((4, 8, 1, 128), dtype=torch.bfloat16, device="cuda"),
                      torch.cuda.Stream()))
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
