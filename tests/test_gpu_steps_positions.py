"""From projections to answers where test_gpu_steps_shared.py does not go: given positions on several axes, into the cache and
through a layer; steps whose common pages are tiles of many rows, eager and captured; steps on a stream of their own; forks that
leave their pages."""
import numpy as np
import pytest
import torch

import paper_2607_07724_amd as ugbs
from gpu_helpers import dev, host
from test_gpu_cache import I32
from test_gpu_heads import check as check_heads, freqs_of, packed, pages, want64
from test_gpu_shared import prefix_parts
from test_gpu_steps_shared import _check

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need an MI355X (gfx950) visible to torch")
    ugbs.lib()


def at_of(g, axes, B, rows):
    return g.integers(-500, 60000, (axes, B, rows))


@pytest.mark.parametrize("B,rows,H,Hkv,d,rot,pairs,axes,norm,dtype", [
    (3, 1, 4, 1, 64, 48, ugbs.HALVES, 3, True, ugbs.E4M3), (2, 150, 8, 2, 128, 96, ugbs.NEIGHBOURS, 2, False, ugbs.INT8),
    (3, 70, 4, 2, 256, 64, ugbs.HALVES, 4, True, ugbs.E4M3), (2, 333, 6, 3, 128, 128, ugbs.HALVES, 3, True, ugbs.E4M3),
    (5, 9, 2, 1, 256, 256, ugbs.NEIGHBOURS, 1, False, ugbs.INT8)])
@pytest.mark.parametrize("by_axis", [True, False])
def test_given_positions_into_the_cache(B, rows, H, Hkv, d, rot, pairs, axes, norm, dtype, by_axis):
    """Byte for byte ugbs_heads_split then ugbs_cache_store, whose Q and K are the formula's; pieces that begin inside pages."""
    g = np.random.default_rng(rows + d + axes)
    mp = pages(2 * rows + 100)
    c = ugbs.Cache.make(B, H, Hkv, d, B * mp + 3, mp, rows=rows, dtype=dtype)
    h = ugbs.Heads.make(B, H, Hkv, d, rows, rot=rot, pairs=pairs, axes=axes, eps=1e-5)
    step, a, b = ugbs.CacheStep(c), ugbs.CacheBuffers(c), ugbs.CacheBuffers(c)
    for t in (a, b):
        t.cache.fill_(0x55)
        t.scales.fill_(3.0)
    w = [torch.from_numpy(g.normal(1, 0.3, d).astype(np.float32)).cuda() if norm else None for _ in range(2)]
    freqs, axis = freqs_of(rot, 1e6), g.integers(0, axes, rot // 2)
    f = torch.tensor(freqs, device="cuda")
    for k in range(2):
        _, xq, xk, xv = packed(g, B, rows, H, Hkv, d, gate=8)
        new = g.integers(0, rows + 1, B)
        new[0] = rows
        step.plan(c, dev(new.astype(I32)))
        pos = at_of(g, axes, B, rows)
        how = dict(q_norm=w[0], k_norm=w[1], positions=dev(pos.astype(I32)), lens=step.q_lens,
                   axis=dev(axis.astype(I32)) if by_axis else None)
        Q, Q2 = (torch.full((B, H, rows, d), 7.0, dtype=BF, device="cuda") for _ in range(2))
        K, V = (torch.full((B, Hkv, rows, d), 7.0, dtype=BF, device="cuda") for _ in range(2))
        ugbs.ugbs_heads_split(h, xq, xk, xv, f, Q, K, V, **how)
        ugbs.ugbs_cache_store(c, K, V, step.slots, a.cache, a.scales)
        ugbs.ugbs_heads_store(h, c, xq, xk, xv, f, Q2, step.slots, b.cache, b.scales, **how)
        assert torch.equal(Q.view(torch.int16), Q2.view(torch.int16))
        assert torch.equal(a.cache, b.cache) and torch.equal(a.scales, b.scales), k
        live = np.arange(rows) < new[:, None]
        for got, x, weight in ((Q2, xq, w[0]), (K, xk, w[1])):
            want, size = want64(x, weight, pos, freqs, axis if by_axis else 0 * axis, rot, pairs, 1e-5, 1.0)
            check_heads(got, np.where(np.broadcast_to(live[:, None, :, None], want.shape), want, 7.0), size)


@pytest.mark.parametrize("grouped", [False, True])
def test_layers_from_rows_with_given_positions(grouped):
    """rows_layer with positions and axes: a prompt, a fork of it, single tokens, against the calls one by one."""
    g = np.random.default_rng(3)
    B, H, Hkv, d, N = 3, 8, 2, 128, 200
    f, axis = torch.tensor(freqs_of(d), device="cuda"), dev(g.integers(0, 3, d // 2).astype(I32))
    w = [torch.from_numpy(g.normal(1, 0.2, d).astype(np.float32)).cuda() for _ in range(2)]
    c = ugbs.Cache.make(B, H, Hkv, d, 40, 10, rows=N)
    step, cb = ugbs.CacheStep(c, shared=grouped), ugbs.CacheBuffers(c)
    cb.cache.zero_()
    cb.scales.zero_()
    group = dict(group=dev(np.zeros(B, I32))) if grouped else {}
    for k, (rows, new) in enumerate(((N, [N, 0, 0]), (1, [1, 1, 1]), (4, [4, 0, 2]), (1, [1, 1, 1]))):
        cr, h = ugbs.Cache.make(B, H, Hkv, d, 40, 10, rows=rows), ugbs.Heads.make(B, H, Hkv, d, rows, axes=3)
        _, xq, xk, xv = packed(g, B, rows, H, Hkv, d)
        pos = dev(at_of(g, 3, B, rows).astype(I32))
        step.plan(cr, dev(np.array(new, I32)), **(group if k else {}))
        if grouped and k:                          # (three pages among more than 16 rows are laid out alone)
            assert (prefix_parts(cr, step.share[:ugbs.ugbs_cache_share_bytes(cr)]) > 0) == (rows == 1)
        Q, O = (torch.zeros((B, H, rows, d), dtype=BF, device="cuda") for _ in range(2))
        before = cb.cache.clone(), cb.scales.clone()
        assert ugbs.rows_layer(h, cr, xq, xk, xv, f, Q, O, cb, step, q_norm=w[0], k_norm=w[1], positions=pos, axis=axis) is O
        _check(cr, cb, step, Q, O)
        Q2 = torch.zeros_like(Q)
        K, V = (torch.zeros((B, Hkv, rows, d), dtype=BF, device="cuda") for _ in range(2))
        ugbs.ugbs_heads_split(h, xq, xk, xv, f, Q2, K, V, q_norm=w[0], k_norm=w[1], positions=pos, axis=axis, lens=step.q_lens)
        ugbs.ugbs_cache_store(cr, K, V, step.slots, *before)
        assert torch.equal(Q, Q2) and torch.equal(before[0], cb.cache) and torch.equal(before[1], cb.scales)
        if k == 0:
            step.fork(0, [1, 2], 192)


def prompts_and_forks(c, cb, step, requests, prompt, seed=1):
    """Request 0 holds `prompt` tokens (any bytes) in the cache's last pages, which are not free; `requests` fork from it."""
    n = pages(prompt)
    cb.cache.copy_(torch.from_numpy(np.random.default_rng(seed).integers(0, 120, tuple(cb.cache.shape), dtype=np.uint8)))
    cb.scales.fill_(2.0 ** -6)
    step.table[0, :n] = torch.arange(c.n_pages - n, c.n_pages, device="cuda", dtype=torch.int32)
    step.free_left.fill_(c.n_pages - n)
    step.kv_lens[0] = prompt
    step.fork(0, requests, prompt // 64 * 64)


@pytest.mark.parametrize("dtype,d", [(ugbs.E4M3, 128), (ugbs.INT8, 64), (ugbs.E4M3, 256)])
def test_drafts_of_many_requests_behind_a_prompt(dtype, d):
    """Steps of 1 and 4 tokens: 22 and 88 rows of a kv head to the common pages, one request alone, one of another prompt's length."""
    g = np.random.default_rng(d)
    B, H, Hkv, prompt = 24, 16, 16, 64 * 24
    made = ugbs.Cache.make(B, H, Hkv, d, 200, 40, rows=4, dtype=dtype)
    step, cb = ugbs.CacheStep(made, shared=True), ugbs.CacheBuffers(made)
    prompts_and_forks(made, cb, step, range(1, 23), prompt + 7)
    group = np.zeros(B, I32)
    group[23], group[5] = 3, -1
    f = torch.tensor(freqs_of(d), device="cuda")
    for rows, new in ((1, np.ones(B, I32)), (4, g.integers(0, 5, B)), (4, np.full(B, 4)), (1, np.ones(B, I32))):
        c, h = ugbs.Cache.make(B, H, Hkv, d, 200, 40, rows=rows, dtype=dtype), ugbs.Heads.make(B, H, Hkv, d, rows)
        _, xq, xk, xv = packed(g, B, rows, H, Hkv, d)
        step.plan(c, dev(new.astype(I32)), group=dev(group))
        assert prefix_parts(c, step.share[:ugbs.ugbs_cache_share_bytes(c)]) > 0
        Q, O = (torch.zeros((B, H, rows, d), dtype=BF, device="cuda") for _ in range(2))
        ugbs.rows_layer(h, c, xq, xk, xv, f, Q, O, cb, step)
        _check(c, cb, step, Q, O)


def test_captured_steps_of_many_rows_share_as_lengths_grow():
    g = np.random.default_rng(42)
    B, H, Hkv, d = 24, 16, 16, 128
    c, h = ugbs.Cache.make(B, H, Hkv, d, 200, 40), ugbs.Heads.make(B, H, Hkv, d)
    x, xq, xk, xv = packed(g, B, 1, H, Hkv, d)
    f = torch.tensor(freqs_of(d), device="cuda")
    new, group = dev(np.ones(B, I32)), dev(np.array([7] * 20 + [-1] * 4, I32))
    sides = []
    for _ in range(2):
        cb, step = ugbs.CacheBuffers(c), ugbs.CacheStep(c, shared=True)
        prompts_and_forks(c, cb, step, range(1, 22), 64 * 24)
        sides.append((cb, step, *(torch.zeros((B, H, 1, d), dtype=BF, device="cuda") for _ in range(2))))

    def one(side):
        cb, step, Q, O = side
        step.plan(c, new, group=group)
        ugbs.rows_layer(h, c, xq, xk, xv, f, Q, O, cb, step)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                  # outside the capture first
        one(sides[0])
    torch.cuda.current_stream().wait_stream(side)
    one(sides[1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one(sides[0])
    torch.cuda.synchronize()
    a, b = sides[0][1], sides[1][1]
    for rep in range(66):                          # across a page border
        x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(rep)).to(BF))
        graph.replay()
        torch.cuda.synchronize()
        assert prefix_parts(c, a.share) > 0
        one(sides[1])
        torch.cuda.synchronize()
        for s, t in zip(sides[0][2:], sides[1][2:]):
            assert torch.equal(s.view(torch.int16), t.view(torch.int16)), rep
        for name in ("slots", "table", "kv_lens", "q_lens", "ctx_lens", "free_left"):
            assert torch.equal(getattr(a, name), getattr(b, name)), (rep, name)
        assert torch.equal(sides[0][0].cache, sides[1][0].cache) and torch.equal(sides[0][0].scales, sides[1][0].scales)
        if rep % 65 == 0:
            _check(c, sides[0][0], a, *sides[0][2:])
    assert host(a.kv_lens).tolist() == [64 * 24 + 67] * 22 + [67] * 2


@pytest.mark.parametrize("many", [False, True])
def test_steps_of_groups_on_a_stream_that_is_given(many):
    """plan(stream=, group=) and the layers on one stream, by its handle, while another one works: the same bits as on the current one."""
    g = np.random.default_rng(8)
    B, H, Hkv, d = (24, 16, 16, 64) if many else (4, 8, 2, 128)
    c, h = ugbs.Cache.make(B, H, Hkv, d, 200, 40), ugbs.Heads.make(B, H, Hkv, d)
    x, xq, xk, xv = packed(g, B, 1, H, Hkv, d)
    f = torch.tensor(freqs_of(d), device="cuda")
    new, group = dev(np.ones(B, I32)), dev(np.zeros(B, I32))
    stream, got = torch.cuda.Stream(), []
    for how in (dict(), dict(stream=stream.cuda_stream)):
        cb, step = ugbs.CacheBuffers(c), ugbs.CacheStep(c, shared=True)
        prompts_and_forks(c, cb, step, range(1, B), 64 * 24)
        Q, O = (torch.zeros((B, H, 1, d), dtype=BF, device="cuda") for _ in range(2))
        torch.cuda.synchronize()
        for _ in range(3):
            step.plan(c, new, group=group, **how)
            ugbs.rows_layer(h, c, xq, xk, xv, f, Q, O, cb, step, **({"stream": stream.cuda_stream} if how else {}))
            torch.randn(1 << 20, device="cuda").sum()
        torch.cuda.synchronize()
        assert prefix_parts(c, step.share) > 0
        _check(c, cb, step, Q, O)
        got.append((Q, O, cb.cache, cb.scales, step.kv_lens, step.slots, step.table))
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(*got))


def test_forks_that_end_give_back_their_own_pages():
    """Two forks, of 192 and 256 tokens, leave what they share and are released: their own pages come back, no others."""
    B, H, Hkv, d = 6, 4, 2, 64
    c = ugbs.Cache.make(B, H, Hkv, d, 80, 20, rows=256)
    one = ugbs.Cache.make(B, H, Hkv, d, 80, 20)
    step = ugbs.CacheStep(c, shared=True)
    step.plan(c, dev(np.array([200, 0, 0, 256, 0, 0], I32)))
    step.fork(0, [1, 2], 192)
    step.fork(3, torch.tensor([4, 5], device="cuda"), 256)
    step.plan(c, dev(np.array([1, 5, 1, 1, 70, 1], I32)))
    free, table = int(step.free_left.item()), host(step.table)
    own = {int(table[1, 3]), int(table[4, 4]), int(table[4, 5])}
    step.leave([1], 192)
    step.leave(torch.tensor([4, 4], device="cuda"), 256)
    step.plan(one, dev(np.array([0, -1, 0, 0, -1, 0], I32)))
    assert int(step.free_left.item()) == free + 3
    assert set(host(step.free_pages)[free:free + 3].tolist()) == own
    assert host(step.kv_lens).tolist() == [201, 0, 193, 257, 0, 257]


def test_forks_of_more_than_the_source_has_and_numbers_outside_the_batch():
    """After pages were given back and taken again by another request: entries behind the source's tokens are not taken along."""
    c = ugbs.Cache.make(4, 4, 1, 64, 12, 6, rows=320)
    step = ugbs.CacheStep(c)
    step.plan(c, dev(np.array([320, 0, 0, 0], I32)))
    step.plan(c, dev(np.array([-1, 0, 0, 0], I32)))
    step.plan(c, dev(np.array([100, 300, 0, 0], I32)))      # request 0's row still lists pages that are request 1's now
    step.fork(0, torch.tensor([2, -9, 4, 99], device="cuda"), 320)
    table = host(step.table)
    assert host(step.kv_lens).tolist() == [100, 300, 64, 0]
    assert table[2].tolist() == [table[0, 0], -1, -1, -1, -1, -1] and (table[3] == -1).all()
    step.plan(c, dev(np.array([0, 0, 3, 0], I32)))
    assert host(step.kv_lens).tolist() == [100, 300, 67, 0]
    table = host(step.table)
    assert table[2, 1] >= 0 and table[2, 1] not in set(table[0, :2].tolist()) | set(table[1, :5].tolist())
