"""From projections to answers: prompts, requests that fork from them, steps of single tokens and of drafts over common
pages, on the GPU, against the same steps done call by call (ugbs_heads_split, ugbs_cache_store, and the 64-bit oracle)."""
import math

import numpy as np
import pytest
import torch

import paper_2607_07724_amd as ugbs
from gpu_helpers import bf16_to_f64, dev, host, host_bits
from test_gpu_cache import I32, Mirror, reference
from test_gpu_heads import freqs_of, packed

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need an MI355X (gfx950) visible to torch")
    ugbs.lib()


def _mirror(c, cbufs, step):
    """What the step and the cache hold, for the oracle."""
    m = Mirror(c)
    m.table, m.kv, m.q = host(step.table), host(step.kv_lens), host(step.q_lens)
    m.raw, m.scales = host(cbufs.cache), host(cbufs.scales)
    return m


def _check(c, cbufs, step, Q, O):
    m = _mirror(c, cbufs, step)
    got, Qv = bf16_to_f64(host_bits(O)), bf16_to_f64(host_bits(Q))
    tiles = c.batch * c.rows * c.n_heads // c.n_kv_heads > (32 if c.head_dim < 256 else 16)
    for b in range(c.batch):
        n = int(m.q[b])
        want, tol = reference(m, b, Qv[b], int(m.kv[b]), n, 1 / math.sqrt(c.head_dim), tiles)
        assert (np.abs(got[b, :, :n] - want[:, :n]) <= tol[:, :n]).all(), b


@pytest.mark.parametrize("dtype,d,H,Hkv,norm", [(ugbs.E4M3, 128, 4, 2, False), (ugbs.INT8, 64, 2, 1, True), (ugbs.E4M3, 256, 4, 2, True)])
def test_a_prompt_then_forks_then_steps(dtype, d, H, Hkv, norm):
    g = np.random.default_rng(d)
    B, N = 6, 256                                  # requests 0 and 3 bring prompts; 1, 2 fork from 0, 4, 5 from 3
    c = ugbs.Cache.make(B, H, Hkv, d, 80, 20, rows=N, dtype=dtype)
    step, cbufs = ugbs.CacheStep(c, shared=True), ugbs.CacheBuffers(c)
    cbufs.cache.zero_()
    cbufs.scales.zero_()
    f = torch.tensor(freqs_of(d), device="cuda")
    w = [torch.from_numpy(g.normal(1, 0.2, d).astype(np.float32)).cuda() if norm else None for _ in range(2)]
    group = dev(np.array([0, 0, 0, 1, 1, 1], I32))

    def one(rows, new, **kw):
        cr = ugbs.Cache.make(B, H, Hkv, d, 80, 20, rows=rows, dtype=dtype)
        h = ugbs.Heads.make(B, H, Hkv, d, rows)
        _, xq, xk, xv = packed(g, B, rows, H, Hkv, d)
        step.plan(cr, dev(np.array(new, I32)), **kw)
        Q, O = (torch.zeros((B, H, rows, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        before = cbufs.cache.clone(), cbufs.scales.clone()
        ugbs.rows_layer(h, cr, xq, xk, xv, f, Q, O, cbufs, step, q_norm=w[0], k_norm=w[1])
        _check(cr, cbufs, step, Q, O)
        # the cache by the separate calls
        K, V = (torch.zeros((B, Hkv, rows, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        ugbs.ugbs_heads_split(h, xq, xk, xv, f, torch.empty_like(Q), K, V, q_norm=w[0], k_norm=w[1], first=step.ctx_lens, lens=step.q_lens)
        ugbs.ugbs_cache_store(cr, K, V, step.slots, *before)
        assert torch.equal(before[0], cbufs.cache) and torch.equal(before[1], cbufs.scales)

    one(N, [200, 0, 0, 256, 0, 0])                 # whole prompts (more rows than are shared)
    step.fork(0, [1, 2], 192)
    step.fork(3, torch.tensor([4, 5], device="cuda"), 256)
    assert host(step.kv_lens).tolist() == [200, 192, 192, 256, 256, 256]
    one(1, [1, 1, 1, 1, 1, 1], group=group)
    one(5, [5, 0, 2, 1, 5, 3], group=group)        # drafts
    for _ in range(3):
        one(1, [1] * 6, group=group)
    one(1, [1] * 6)                                # the same without groups
    # two of the forks end: the pages they share stay, their own come back
    free = int(step.free_left.item())
    step.leave([1, 4], 256)
    step.plan(ugbs.Cache.make(B, H, Hkv, d, 80, 20, dtype=dtype), dev(np.array([1, -1, 1, 1, -1, 1], I32)), group=group)
    held = (192 + 1 + 3 + 1 + 63) // 64 - 4, (256 + 1 + 5 + 3 + 1 + 63) // 64 - 4
    assert int(step.free_left.item()) == free + sum(max(x, 0) for x in held)
    one(1, [1, 0, 1, 1, 0, 1], group=group)


def test_captured_steps_of_groups_replay_as_lengths_grow():
    """plan, layout, projection to cache and attention in one graph; each replay against the same step done eagerly."""
    g = np.random.default_rng(41)
    B, H, Hkv, d = 5, 4, 2, 128
    c = ugbs.Cache.make(B, H, Hkv, d, 64, 20)
    h = ugbs.Heads.make(B, H, Hkv, d)
    x, xq, xk, xv = packed(g, B, 1, H, Hkv, d)
    f = torch.tensor(freqs_of(d), device="cuda")
    new, group = dev(np.ones(B, I32)), dev(np.array([7, 7, -1, 7, 7], I32))
    sides = []
    for _ in range(2):
        cbufs, step = ugbs.CacheBuffers(c), ugbs.CacheStep(c, shared=True)
        cbufs.cache.copy_(torch.from_numpy(np.random.default_rng(1).integers(0, 120, tuple(cbufs.cache.shape), dtype=np.uint8)))
        cbufs.scales.fill_(2.0 ** -6)
        step.table[0, :4] = torch.arange(60, 64, device="cuda", dtype=torch.int32)
        step._after[B] = 60                        # the prompt's pages are not free
        step.kv_lens[0] = 256
        step.fork(0, [1, 3, 4], 256)
        sides.append((cbufs, step, *(torch.zeros((B, H, 1, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))))

    def one(side):
        cbufs, step, Q, O = side
        step.plan(c, new, group=group)
        ugbs.rows_layer(h, c, xq, xk, xv, f, Q, O, cbufs, step)

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
    for rep in range(70):                          # across a page border
        x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(rep)).to(torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        sides[0][1].slots.clone()
        one(sides[1])
        torch.cuda.synchronize()
        for a, b in zip(sides[0][2:], sides[1][2:]):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16)), rep
        assert torch.equal(sides[0][0].cache, sides[1][0].cache) and torch.equal(sides[0][1].kv_lens, sides[1][1].kv_lens)
        if rep % 23 == 0:
            _check(c, sides[0][0], sides[0][1], *sides[0][2:])
    assert host(sides[0][1].kv_lens).tolist() == [327, 327, 71, 327, 327]


def test_groups_need_a_step_made_for_them_and_forks_whole_pages():
    c = ugbs.Cache.make(2, 4, 1, 64, 8, 4)
    step = ugbs.CacheStep(c)
    with pytest.raises(ValueError, match="shared=True"):
        step.plan(c, dev(np.ones(2, I32)), group=dev(np.zeros(2, I32)))
    for tokens in (1, 65, -64, 64 * 5):
        with pytest.raises(ValueError, match="whole pages"):
            step.fork(0, [1], tokens)


def test_layers_of_another_shape_than_the_steps_layout_are_refused():
    c, other = ugbs.Cache.make(2, 4, 1, 64, 8, 4, rows=2), ugbs.Cache.make(2, 4, 1, 64, 8, 4, rows=1)
    step, cb = ugbs.CacheStep(c, shared=True), ugbs.CacheBuffers(c)
    step.plan(c, dev(np.ones(2, I32)), group=dev(np.zeros(2, I32)))
    Q = torch.zeros((2, 4, 1, 64), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="another cache"):
        step.attend(other, Q, torch.empty_like(Q), cb)
    step.plan(other, dev(np.ones(2, I32)))                    # without groups there is no layout
    step.attend(other, Q, torch.empty_like(Q), cb)
