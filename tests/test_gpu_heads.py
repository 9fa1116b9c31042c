"""From a projection's rows to heads on the GPU, against the formula in 64 bits.

Tolerance of a result y of a pair (u, v), in units of 2^-24 of |u| + |v|: the norm 13 (sums of squares 20, halved by
the root; root 2, weight 1), cos and sin 8 (angle 2^-23 absolute, series 2 roundings and 2^-28), products and sum 4,
gain 2: 27, taken as 32; and half a step of bf16, 2^-8 of y.
"""
import math

import numpy as np
import pytest
import torch

import paper_2607_07724_amd as ugbs

pytestmark = pytest.mark.gpu

BF = torch.bfloat16
I32 = torch.int32


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need an MI355X (gfx950) visible to torch")
    ugbs.lib()


def freqs_of(rot, theta=1e4):
    return theta ** (-2.0 * np.arange(rot // 2) / max(rot, 1))


def packed(g, B, rows, H, Hkv, d, gate=0, pad=0):
    """A packed projection and the views of its queries (each followed by `gate` numbers), keys and values."""
    width = H * (d + gate) + 2 * Hkv * d + pad
    x = torch.from_numpy(g.normal(0, 2, (B, rows, width)).astype(np.float32)).cuda().to(BF)
    a = H * (d + gate)
    return (x, x[..., :a].view(B, rows, H, d + gate)[..., :d], x[..., a:a + Hkv * d].view(B, rows, Hkv, d),
            x[..., a + Hkv * d:a + 2 * Hkv * d].view(B, rows, Hkv, d))


def want64(x, weight, pos, freqs, axis, rot, pairs, eps, gain):
    """[B,rows,heads,d] -> [B,heads,rows,d] in 64 bits, and each number's |u| + |v|; pos [axes,B,rows]."""
    x = x.double().cpu().numpy()
    B, rows, heads, d = x.shape
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight.double().cpu().numpy()
    size = np.abs(x)
    y = x.copy()
    if rot:
        j = np.arange(rot // 2)
        a, b = (j, j + rot // 2) if pairs == ugbs.HALVES else (2 * j, 2 * j + 1)
        t = np.moveaxis(pos[axis], 0, -1).astype(np.float64) * freqs          # [B,rows,rot/2]
        c, s = (gain * f(t)[:, :, None] for f in (np.cos, np.sin))
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
        size = size.copy()
        size[..., a] = size[..., b] = abs(gain) * (np.abs(x[..., a]) + np.abs(x[..., b]))
    return y.transpose(0, 2, 1, 3), size.transpose(0, 2, 1, 3)


def check(got, want, size, far=0.0):
    err = np.abs(got.double().cpu().numpy() - want)
    tol = 2.0 ** -8 * np.abs(want) + (32 * 2.0 ** -24 + far) * size + 2.0 ** -133
    assert (err <= tol * (1 + 2.0 ** -7)).all(), float((err / tol).max())


def run(h, xq, xk, xv, fill=7.0, **kw):
    B, rows, d = h.batch, h.rows, h.head_dim
    out = [torch.full((B, n, rows, d), fill, dtype=BF, device="cuda") for n in (h.n_heads, h.n_kv_heads, h.n_kv_heads)]
    ugbs.ugbs_heads_split(h, xq, xk, xv, kw.pop("freqs"), *out, **kw)
    return out


CASES = [
    # B, rows, H, Hkv, d, rot, pairs, norm, gate
    (1, 1, 4, 1, 64, 64, ugbs.HALVES, False, 0),
    (1, 1, 1, 1, 128, 128, ugbs.NEIGHBOURS, True, 0),
    (3, 7, 6, 3, 128, 128, ugbs.HALVES, True, 0),
    (2, 65, 28, 4, 128, 128, ugbs.HALVES, False, 0),
    (48, 1, 32, 8, 128, 128, ugbs.NEIGHBOURS, False, 0),
    (5, 33, 16, 2, 256, 64, ugbs.HALVES, True, 256),
    (2, 9, 3, 3, 256, 256, ugbs.HALVES, True, 8),
    (2, 17, 3, 3, 256, 240, ugbs.NEIGHBOURS, False, 16),
    (4, 31, 8, 2, 64, 16, ugbs.HALVES, True, 0),
    (4, 5, 8, 2, 64, 48, ugbs.NEIGHBOURS, True, 64),
    (2, 300, 5, 5, 128, 0, ugbs.HALVES, True, 0),
    (2, 3, 5, 5, 128, 0, ugbs.HALVES, False, 0),
    (1, 5000, 7, 1, 128, 96, ugbs.HALVES, False, 0),
]


@pytest.mark.parametrize("B,rows,H,Hkv,d,rot,pairs,norm,gate", CASES)
def test_split_equals_the_formula(B, rows, H, Hkv, d, rot, pairs, norm, gate):
    g = np.random.default_rng(d + rows + H)
    _, xq, xk, xv = packed(g, B, rows, H, Hkv, d, gate, pad=24)
    h = ugbs.Heads.make(B, H, Hkv, d, rows, rot=rot, pairs=pairs, eps=1e-5, gain=1.25 if rot == 48 else 0.0)
    gain = 1.25 if rot == 48 else 1.0
    w = [torch.from_numpy(g.normal(1, 0.3, d).astype(np.float32)).cuda() if norm else None for _ in range(2)]
    freqs, first, lens = freqs_of(rot), g.integers(0, 5000, B), g.integers(0, rows + 1, B)
    lens[0] = rows
    dev = dict(dtype=I32, device="cuda")
    Q, K, V = run(h, xq, xk, xv, freqs=torch.tensor(freqs, device="cuda"), q_norm=w[0], k_norm=w[1],
                  first=torch.tensor(first, **dev), lens=torch.tensor(lens, **dev))
    pos = (first[:, None] + np.arange(rows))[None]
    live = np.arange(rows) < lens[:, None]
    for got, x, weight, r in ((Q, xq, w[0], rot), (K, xk, w[1], rot), (V, xv, None, 0)):
        want, size = want64(x, weight, pos, freqs, np.zeros(rot // 2, int), r, pairs, 1e-5, gain)
        m = np.broadcast_to(live[:, None, :, None], want.shape)
        check(got, np.where(m, want, 7.0), size)              # rows behind the last are left as they are
    assert torch.equal(V[0], xv[0].transpose(0, 1))


def test_positions_given_and_axes():
    g = np.random.default_rng(2)
    B, rows, H, Hkv, d, rot = 2, 50, 4, 2, 128, 96
    _, xq, xk, xv = packed(g, B, rows, H, Hkv, d)
    freqs = freqs_of(rot, 1e6)
    axis = g.integers(0, 3, rot // 2)
    pos = g.integers(-1000, 100000, (3, B, rows))
    dev = dict(dtype=I32, device="cuda")
    f = torch.tensor(freqs, device="cuda")
    h = ugbs.Heads.make(B, H, Hkv, d, rows, rot=rot, axes=3)
    wild = axis.copy()                                        # axes outside 0..axes-1 are the nearest
    wild[axis == 0], wild[axis == 2] = -5, 99
    for ax in (axis, wild):
        Q, K, _ = run(h, xq, xk, xv, freqs=f, positions=torch.tensor(pos, **dev), axis=torch.tensor(ax, **dev))
        for got, x in ((Q, xq), (K, xk)):
            check(got, *want64(x, None, pos, freqs, axis, rot, ugbs.HALVES, 0, 1.0))
    # without an axis for each pair all go by the first one; without positions row i is at i
    Q, K, _ = run(h, xq, xk, xv, freqs=f, positions=torch.tensor(pos, **dev))
    check(Q, *want64(xq, None, pos, freqs, np.zeros(rot // 2, int), rot, ugbs.HALVES, 0, 1.0))
    Q, K, _ = run(h, xq, xk, xv, freqs=f)
    at = np.broadcast_to(np.arange(rows), (1, B, rows))
    check(K, *want64(xk, None, at, freqs, np.zeros(rot // 2, int), rot, ugbs.HALVES, 0, 1.0))


def test_far_positions_keep_their_angles():
    """|t| up to 2^31, where 2^-51 |t| is 2^-20; the oracle's own angles (64-bit, cos of the reduced number) are as far off."""
    g = np.random.default_rng(3)
    B, rows, d = 1, 64, 64
    _, xq, xk, xv = packed(g, B, rows, 2, 1, d)
    pos = np.concatenate([2 ** 31 - 1 - np.arange(16), -2 ** 31 + np.arange(16), 2 ** 24 + np.arange(16), 1000003 + np.arange(16)])[None, None]
    freqs = freqs_of(d)
    h = ugbs.Heads.make(B, 2, 1, d, rows)
    Q, _, _ = run(h, xq, xk, xv, freqs=torch.tensor(freqs, device="cuda"), positions=torch.tensor(pos, dtype=I32, device="cuda"))
    check(Q, *want64(xq, None, pos, freqs, np.zeros(32, int), d, ugbs.HALVES, 0, 1.0), far=2.0 ** -19)
    # first[b] + i may pass 2^31
    Q, _, _ = run(h, xq, xk, xv, freqs=torch.tensor(freqs, device="cuda"), first=torch.tensor([2 ** 31 - 10], dtype=I32, device="cuda"))
    at = (2 ** 31 - 10 + np.arange(rows, dtype=np.int64))[None, None]
    check(Q, *want64(xq, None, at, freqs, np.zeros(32, int), d, ugbs.HALVES, 0, 1.0), far=2.0 ** -19)


def test_every_quadrant_and_the_axes_of_the_circle():
    """One channel pair at angles of whole eighths of a turn: signs and the exchange of sine and cosine."""
    rows, d = 64, 64
    x = torch.zeros((1, rows, 1, d), dtype=BF, device="cuda")
    x[..., 0] = 1.0
    f = torch.zeros(32, dtype=torch.float64, device="cuda")
    f[0] = math.pi / 8
    h = ugbs.Heads.make(1, 1, 1, d, rows)
    Q, _, _ = run(h, x, x, x, freqs=f, positions=torch.arange(-32, 32, dtype=I32, device="cuda").view(1, 1, rows))
    t = np.arange(-32, 32) * (math.pi / 8)
    got = Q[0, 0].double().cpu().numpy()
    assert (np.abs(got[:, 0] - np.cos(t)) <= 2.0 ** -8 * np.abs(np.cos(t)) + 2.0 ** -19).all()
    assert (np.abs(got[:, 32] - np.sin(t)) <= 2.0 ** -8 * np.abs(np.sin(t)) + 2.0 ** -19).all()


def test_rows_of_zeros_infinities_and_nan_stay_in_their_rows():
    g = np.random.default_rng(4)
    B, rows, H, Hkv, d = 1, 40, 4, 2, 128
    x, xq, xk, xv = packed(g, B, rows, H, Hkv, d)
    f = torch.tensor(freqs_of(d), device="cuda")
    w = torch.ones(d, device="cuda")
    h = ugbs.Heads.make(B, H, Hkv, d, rows)
    base = run(h, xq, xk, xv, freqs=f, q_norm=w, k_norm=w)
    x[0, 3, :] = 0                                            # a token of zeros: 0 / sqrt(eps) = 0
    x[0, 5, 7] = float("nan")
    x[0, 6, 9] = float("inf")
    got = run(h, xq, xk, xv, freqs=f, q_norm=w, k_norm=w)
    assert (got[0][0, :, 3] == 0).all() and (got[1][0, :, 3] == 0).all()
    assert torch.isnan(got[0][0, 0, 5]).all() and torch.isnan(got[0][0, 0, 6, 9])
    for a, b in zip(base, got):
        keep = torch.tensor([i not in (3, 5, 6) for i in range(rows)], device="cuda")
        assert torch.equal(a[:, :, keep], b[:, :, keep])
    assert torch.equal(base[0][0, 1:, 5:7], got[0][0, 1:, 5:7])      # other heads of the same tokens


def test_rows_read_twice_and_separate_projections():
    """Stride 0 along the batch and along the heads; queries, keys and values as tensors of their own."""
    g = np.random.default_rng(5)
    B, rows, H, d = 3, 10, 4, 64
    one = torch.from_numpy(g.normal(0, 1, (rows, d)).astype(np.float32)).cuda().to(BF)
    xq = one[None, :, None].expand(B, rows, H, d)
    xk, xv = (torch.from_numpy(g.normal(0, 1, (B, rows, 1, d)).astype(np.float32)).cuda().to(BF) for _ in range(2))
    f = torch.tensor(freqs_of(d), device="cuda")
    h = ugbs.Heads.make(B, H, 1, d, rows)
    Q, K, V = run(h, xq, xk, xv, freqs=f)
    whole = run(h, xq.contiguous(), xk, xv, freqs=f)
    assert all(torch.equal(a, b) for a, b in zip((Q, K, V), whole))
    assert torch.equal(Q, Q[:1, :1].expand_as(Q))


def test_split_into_what_the_prefill_takes_on_a_stream_and_in_a_graph():
    """A layer's queries, keys and values straight into the prefill; captured, replayed on new rows, on its own stream."""
    g = np.random.default_rng(6)
    B, rows, H, Hkv, d = 1, 1024, 4, 1, 64
    x, xq, xk, xv = packed(g, B, rows, H, Hkv, d)
    f = torch.tensor(freqs_of(d), device="cuda")
    h = ugbs.Heads.make(B, H, Hkv, d, rows)
    p = ugbs.Problem.make(B, H, Hkv, rows, d, 4, 0.25)
    bufs = ugbs.Buffers(p)
    Q, K, V = run(h, xq, xk, xv, freqs=f)
    O = torch.zeros_like(Q)
    ugbs.prefill(p, Q, K, V, O, bufs)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    Q2, K2, V2, O2 = (torch.zeros_like(t) for t in (Q, K, V, O))
    with torch.cuda.stream(side):
        ugbs.ugbs_heads_split(h, xq, xk, xv, f, Q2, K2, V2)
        ugbs.prefill(p, Q2, K2, V2, O2, bufs)
    side.synchronize()
    assert torch.equal(O, O2) and torch.equal(K, K2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ugbs.ugbs_heads_split(h, xq, xk, xv, f, Q2, K2, V2)
        ugbs.prefill(p, Q2, K2, V2, O2, bufs)
    for k in range(3):
        x.copy_(torch.from_numpy(g.normal(0, 2, tuple(x.shape)).astype(np.float32)).cuda())
        graph.replay()
        torch.cuda.synchronize()
        want = run(h, xq, xk, xv, freqs=f)
        ugbs.prefill(p, *want, O, bufs)
        assert torch.equal(O, O2) and all(torch.equal(a, b) for a, b in zip(want, (Q2, K2, V2)))


def test_more_elements_than_32_bits_count():
    """Rows behind 2^31 elements of the projection and of the queries."""
    B, rows, H, Hkv, d = 2, 33000, 130, 1, 256
    if torch.cuda.mem_get_info()[0] < 24e9:
        pytest.skip("needs 24 GB")
    xq = torch.zeros((B, rows, H, d), dtype=BF, device="cuda")
    xk, xv = (torch.zeros((B, rows, Hkv, d), dtype=BF, device="cuda") for _ in range(2))
    g = torch.Generator(device="cuda").manual_seed(1)
    for i in (0, 17, rows - 1):
        xq[:, i] = torch.randn((B, H, d), generator=g, device="cuda").to(BF)
    h = ugbs.Heads.make(B, H, Hkv, d, rows, rot=0)
    Q, K, V = run(h, xq, xk, xv, freqs=None)
    assert Q.numel() > 2 ** 31
    for i in (0, 17, rows - 1):
        assert torch.equal(Q[:, :, i], xq[:, i])
    assert int((Q[1, -1, -2] != 0).sum()) == 0


# ---------------------------------------------------------------- straight into the cache

def pages(n):
    return -(-n // 64)


STORES = [
    # B, rows, H, Hkv, d, rot, pairs, norm, dtype
    (1, 1, 4, 1, 64, 64, ugbs.HALVES, False, ugbs.E4M3),
    (48, 1, 32, 8, 128, 128, ugbs.NEIGHBOURS, False, ugbs.E4M3),
    (5, 3, 6, 3, 128, 96, ugbs.HALVES, True, ugbs.INT8),
    (3, 200, 8, 2, 64, 32, ugbs.HALVES, True, ugbs.INT8),
    (2, 131, 28, 4, 128, 128, ugbs.HALVES, False, ugbs.E4M3),
    (2, 777, 4, 2, 256, 64, ugbs.HALVES, True, ugbs.INT8),
    (1, 257, 2, 1, 256, 256, ugbs.HALVES, True, ugbs.E4M3),
    (2, 70, 2, 1, 256, 256, ugbs.NEIGHBOURS, False, ugbs.INT8),
    (2, 70, 2, 1, 128, 0, ugbs.HALVES, True, ugbs.E4M3),
    (2, 70, 2, 1, 128, 0, ugbs.HALVES, False, ugbs.E4M3),
]


@pytest.mark.parametrize("B,rows,H,Hkv,d,rot,pairs,norm,dtype", STORES)
def test_store_equals_split_then_cache_store_byte_for_byte(B, rows, H, Hkv, d, rot, pairs, norm, dtype):
    g = np.random.default_rng(rows + d + B)
    mp = pages(rows + 300)
    c = ugbs.Cache.make(B, H, Hkv, d, B * mp + 3, mp, rows=rows, dtype=dtype)
    h = ugbs.Heads.make(B, H, Hkv, d, rows, rot=rot, pairs=pairs)
    step, a, b = ugbs.CacheStep(c), ugbs.CacheBuffers(c), ugbs.CacheBuffers(c)
    for t in (a, b):
        t.cache.fill_(0x55)
        t.scales.fill_(3.0)
    w = [torch.from_numpy(g.normal(1, 0.3, d).astype(np.float32)).cuda() if norm else None for _ in range(2)]
    f = torch.tensor(freqs_of(rot), device="cuda") if rot else None
    for k in range(3):                        # the pieces begin inside pages, ever louder: scales grow
        _, xq, xk, xv = packed(g, B, rows, H, Hkv, d, gate=8)
        new = g.integers(0, rows + 1, B) if k else np.full(B, min(rows, 37))
        new = np.minimum(new, 64 * mp - step.kv_lens.cpu().numpy())
        xk, xv = xk * 2.0 ** (3 * k), xv * 2.0 ** (2 * k)
        step.plan(c, torch.tensor(new, dtype=I32, device="cuda"))
        how = dict(q_norm=w[0], k_norm=w[1], first=step.ctx_lens, lens=step.q_lens)
        Q, K, V = run(h, xq, xk, xv, freqs=f, **how)
        ugbs.ugbs_cache_store(c, K, V, step.slots, a.cache, a.scales)
        Q2 = torch.full_like(Q, 7.0)
        ugbs.ugbs_heads_store(h, c, xq, xk, xv, f, Q2, step.slots, b.cache, b.scales, **how)
        assert torch.equal(Q.view(torch.int16), Q2.view(torch.int16))
        assert torch.equal(a.cache, b.cache) and torch.equal(a.scales, b.scales), k


def test_store_with_pages_that_are_none_and_numbers_that_are_not_finite():
    g = np.random.default_rng(9)
    B, rows, H, Hkv, d = 2, 150, 4, 2, 128
    c = ugbs.Cache.make(B, H, Hkv, d, 12, 4, rows=rows)
    h = ugbs.Heads.make(B, H, Hkv, d, rows)
    x, xq, xk, xv = packed(g, B, rows, H, Hkv, d)
    x[0, 70, H * d + 3] = float("inf")
    x[1, 20, H * d + Hkv * d + 5] = float("nan")
    pos = np.arange(rows) + np.array([[10], [0]])
    table = np.array([[-1, 3, 5], [4, -1, 8]])
    page = np.take_along_axis(table, pos // 64, 1)
    slots = torch.tensor(np.where(page >= 0, page * 64 + pos % 64, -1), dtype=I32, device="cuda")
    slots[1, 100:] = -1
    f = torch.tensor(freqs_of(d), device="cuda")
    a, b = ugbs.CacheBuffers(c), ugbs.CacheBuffers(c)
    for t in (a, b):
        t.cache.fill_(0x31)
        t.scales.fill_(2.0)
    Q, K, V = run(h, xq, xk, xv, freqs=f)
    ugbs.ugbs_cache_store(c, K, V, slots, a.cache, a.scales)
    ugbs.ugbs_heads_store(h, c, xq, xk, xv, f, torch.zeros_like(Q), slots, b.cache, b.scales)
    assert torch.equal(a.cache, b.cache) and torch.equal(a.scales, b.scales)
    assert not torch.equal(a.cache[3], torch.full_like(a.cache[3], 0x31)) and bool((a.cache[7] == 0x31).all())
