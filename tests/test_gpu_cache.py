"""The cache's entry points on the GPU against the 64-bit oracle (cache_oracle.py)."""
import math

import numpy as np
import pytest
import torch

import cache_oracle as co
import paper_2607_07724_amd as ugbs

from gpu_helpers import bf16_to_f64, dev, dev_bf16, host, host_bits

pytestmark = pytest.mark.gpu

PAGE = 64
I32 = np.int32


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need an MI355X (gfx950) visible to torch")
    ugbs.lib()


def bf16(x):
    """float array -> (bf16 bits, their values in 64 bits)."""
    from paper_2607_07724_amd import synth
    b = synth.bf16_bits(np.asarray(x, np.float32))
    return b, bf16_to_f64(b)


def pages(n):
    return -(-n // PAGE)


class Contents:
    """A cache in which request b holds lens[b] tokens; what is no token's is noise (NaN bytes among it)."""

    def __init__(self, g, lens, Hkv, d, dtype, max_pages=None, n_pages=None, loud=1.0):
        B = len(lens)
        held = [pages(n) for n in lens]
        self.max_pages = max_pages or max(1, max(held))
        self.n_pages = n_pages or sum(held) + 4
        order = g.permutation(self.n_pages)
        self.table = np.full((B, self.max_pages), -1, I32)
        self.dtype, self.d, self.lens, self.Hkv = dtype, d, list(lens), Hkv
        shape = (self.n_pages, Hkv, PAGE, d)
        top = co.TOP[dtype]
        num = [co.nearest(np.clip(g.normal(0, top / 4, shape), -top, top), dtype) for _ in range(2)]
        self.raw = g.integers(0, 256, (self.n_pages, Hkv, 2, PAGE * d), dtype=np.uint8)
        self.scales = (2.0 ** g.integers(-9, -6, (self.n_pages, Hkv, 2)) * loud).astype(np.float32)
        enc = co.encode(*num, dtype)
        at = 0
        live = np.zeros((self.n_pages, PAGE), bool)
        for b, n in enumerate(lens):
            self.table[b, :held[b]] = order[at:at + held[b]]
            for j in range(held[b]):
                live[order[at + j], :min(PAGE, n - PAGE * j)] = True
            at += held[b]
        for w, where in enumerate((co.key_at(d), co.value_at(d))):
            keep = np.zeros((self.n_pages, PAGE * d), bool)
            keep[:, where] = live[:, :, None]
            self.raw[:, :, w] = np.where(keep[:, None], enc[:, :, w], self.raw[:, :, w])
        unused = ~live.any(1)
        self.scales[unused] = np.nan

    def device(self):
        return dev(self.raw), dev(self.scales), dev(self.table)

    def tokens(self, b, n):
        """Keys, values [Hkv, n, d] in 64 bits and whether each position lies in a page."""
        k, v = np.zeros((self.Hkv, n, self.d)), np.zeros((self.Hkv, n, self.d))
        there = np.zeros(n, bool)
        for j in range(pages(n)):
            p = int(self.table[b, j])
            a, z = PAGE * j, min(n, PAGE * (j + 1))
            if 0 <= p < self.n_pages:
                kk, vv = co.decode(self.raw[p:p + 1], self.scales[p:p + 1], self.dtype, self.d)
                k[:, a:z], v[:, a:z], there[a:z] = kk[0, :, :z - a], vv[0, :, :z - a], True
        return k, v, there


# ---------------------------------------------------------------- plan

def _plan_case(g, B, max_pages, rows, stock, wild=False):
    ctx = g.integers(0, PAGE * max_pages - rows + 1, B)
    new = g.integers(0, rows + 1, B)
    new[g.random(B) < 0.15] = -1
    new[g.random(B) < 0.2] = min(1, rows)
    ctx[g.random(B) < 0.2] = 0
    if wild:
        for x, values in ((ctx, (-5, PAGE * max_pages + 1, 2 ** 31 - 1, -2 ** 31, PAGE * max_pages)), (new, (rows + 1, -2, 2 ** 31 - 1, -2 ** 31))):
            pick = g.random(B) < 0.2
            x[pick] = g.choice(values, pick.sum())
    held = [-(-int(c) // PAGE) if 0 <= c <= PAGE * max_pages else 0 for c in ctx]
    n_pages = sum(held) + 50
    order = g.permutation(n_pages)
    table = np.full((B, max_pages), -1, I32)
    at = 0
    for b in range(B):
        table[b, :held[b]] = order[at:at + held[b]]
        at += held[b]
    stack = np.full(n_pages, -7, I32)
    count = int(stock * (n_pages - at))
    stack[:count] = order[at:at + count]
    return ctx.astype(I32), new.astype(I32), stack, count, table


def _run_plan(ctx, new, stack, count, table, rows):
    B, mp = table.shape
    c = ugbs.Cache.make(B, 1, 1, 64, len(stack), mp, rows=rows)
    tb, st = dev(table), dev(stack)
    kv, q, left = (torch.full((n,), -9, dtype=torch.int32, device="cuda") for n in (B, B, 1))
    slots = torch.full((B, rows), -9, dtype=torch.int32, device="cuda")
    ugbs.ugbs_cache_plan(c, dev(ctx), dev(new), st, dev(np.array([count], I32)), tb, kv, q, slots, left)
    return [host(x) for x in (st, tb, kv, q, slots)] + [int(left.item())]


@pytest.mark.parametrize("B,max_pages,rows,stock,wild", [
    (1, 1, 1, 1, False), (1, 3, 64, 1, False), (5, 4, 100, 0.5, False), (64, 6, 3, 1, False), (65, 9, 65, 0.6, False),
    (257, 5, 7, 0.3, True), (1000, 3, 130, 0.1, True), (4096, 2, 1, 0.5, True), (3, 80, 4096, 1, False), (300, 4, 64, 0, False)])
def test_plan_equals_the_oracle(B, max_pages, rows, stock, wild):
    g = np.random.default_rng(B + rows)
    for _ in range(3):
        ctx, new, stack, count, table = _plan_case(g, B, max_pages, rows, stock, wild)
        got = _run_plan(ctx, new, stack, count, table, rows)
        want = co.plan(ctx, new, stack, count, table, rows)
        for name, a, b in zip(("free_pages", "table", "kv_lens", "q_lens", "slots", "free_left"), got, want):
            assert np.array_equal(a, b), name


def test_plan_takes_counts_outside_the_stack_and_entries_that_are_no_page():
    for count in (-3, 2 ** 31 - 1):
        ctx, new = np.array([10, 100, 0], I32), np.array([5, -1, 64], I32)
        table = np.array([[99, -1], [4, 5], [-1, -1]], I32)        # request 0's page does not exist
        stack = np.arange(8, dtype=I32)
        got = _run_plan(ctx, new, stack, count, table, 64)
        want = co.plan(ctx, new, stack, count, table, 64)
        for a, b in zip(got, want):
            assert np.array_equal(a, b)


# ---------------------------------------------------------------- store and load

def _slots(table, starts, counts, rows):
    out = np.full((len(starts), rows), -1, I32)
    for b, (a, n) in enumerate(zip(starts, counts)):
        for i in range(n):
            out[b, i] = table[b, (a + i) // PAGE] * PAGE + (a + i) % PAGE
    return out


def _load(c, cache, scales, table, start, count, width, fill=float("nan")):
    K = torch.full((c.batch, c.n_kv_heads, width, c.head_dim), fill, dtype=torch.bfloat16, device="cuda")
    V = torch.full_like(K, fill)
    ugbs.ugbs_cache_load(c, cache, scales, table, dev(np.array(start, I32)), dev(np.array(count, I32)), K, V)
    return bf16_to_f64(host_bits(K)), bf16_to_f64(host_bits(V))


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype", [ugbs.E4M3, ugbs.INT8])
@pytest.mark.parametrize("rows,lens", [
    (1, [0, 1, 62, 63, 64, 65, 127, 130]),      # one token each, at every kind of place
    (5, [0, 59, 60, 63, 64, 3]),                # pieces that cross into the next page
    (64, [0, 1, 64, 63]),                       # whole pages, and pages split by the start
    (200, [0, 37, 128]),
])
def test_store_equals_the_oracle(d, dtype, rows, lens):
    g = np.random.default_rng(rows * d + dtype)
    B, Hkv = len(lens), 2
    counts = [int(x) for x in g.integers(0, rows + 1, B)]
    counts[0] = rows
    full = [n + m for n, m in zip(lens, counts)]
    x = Contents(g, full, Hkv, d, dtype)
    # sizes from far below to far above what the page holds, so that scales stay, and grow
    size = 2.0 ** g.integers(-6, 9, (B, 1, rows, 1))
    Kb, K = bf16(g.normal(0, 1, (B, Hkv, rows, d)) * size)
    Vb, V = bf16(g.normal(0, 1, (B, Hkv, rows, d)) * size[:, :, ::-1])
    slots = _slots(x.table, lens, counts, rows)
    live = np.arange(rows) < np.array(counts)[:, None]
    Kb = np.where(live[:, None, :, None], Kb, 0x7FC0).astype(np.uint16)      # NaN where there is no token
    Vb = np.where(live[:, None, :, None], Vb, 0x7F80).astype(np.uint16)
    want_raw, want_scales = co.store(K, V, slots, x.raw, x.scales, dtype)
    c = ugbs.Cache.make(B, Hkv, Hkv, d, x.n_pages, x.max_pages, rows=rows, dtype=dtype)
    cache, scales, table = x.device()
    ugbs.ugbs_cache_store(c, dev_bf16(Kb), dev_bf16(Vb), dev(slots), cache, scales)
    assert np.array_equal(host(scales).view(np.uint32), want_scales.view(np.uint32))
    # byte for byte over the whole cache (a number's zero may have either sign)
    got, used = host(cache), np.isin(np.arange(x.n_pages), np.unique(slots[slots >= 0] // PAGE))
    assert np.array_equal(got[~used], x.raw[~used])
    if dtype == ugbs.E4M3:
        got, want_raw = (np.where(y == 128, 0, y) for y in (got, want_raw))
    for p in np.flatnonzero(used):
        t1 = 1 + max(int(s) % PAGE for s in slots[slots >= 0] if s // PAGE == p)
        for w, at in enumerate((co.key_at(d), co.value_at(d))):
            assert np.array_equal(got[p, :, w][:, at[:t1]], want_raw[p, :, w][:, at[:t1]]), (p, w)
            assert np.array_equal(host(cache)[p, :, w][:, at[t1:]], x.raw[p, :, w][:, at[t1:]]), (p, w)


@pytest.mark.parametrize("dtype", [ugbs.E4M3, ugbs.INT8])
def test_every_bf16_number_is_rounded_once(dtype):
    """All finite bf16 numbers, 64 tokens of 128 channels at a time, sorted by size so that one page
    holds neighbours: bytes and scales as the oracle's, up to the largest number there is."""
    bits = np.arange(65536, dtype=np.uint32).astype(np.uint16)
    bits = bits[(bits & 0x7F80) != 0x7F80]
    bits = bits[np.argsort(bits & 0x7FFF, kind="stable")]
    n = 64 * 128
    B = -(-len(bits) // n)
    bits = np.resize(bits, B * n).reshape(B, 1, 64, 128)
    x = bf16_to_f64(bits)
    table = np.arange(B, dtype=I32)[:, None]
    slots = _slots(table, [0] * B, [64] * B, 64)
    raw, sc = np.zeros((B, 1, 2, n), np.uint8), np.zeros((B, 1, 2), np.float32)
    want_raw, want_sc = co.store(x, x, slots, raw, sc, dtype)
    c = ugbs.Cache.make(B, 1, 1, 128, B, 1, rows=64, dtype=dtype)
    cache, scales = dev(raw), dev(sc)
    t = dev_bf16(bits)
    ugbs.ugbs_cache_store(c, t, t, dev(slots), cache, scales)
    assert np.array_equal(host(scales), want_sc)
    got = host(cache)
    zero = 128 if dtype == ugbs.E4M3 else 0
    assert np.array_equal(np.where(got == zero, 0, got), np.where(want_raw == zero, 0, want_raw))


def test_store_leaves_out_what_it_may_not_write():
    """Slots in no page, and rows whose slot does not follow, are left out; the rest is stored."""
    g = np.random.default_rng(3)
    d, rows, n_pages = 64, 8, 4
    slots = np.array([[PAGE * 9 + i for i in range(8)],                       # page 9 of 4
                      [-1] * 8,
                      [5, 6, 7, 40, 9, 10, -1, 12],                           # 40 does not follow 7
                      [PAGE + 62, PAGE + 63, 2 * PAGE + 1, 2 * PAGE + 2, -1, -1, -1, -1]], I32)   # page 2 begins at token 1
    Kb, K = bf16(g.normal(0, 1, (4, 1, rows, d)))
    c = ugbs.Cache.make(4, 1, 1, d, n_pages, 2, rows=rows)
    raw = np.zeros((n_pages, 1, 2, PAGE * d), np.uint8)
    sc = np.full((n_pages, 1, 2), 2.0 ** -6, np.float32)
    cache, scales = dev(raw), dev(sc)
    ugbs.ugbs_cache_store(c, dev_bf16(Kb), dev_bf16(Kb), dev(slots), cache, scales)
    k, v = co.decode(host(cache), host(scales), 0, d)
    used = np.zeros((n_pages, PAGE), bool)
    for b, i in ((2, 0), (2, 1), (2, 2), (2, 4), (2, 5), (2, 7), (3, 0), (3, 1)):
        p, t = divmod(int(slots[b, i]), PAGE)
        used[p, t] = True
        for y, w in ((k, 0), (v, 1)):
            s = float(host(scales)[p, 0, w])
            assert np.array_equal(y[p, 0, t], co.nearest(K[b, 0, i] / s, 0) * s), (b, i)
    assert not k[:, 0][~used].any() and not v[:, 0][~used].any()


@pytest.mark.parametrize("d,dtype,Hkv", [(64, 0, 3), (128, 0, 2), (128, 1, 1), (256, 1, 2), (256, 0, 1), (64, 1, 4)])
def test_load_is_exact_and_touches_only_its_rows(d, dtype, Hkv):
    g = np.random.default_rng(d + dtype)
    lens = [1, 64, 100, 333, 0, 200]
    x = Contents(g, lens, Hkv, d, dtype, max_pages=7)
    x.table[3, 2] = x.n_pages                      # no page: zeros
    x.table[3, 4] = -1
    cache, scales, table = x.device()
    width = 150
    start = [0, 0, 37, 65, 0, -5]
    count = [1, 64, 63, 500, 0, 150]
    c = ugbs.Cache.make(len(lens), Hkv, Hkv, d, x.n_pages, x.max_pages, dtype=dtype)
    K, V = _load(c, cache, scales, table, start, count, width)
    for b, n in enumerate(lens):
        m, a = min(count[b], width), max(start[b], 0)
        k, v, there = x.tokens(b, a + m)
        k[:, ~there], v[:, ~there] = 0, 0
        assert np.array_equal(K[b, :, :m], k[:, a:]) and np.array_equal(V[b, :, :m], v[:, a:])
        assert np.isnan(K[b, :, m:]).all() and np.isnan(V[b, :, m:]).all()


def test_load_behind_the_table_gives_zeros():
    g = np.random.default_rng(8)
    x = Contents(g, [128, 128], 1, 64, 0)
    c = ugbs.Cache.make(2, 1, 1, 64, x.n_pages, 2)
    K, _ = _load(c, *x.device(), [70, 2 ** 31 - 1], [128, 128], 128)
    k, _, _ = x.tokens(0, 128)
    assert np.array_equal(K[0, :, :58], k[:, 70:]) and not K[0, :, 58:].any() and not K[1].any()


# ---------------------------------------------------------------- attention

def reference(x, b, Qv, kv, q, scale, tiles=False):
    """The oracle's O [H, q, d] and how far the kernel's may be off, elementwise.

    With p the probabilities: their rounding to bf16 is off by 2^-8 of each; a score is a sum of d fp32
    products and three more fp32 roundings, off by (d + 3) 2^-24 sum |q k| scale, which moves p, and the
    sum that divides it, by as much, relatively (e^x - 1 <= 1.01 x here); the exponential, the scale by
    2^x of a moved maximum and the sums over n keys add (n + 64) 2^-24; the result's rounding 2^-8 |O|.

    tiles (many rows, e4m3, d 128 and 256): a query channel is two e4m3 numbers, off by 2^-22 of the
    largest of the 32 channels (in a row) that share a scale."""
    k, v, there = x.tokens(b, max(kv, 0))
    O, sizes, spread = co.attend(Qv, k, v, there, kv, q, scale)
    rel = 2.0 ** -8 + 2.02 * (x.d + 3) * 2.0 ** -24 * spread + (len(there) + 64) * 2.0 ** -24
    if tiles and x.d >= 128 and x.dtype == ugbs.E4M3:
        m = np.repeat(np.abs(Qv).reshape(Qv.shape[:2] + (x.d // 32, 32)).max(3), 32, axis=2)
        big = np.abs(k).max(1, initial=0)                              # [Hkv, d], at least every key's
        rel += 2.02 * 2.0 ** -22 * (m * np.repeat(big, Qv.shape[0] // k.shape[0], 0)[:, None]).sum(2) * scale
    return O, rel[..., None] * sizes * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(O) + 1e-30


def run_attend(c, x, Qb, kv, q, workspace=True, fill=7.0):
    cache, scales, table = x.device()
    O = torch.full(Qb.shape, fill, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(max(256, ugbs.ugbs_cache_workspace_bytes(c)), dtype=torch.uint8, device="cuda")
    ws.fill_(255)                                  # its contents do not matter
    ugbs.ugbs_cache_attend(c, dev_bf16(Qb), cache, scales, table, dev(np.array(kv, I32)), dev(np.array(q, I32)), O, ws)
    torch.cuda.synchronize()
    return O


def check_attend(g, lens, q, rows, H, Hkv, d, dtype, max_pages=None, scale=0.0, spoil=None, loud=1.0, temper=1.0, channels=1.0):
    x = Contents(g, lens, Hkv, d, dtype, max_pages=max_pages, loud=loud)
    if spoil:
        spoil(x)
    B = len(lens)
    Qb, Qv = bf16(g.normal(0, temper, (B, H, rows, d)) * channels)
    for b in range(B):
        Qb[b, :, q[b]:] = 0x7FC0                   # rows without a token are not read
    c = ugbs.Cache.make(B, H, Hkv, d, x.n_pages, x.max_pages, rows=rows, dtype=dtype, scale=scale)
    O = run_attend(c, x, Qb, lens, q)
    got = bf16_to_f64(host_bits(O))
    for b in range(B):
        want, tol = reference(x, b, Qv[b], lens[b], q[b], scale or 1 / math.sqrt(d), rows * H // Hkv > (32 if d < 256 else 16))
        off = np.abs(got[b, :, :q[b]] - want[:, :q[b]])
        assert (off <= tol[:, :q[b]]).all(), (b, float((off - tol[:, :q[b]]).max()), np.argwhere(~(off <= tol[:, :q[b]]))[:3])
        assert (got[b, :, q[b]:] == 7.0).all(), b
    return O


HEADS = [(4, 1), (8, 2), (7, 1), (3, 3), (16, 2), (32, 1), (40, 1), (1, 1)]


@pytest.mark.parametrize("H,Hkv", HEADS)
@pytest.mark.parametrize("d,dtype", [(64, 0), (128, 0), (128, 1), (256, 0), (256, 1), (64, 1)])
def test_one_token_at_every_kind_of_length(H, Hkv, d, dtype):
    g = np.random.default_rng(H * d + dtype)
    lens = [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300, 0, 511]
    check_attend(g, lens, [1] * len(lens), 1, H, Hkv, d, dtype)


@pytest.mark.parametrize("rows,H,Hkv,d,dtype", [
    (2, 8, 2, 128, 0), (4, 28, 4, 128, 0), (5, 16, 2, 256, 1), (3, 3, 3, 64, 0), (16, 4, 4, 128, 1), (17, 7, 1, 64, 0),
    (64, 4, 2, 128, 0), (65, 2, 1, 256, 0), (100, 6, 3, 64, 1), (130, 5, 1, 128, 0), (200, 2, 2, 256, 1)])
def test_several_tokens(rows, H, Hkv, d, dtype):
    g = np.random.default_rng(rows * d + H)
    lens = [rows, rows + 1, 64 * (rows // 64 + 1), rows + 200, 3, 0, rows + 63]
    q = [min(rows, n) for n in lens]
    q[1], q[3] = max(1, rows // 2), rows
    check_attend(g, lens, q, rows, H, Hkv, d, dtype)


@pytest.mark.parametrize("rows,H,Hkv,d,dtype,lens", [
    (1, 8, 2, 128, 0, [3000, 1, 700, 64, 20000]),
    (1, 4, 1, 64, 1, [40000]),
    (1, 28, 4, 128, 0, [9001, 9000, 8999]),
    (1, 16, 2, 256, 0, [12345, 0, 77]),
    (3, 16, 2, 256, 1, [5000, 4097, 3]),
    (40, 8, 2, 128, 0, [6000, 40, 1000]),
    (150, 4, 1, 64, 0, [7000]),
])
def test_long_requests_are_split_and_joined(rows, H, Hkv, d, dtype, lens):
    g = np.random.default_rng(rows + H + d)
    check_attend(g, lens, [min(rows, n) for n in lens], rows, H, Hkv, d, dtype, max_pages=4096)


@pytest.mark.parametrize("rows,H,Hkv,d,dtype,lens", [
    (600, 16, 8, 64, 0, [9000]),                   # 152 tiles in three parts each
    (300, 16, 8, 256, 1, [4000]),
    (257, 16, 4, 128, 0, [3000, 257, 1000]),
    (130, 12, 4, 256, 0, [5000, 64]),
    (1000, 4, 1, 128, 0, [1000]),                  # a whole prompt
    (515, 7, 1, 128, 1, [515, 600, 2000]),
])
def test_pieces_of_prompts(rows, H, Hkv, d, dtype, lens):
    g = np.random.default_rng(rows + d)
    check_attend(g, lens, [min(rows, n) for n in lens], rows, H, Hkv, d, dtype, max_pages=200)


@pytest.mark.parametrize("B,rows,H,Hkv,d,dtype,longest", [
    (64, 1, 4, 2, 64, 0, 9000), (65, 1, 4, 2, 64, 0, 0), (256, 1, 4, 1, 64, 1, 5000), (257, 1, 4, 2, 64, 0, 9000),
    (300, 9, 4, 1, 64, 0, 3000), (300, 3, 8, 1, 128, 0, 0), (700, 20, 2, 1, 64, 1, 2500), (4096, 1, 2, 1, 64, 0, 1500)])
def test_many_requests_among_them_a_long_one(B, rows, H, Hkv, d, dtype, longest):
    g = np.random.default_rng(B + rows)
    lens = [int(n) for n in g.integers(0, 130 if B > 500 else 200, B)]
    lens[B // 2 + 7] = longest
    q = [int(min(n, m)) for n, m in zip(lens, g.integers(0, rows + 1, B))]
    q[B // 2 + 7] = min(rows, longest)
    check_attend(g, lens, q, rows, H, Hkv, d, dtype, max_pages=200)


@pytest.mark.parametrize("B,rows,H,Hkv,d,dtype,longest", [
    (64, 1, 4, 1, 128, 0, 30000), (300, 1, 4, 1, 128, 1, 40000), (64, 3, 8, 1, 256, 0, 20000), (70, 9, 4, 1, 64, 0, 40000),
    (300, 20, 4, 1, 128, 0, 30000), (100, 2, 8, 2, 128, 0, 33333), (260, 5, 4, 2, 256, 1, 50000)])
def test_tiles_of_many_parts_among_many_tiles(B, rows, H, Hkv, d, dtype, longest):
    g = np.random.default_rng(B + rows + d)
    lens = [int(n) for n in g.integers(0, 70, B)]
    lens[B // 3], lens[B - 1] = longest, 3000      # above 32 parts a tile, and a few
    q = [int(min(n, m)) for n, m in zip(lens, g.integers(0, rows + 1, B))]
    q[B // 3] = q[B - 1] = rows
    check_attend(g, lens, q, rows, H, Hkv, d, dtype, max_pages=1000)


def test_sharp_and_flat_softmax():
    """Scores that differ by hundreds (one key takes all) and by nothing."""
    for temper in (0.0, 60.0):
        g = np.random.default_rng(5)
        check_attend(g, [500, 64, 1000], [1, 1, 1], 1, 4, 1, 128, 0, temper=temper)
        check_attend(g, [500, 640], [100, 30], 100, 4, 1, 128, 1, temper=temper)


@pytest.mark.parametrize("d", [128, 256])
@pytest.mark.parametrize("rows", [1, 70])
def test_channels_of_very_different_size(rows, d):
    """Query channels from 1 to 2^-17 of the largest, and keys that make up for some of it."""
    g = np.random.default_rng(d + rows)
    channels = 2.0 ** -g.integers(0, 18, d) * 30

    def spoil(x):                                  # the loudest quarter of the channels has keys of 0
        k, v = co.decode(x.raw, np.ones_like(x.scales), x.dtype, d)
        live = np.isfinite(k)
        k[..., channels > 2.0 ** -4 * 30] = 0
        enc = co.encode(np.where(live, k, 0), np.where(np.isfinite(v), v, 0), x.dtype)
        x.raw[:, :, 0] = enc[:, :, 0]
    check_attend(g, [300, 128], [min(rows, n) for n in (300, 128)], rows, 4, 2, d, 0, spoil=spoil, channels=channels, scale=1.0)


def test_pages_of_very_different_scales():
    def spoil(x):
        x.scales[:, :, 1] *= 2.0 ** g.integers(-40, 40, x.scales[:, :, 1].shape)
        x.scales[:, :, 0] *= 2.0 ** g.integers(-60, 1, x.scales[:, :, 0].shape)
    g = np.random.default_rng(6)
    check_attend(g, [1000, 130], [1, 1], 1, 8, 2, 128, 0, spoil=spoil)
    check_attend(g, [1000, 130], [70, 70], 70, 8, 2, 128, 1, spoil=spoil)


@pytest.mark.parametrize("rows", [1, 70])
def test_entries_that_are_no_page_are_left_out(rows):
    """Rows that then see no key at all give 0."""
    def spoil(x):
        x.table[0, 1] = -1
        x.table[0, 3] = x.n_pages
        x.table[1, :] = 2 ** 31 - 1
        x.table[2, 0] = -2 ** 31
    g = np.random.default_rng(rows)
    for d in (64, 128, 256):
        O = check_attend(g, [400, 200, 64 + rows], [rows] * 3, rows, 4, 2, d, 0, spoil=spoil)
        assert not O[1].any()


@pytest.mark.parametrize("rows", [1, 70])
def test_more_new_tokens_than_cached_ones(rows):
    """kv_len < q_len: the first rows sit before the cache and see nothing; their O is 0."""
    g = np.random.default_rng(rows)
    for d in (64, 256):
        O = check_attend(g, [0, rows // 2, rows], [rows] * 3, rows, 4, 2, d, 1)
        assert not O[0].any() and not O[1, :, :rows - rows // 2].any()


def test_lengths_outside_their_range_are_clamped():
    g = np.random.default_rng(9)
    x = Contents(g, [128, 128, 128], 1, 64, 0)
    Qb, Qv = bf16(g.normal(0, 1, (3, 2, 2, 64)))
    c = ugbs.Cache.make(3, 2, 1, 64, x.n_pages, 2, rows=2)
    O = run_attend(c, x, Qb, [2 ** 31 - 1, -4, 128], [5, 2, -1])
    got = bf16_to_f64(host_bits(O))
    want, tol = reference(x, 0, Qv[0], 128, 2, 1 / 8)
    assert (np.abs(got[0] - want) <= tol).all()
    assert not got[1].any() and (got[2] == 7.0).all()


@pytest.mark.parametrize("rows,lens", [(1, [5000, 300, 9000]), (90, [900, 4000])])
def test_two_calls_give_the_same_bits(rows, lens):
    g = np.random.default_rng(12)
    x = Contents(g, lens, 2, 128, 0, max_pages=300)
    Qb, _ = bf16(g.normal(0, 1, (len(lens), 8, rows, 128)))
    c = ugbs.Cache.make(len(lens), 8, 2, 128, x.n_pages, 300, rows=rows)
    a, b = (run_attend(c, x, Qb, lens, [rows] * len(lens)) for _ in range(2))
    assert torch.equal(a.view(torch.int16), b.view(torch.int16))


@pytest.mark.parametrize("rows", [1, 40])
def test_offsets_pass_32_bits(rows):
    """A cache of more than 4 GiB, its last pages used."""
    d, Hkv, n_pages = 256, 8, 20000                # 5.2e9 bytes
    g = np.random.default_rng(14)
    lens = [150, 70]
    small = Contents(g, lens, Hkv, d, 0)
    shift = n_pages - small.n_pages
    cache = torch.zeros((n_pages, Hkv, 2, PAGE * d), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((n_pages, Hkv, 2), dtype=torch.float32, device="cuda")
    cache[shift:] = dev(small.raw)
    scales[shift:] = dev(small.scales)
    table = np.where(small.table >= 0, small.table + shift, -1).astype(I32)
    Qb, Qv = bf16(g.normal(0, 1, (2, 8, rows, d)))
    c = ugbs.Cache.make(2, 8, Hkv, d, n_pages, small.max_pages, rows=rows)
    O = torch.zeros((2, 8, rows, d), dtype=torch.bfloat16, device="cuda")
    ugbs.ugbs_cache_attend(c, dev_bf16(Qb), cache, scales, dev(table), dev(np.array(lens, I32)), dev(np.array([rows] * 2, I32)), O,
                           torch.empty(max(256, ugbs.ugbs_cache_workspace_bytes(c)), dtype=torch.uint8, device="cuda"))
    for b in range(2):
        want, tol = reference(small, b, Qv[b], lens[b], rows, 1 / 16, rows > 16)
        assert (np.abs(bf16_to_f64(host_bits(O[b])) - want) <= tol).all()
    # a token stored into the last page, and loaded
    c = ugbs.Cache.make(2, 8, Hkv, d, n_pages, small.max_pages)
    Kb, K = bf16(g.normal(0, 1, (2, Hkv, 1, d)))
    slots = np.array([[-1], [(n_pages - 1) * PAGE]], I32)
    ugbs.ugbs_cache_store(c, dev_bf16(Kb), dev_bf16(Kb), dev(slots), cache, scales)
    tb = np.full((2, small.max_pages), n_pages - 1, I32)
    k, v = _load(c, cache, scales, dev(tb), [0, 0], [0, 1], 1)
    for h in range(Hkv):
        s = co.scale_of(np.abs(K[1, h]).max(), 0)
        assert np.array_equal(k[1, h], co.nearest(K[1, h] / s, 0) * s) and np.array_equal(v[1, h], k[1, h])


# ---------------------------------------------------------------- steps

class Mirror:
    """The oracle's state of a run: what CacheStep and CacheBuffers hold."""

    def __init__(self, c):
        self.stack, self.count = np.arange(c.n_pages, dtype=I32), c.n_pages
        self.table = np.full((c.batch, c.max_pages), -1, I32)
        self.kv = np.zeros(c.batch, I32)
        self.raw = np.zeros((c.n_pages, c.n_kv_heads, 2, PAGE * c.head_dim), np.uint8)
        self.scales = np.zeros((c.n_pages, c.n_kv_heads, 2), np.float32)
        self.n_pages, self.Hkv, self.d, self.dtype = c.n_pages, c.n_kv_heads, c.head_dim, c.dtype

    tokens = Contents.tokens

    def step(self, new, K, V, rows):
        self.stack, self.table, self.kv, self.q, slots, self.count = co.plan(self.kv, new, self.stack, self.count, self.table, rows)
        self.raw, self.scales = co.store(K, V, slots, self.raw, self.scales, self.dtype)


def _check_step(mir, O, Qv, scale):
    got = bf16_to_f64(host_bits(O))
    for b in range(Qv.shape[0]):
        n = int(mir.q[b])
        want, tol = reference(mir, b, Qv[b], int(mir.kv[b]), n, scale)
        assert (np.abs(got[b, :, :n] - want[:, :n]) <= tol[:, :n]).all(), b


@pytest.mark.parametrize("dtype", [ugbs.E4M3, ugbs.INT8])
def test_prompts_then_tokens_then_other_requests(dtype):
    """Prompts through the sparse prefill into the cache, single tokens, drafts of several, a request that
    ends and one that takes its pages; after each step O, lengths and free pages are the oracle's."""
    g = np.random.default_rng(30 + dtype)
    B, H, Hkv, d, N = 2, 4, 2, 64, 256
    cp = ugbs.Cache.make(B, H, Hkv, d, 14, 8, rows=N, dtype=dtype)
    cbufs, step, mir = ugbs.CacheBuffers(cp), ugbs.CacheStep(cp), Mirror(cp)
    cbufs.cache.fill_(0)
    p = ugbs.Problem.make(B, H, Hkv, N, d, 4, 0.25)
    Qb, _ = bf16(g.normal(0, 1, (B, H, N, d)))
    Kb, K = bf16(g.normal(0, 1, (B, Hkv, N, d)))
    Vb, V = bf16(g.normal(0, 1, (B, Hkv, N, d)))
    t = [dev_bf16(x) for x in (Qb, Kb, Vb)]
    O, O2 = torch.empty_like(t[0]), torch.empty_like(t[0])
    new = np.array([N, N], I32)
    step.plan(cp, dev(new))
    ugbs.prefill_cached(p, cp, *t, O, ugbs.Buffers(p), cbufs, step)
    ugbs.prefill(p, *t, O2, ugbs.Buffers(p))
    assert torch.equal(O.view(torch.int16), O2.view(torch.int16))      # the prefill itself is what it was
    mir.step(new, K, V, N)
    with pytest.raises(ValueError):
        step.plan(ugbs.Cache.make(B, H, Hkv, d, 14, 8, rows=N + 1), dev(new))
    with pytest.raises(ValueError):
        ugbs.prefill_cached(p, ugbs.Cache.make(B, H, Hkv, d, 14, 8, rows=64), *t, O, None, cbufs, step)
    for rows, new in ((1, [1, 1]), (1, [1, 1]), (5, [5, 2]), (1, [1, -1]), (70, [70, 60]), (70, [70, 70]), (1, [1, 0])):
        c = ugbs.Cache.make(B, H, Hkv, d, 14, 8, rows=rows, dtype=dtype)
        Qb, Qv = bf16(g.normal(0, 1, (B, H, rows, d)))
        Kb, K = bf16(g.normal(0, 2.0, (B, Hkv, rows, d)))
        Vb, V = bf16(g.normal(0, 2.0, (B, Hkv, rows, d)))
        step.plan(c, dev(np.array(new, I32)))
        O = torch.zeros((B, H, rows, d), dtype=torch.bfloat16, device="cuda")
        ugbs.cache_layer(c, dev_bf16(Qb), dev_bf16(Kb), dev_bf16(Vb), O, cbufs, step)
        mir.step(np.array(new, I32), K, V, rows)
        assert np.array_equal(host(step.kv_lens), mir.kv) and np.array_equal(host(step.q_lens), mir.q)
        assert int(step.free_left.item()) == mir.count and np.array_equal(host(step.table), mir.table)
        _check_step(mir, O, Qv, 1 / math.sqrt(d))


def test_a_captured_step_replays_as_lengths_grow():
    """plan, store and attend of single tokens in one graph, eager work and synchronisation in between;
    each replay against the same step done eagerly on a copy, bit for bit."""
    g = np.random.default_rng(40)
    B, H, Hkv, d = 3, 8, 2, 128
    c = ugbs.Cache.make(B, H, Hkv, d, 64, 20)
    Qb, Kb, Vb = (bf16(g.normal(0, 1, (B, h, 1, d)))[0] for h in (H, Hkv, Hkv))
    Q, K, V = dev_bf16(Qb), dev_bf16(Kb), dev_bf16(Vb)
    new = dev(np.array([1, 1, 1], I32))
    sides = []
    for _ in range(2):
        cbufs, step = ugbs.CacheBuffers(c), ugbs.CacheStep(c)
        cbufs.cache.zero_()
        cbufs.scales.zero_()
        sides.append((cbufs, step, torch.zeros_like(Q)))

    def one(side):
        cbufs, step, O = side
        step.plan(c, new)
        ugbs.cache_layer(c, Q, K, V, O, cbufs, step)

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
    for rep in range(130):                         # across two page borders
        Q.copy_(torch.randn(Q.shape, generator=torch.Generator().manual_seed(rep)).to(torch.bfloat16))
        K.copy_(Q[:, :Hkv] * (1 + rep % 7))
        V.copy_(Q[:, Hkv:2 * Hkv] * (1 + rep % 5))
        graph.replay()
        torch.cuda.synchronize()
        sides[0][1].slots.clone()
        one(sides[1])
        torch.cuda.synchronize()
        assert torch.equal(sides[0][2].view(torch.int16), sides[1][2].view(torch.int16)), rep
        assert torch.equal(sides[0][1].table, sides[1][1].table) and torch.equal(sides[0][1].kv_lens, sides[1][1].kv_lens)
    assert sides[0][1].kv_lens.tolist() == [131] * 3


def test_two_graphs_share_a_workspace():
    """Captured calls of different sizes over one workspace, replayed in turn."""
    g = np.random.default_rng(45)
    x = Contents(g, [5000, 300], 2, 128, 0, max_pages=100)
    cache, scales, table = x.device()
    kv, q1 = dev(np.array([5000, 300], I32)), dev(np.array([1, 1], I32))
    calls = []
    for rows, n in ((1, 1), (40, 40)):
        c = ugbs.Cache.make(2, 8, 2, 128, x.n_pages, 100, rows=rows)
        Qb, Qv = bf16(g.normal(0, 1, (2, 8, rows, 128)))
        calls.append((c, dev_bf16(Qb), Qv, dev(np.array([n, n], I32)), torch.zeros((2, 8, rows, 128), dtype=torch.bfloat16, device="cuda")))
    ws = torch.empty(max(ugbs.ugbs_cache_workspace_bytes(y[0]) for y in calls), dtype=torch.uint8, device="cuda")
    graphs = []
    for c, Q, _, q, O in calls:
        ugbs.ugbs_cache_attend(c, Q, cache, scales, table, kv, q, O, ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            ugbs.ugbs_cache_attend(c, Q, cache, scales, table, kv, q, O, ws)
        graphs.append(graph)
    want = [O.clone() for *_, O in calls]
    for rep in range(4):
        for *_, O in calls:
            O.fill_(3.0)
        ws.fill_(rep)
        for graph in graphs if rep % 2 else graphs[::-1]:
            graph.replay()
        torch.cuda.synchronize()
        for (c, _, Qv, q, O), w in zip(calls, want):
            assert torch.equal(O.view(torch.int16), w.view(torch.int16)), rep
    for c, _, Qv, q, O in calls:
        for b in range(2):
            ref, tol = reference(x, b, Qv[b], [5000, 300][b], c.rows, 1 / math.sqrt(128), c.rows > 1)
            assert (np.abs(bf16_to_f64(host_bits(O[b])) - ref) <= tol).all()


def test_streams_of_their_own():
    """Two calls at once on two streams, each with its workspace, given as handle and as current stream."""
    g = np.random.default_rng(50)
    lens = [4000, 900]
    x = Contents(g, lens, 2, 128, 0, max_pages=100)
    Qb, Qv = bf16(g.normal(0, 1, (2, 8, 1, 128)))
    c = ugbs.Cache.make(2, 8, 2, 128, x.n_pages, 100)
    cache, scales, table = x.device()
    kv, q, Q = dev(np.array(lens, I32)), dev(np.array([1, 1], I32)), dev_bf16(Qb)
    outs = [torch.zeros_like(Q) for _ in range(2)]
    ws = [torch.empty(ugbs.ugbs_cache_workspace_bytes(c), dtype=torch.uint8, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    s = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        ugbs.ugbs_cache_attend(c, Q, cache, scales, table, kv, q, outs[0], ws[0], stream=s[0].cuda_stream)
        with torch.cuda.stream(s[1]):
            ugbs.ugbs_cache_attend(c, Q, cache, scales, table, kv, q, outs[1], ws[1])
    torch.cuda.synchronize()
    for b in range(2):
        want, tol = reference(x, b, Qv[b], lens[b], 1, 1 / math.sqrt(128))
        for O in outs:
            assert (np.abs(bf16_to_f64(host_bits(O[b])) - want) <= tol).all()


def test_a_step_on_streams_given_as_handles():
    g = np.random.default_rng(55)
    c = ugbs.Cache.make(2, 4, 2, 64, 20, 4)
    Qb, Kb, Vb = (bf16(g.normal(0, 1, (2, h, 1, 64)))[0] for h in (4, 2, 2))
    t = [dev_bf16(x) for x in (Qb, Kb, Vb)]
    new = dev(np.array([1, 1], I32))
    side = torch.cuda.Stream()
    outs = []
    for stream in (None, side.cuda_stream, 0):
        cbufs, step = ugbs.CacheBuffers(c), ugbs.CacheStep(c)
        O = torch.zeros_like(t[0])
        torch.cuda.synchronize()
        for _ in range(3):
            step.plan(c, new, stream)
            ugbs.cache_layer(c, *t, O, cbufs, step, stream)
        torch.cuda.synchronize()
        assert step.kv_lens.tolist() == [3, 3] and int(step.free_left.item()) == 18
        outs.append(O)
    assert all(torch.equal(outs[0].view(torch.int16), x.view(torch.int16)) for x in outs)


def test_cached_prompt_through_the_sparse_prefill():
    """Loaded keys and values are bf16 tensors like any other: the prefill over them equals the prefill
    over the same numbers."""
    g = np.random.default_rng(60)
    B, H, Hkv, d, N = 1, 4, 2, 128, 512
    c = ugbs.Cache.make(B, H, Hkv, d, 10, 8, rows=N)
    cbufs, step = ugbs.CacheBuffers(c), ugbs.CacheStep(c)
    Kb, Kv = bf16(g.normal(0, 1, (B, Hkv, N, d)))
    Vb, Vv = bf16(g.normal(0, 1, (B, Hkv, N, d)))
    step.plan(c, dev(np.array([N], I32)))
    ugbs.ugbs_cache_store(c, dev_bf16(Kb), dev_bf16(Vb), step.slots, cbufs.cache, cbufs.scales)
    K, V = (torch.empty((B, Hkv, N, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    ugbs.ugbs_cache_load(c, cbufs.cache, cbufs.scales, step.table, zero, step.kv_lens, K, V)
    for got, x in ((K, Kv), (V, Vv)):
        y = x.reshape(Hkv, N // PAGE, PAGE, d)
        want = np.empty_like(y)
        for h in range(Hkv):
            for j in range(N // PAGE):
                s = co.scale_of(np.abs(y[h, j]).max(), 0)
                want[h, j] = co.nearest(y[h, j] / s, 0) * s
        assert np.array_equal(bf16_to_f64(host_bits(got)).reshape(y.shape), want)
    p = ugbs.Problem.make(B, H, Hkv, N, d, 4, 0.25, ugbs.QUEST)
    Qb, _ = bf16(g.normal(0, 1, (B, H, N, d)))
    O = torch.empty((B, H, N, d), dtype=torch.bfloat16, device="cuda")
    ugbs.prefill(p, dev_bf16(Qb), K, V, O, ugbs.Buffers(p))
    assert bool(torch.isfinite(O.float()).all())
