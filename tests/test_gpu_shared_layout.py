"""The layout that ugbs_cache_share writes, read back: every page of every request is attended once, by the parts of its group's
prefix or by its own; the rows of the parts' sums lie in the workspace and do not overlap; there is room for all parts."""
import numpy as np
import pytest
import torch

import paper_2607_07724_amd as ugbs
from gpu_helpers import dev, host

pytestmark = pytest.mark.gpu

I32 = np.int32
OF_PREFIX = 1 << 24


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need an MI355X (gfx950) visible to torch")
    ugbs.lib()


def align(n):
    return -(-n // 256) * 256


def layout(c, group, table, kv, q):
    """The arrays of a layout, in the order in which they lie in it (cache_attend.h, Share)."""
    B, G = c.batch, c.n_heads // c.n_kv_heads
    total = ugbs.ugbs_cache_share_bytes(c)
    share = torch.full((total,), 171, dtype=torch.uint8, device="cuda")
    ugbs.ugbs_cache_share(c, dev(group), dev(table), dev(kv), dev(q), share)
    raw = host(share).view(I32)
    own = raw[:8 * B].reshape(B, 2, 4)
    first = 2 * align(32 * B)
    last = total - align(16 * B) - align(8 * B * c.rows * G)
    parts = raw[first // 4:last // 4]
    parts = parts[:len(parts) // 8 * 8].reshape(-1, 8)
    parts = parts[(parts != -1414812757).any(1)]               # (the end of the last 256 bytes is not written: 0xab..)
    return own, parts[parts[:, 0] >= 0], raw[last // 4:last // 4 + 2 * B * c.rows * G].reshape(-1, 2)


def check(c, group, table, kv, q):
    B, H, Hkv, rows, d = c.batch, c.n_heads, c.n_kv_heads, c.rows, c.head_dim
    G = H // Hkv
    own, parts, row = layout(c, group, table, kv, q)
    many = 32 if d == 256 else 64
    tile = lambda n, some: 16 if n <= 16 else 32 if some and n <= 32 else many
    own_rows, prefix_rows = tile(rows * G, True), tile(B * rows * G, False)
    sums = ugbs.ugbs_cache_shared_workspace_bytes(c) // (4 * d + 8)
    used = np.zeros(sums, bool)
    # pages seen by each (request, kv head, query row): as intervals, collected per key
    seen = {}
    for b, kvh, t, p0, p1, at, n, more in parts.tolist():
        assert 0 <= p0 <= p1 <= c.max_pages
        prefix = kvh >= OF_PREFIX
        kvh -= OF_PREFIX if prefix else 0
        size = prefix_rows if prefix else own_rows
        live = min(size, n * G - t * size)
        assert 0 <= kvh < Hkv and live > 0
        if at >= 0:
            assert at + live <= sums and not used[at:at + live].any()
            used[at:at + live] = True
        else:
            assert not prefix
        for r in range(t * size, t * size + live):
            if prefix:
                q_row, last = row[more * G + r].tolist()
                i, bh = q_row % rows, q_row // rows
                who = bh // H
                assert bh % H == r % G and last == kv[who] - q[who] + i and i < q[who]
                key = who, kvh, i * G + r % G
            else:
                assert n == q[b] and more == kv[b]
                key = b, kvh, r
            seen.setdefault(key, []).append((p0, p1, at < 0))
    for b in range(B):
        for r in range(q[b] * G):
            end = -(-max(0, kv[b] - q[b] + r // G + 1) // 64)          # pages that the row sees
            for kvh in range(Hkv):
                mine = sorted(seen.pop((b, kvh, r)))
                assert mine[0][0] == 0 and all(x[1] == y[0] for x, y in zip(mine, mine[1:])) and mine[-1][1] >= end, (b, kvh, r, mine)
                assert len(mine) == 1 or not any(x[2] for x in mine)
    assert not seen
    return parts


@pytest.mark.parametrize("seed", range(24))
def test_every_page_is_attended_once(seed):
    g = np.random.default_rng(seed)
    H, Hkv = [(4, 1), (8, 2), (7, 1), (16, 2), (3, 3), (32, 1), (28, 4)][seed % 7]
    d = [64, 128, 256][seed % 3]
    G = H // Hkv
    rows = int(g.integers(1, max(2, min(9, 64 // G + 1))))
    B = int(g.choice([2, 3, 17, 64, 65, 200, 257, 300, 1030] if seed % 2 else [2, 5, 30, 90]))
    mp = int(g.choice([3, 9, 40, 300, 2500]))
    if B > 100:
        mp = min(mp, 40)
    c = ugbs.Cache.make(B, H, Hkv, d, 1 << 20, mp, rows=rows)
    group = g.integers(-1, max(1, B // int(g.integers(1, 12))), B).astype(I32)
    # lengths that spread over orders of magnitude, some requests without new tokens
    kv = np.minimum(np.exp(g.uniform(0, np.log(64 * mp), B)).astype(int) + rows, 64 * mp).astype(I32)
    if seed % 4 == 0:
        kv[:] = 64 * mp - g.integers(0, 64, B)
    q = np.minimum(g.integers(0, rows + 1, B), kv).astype(I32)
    table = g.permutation(1 << 20)[:B * mp].reshape(B, mp).astype(I32)
    for n in np.unique(group[group >= 0]):
        who = np.flatnonzero(group == n)
        common = int(g.integers(0, mp + 1))
        table[who, :common] = table[who[0], :common]
    check(c, group, table, kv, q)


@pytest.mark.parametrize("B,H,Hkv,d,mp", [(4, 28, 4, 128, 4096), (9, 32, 8, 64, 3000), (40, 16, 2, 256, 700), (2, 1, 1, 64, 4096), (64, 4, 1, 128, 500)])
def test_one_long_prefix_uses_the_chip(B, H, Hkv, d, mp):
    c = ugbs.Cache.make(B, H, Hkv, d, 1 << 20, mp)
    table = np.broadcast_to(np.arange(mp, dtype=I32), (B, mp)).copy()
    table[:, -2:] = 10000 + np.arange(2 * B).reshape(B, 2)
    kv = np.full(B, 64 * mp - 7, I32)
    parts = check(c, np.zeros(B, I32), table, kv, np.ones(B, I32))
    prefix = parts[parts[:, 1] >= OF_PREFIX]
    assert prefix[:, 4].max() == mp - 2 and 100 <= len(prefix) <= 520
