"""Tokens that are not finite, stored into the cache: the other tokens of their pages stay what they are."""
import numpy as np
import pytest
import torch

import cache_oracle as co
import paper_2607_07724_amd as ugbs

from gpu_helpers import bf16_to_f64, dev, dev_bf16, host, host_bits
from test_gpu_cache import I32, PAGE, Contents, _load, _slots, bf16, run_attend

pytestmark = pytest.mark.gpu

INF, NAN = 0x7F80, 0x7FC0


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need an MI355X (gfx950) visible to torch")
    ugbs.lib()


@pytest.mark.parametrize("dtype", [ugbs.E4M3, ugbs.INT8])
@pytest.mark.parametrize("rows,lens,d", [
    (1, [40, 1, 63, 64, 0], 64),            # one token into pages in use, and new ones
    (5, [30, 62, 0], 128),
    (64, [0, 0, 17], 256),                  # whole pages
    (130, [0, 33], 128),
])
def test_other_tokens_keep_their_numbers(rows, lens, d, dtype):
    g = np.random.default_rng(rows + d + dtype)
    B, H, Hkv = len(lens), 4, 2
    x = Contents(g, [n + rows for n in lens], Hkv, d, dtype)
    bits, spoilt = [], []
    for _ in range(2):
        b, _ = bf16(g.normal(0, 1, (B, Hkv, rows, d)))
        b[0, 0, rows // 2] = NAN                         # a whole token
        at = g.random(b.shape) < 0.01
        at[:, :, 0, 3] = True
        b[at] = g.choice(np.array([INF, INF | 0x8000, NAN, 0x7F81, 0xFFFF], np.uint16), at.sum())
        bits.append(b)
        spoilt.append((b & 0x7F80) == 0x7F80)
    slots = _slots(x.table, lens, [rows] * B, rows)
    K, V = (bf16_to_f64(np.where(s, 0, b).astype(np.uint16)) for b, s in zip(bits, spoilt))
    raw, sc = co.store(K, V, slots, x.raw, x.scales, dtype)
    top = co.encode(*(np.full((1, 1, PAGE, d), y) for y in (co.TOP[dtype], -co.TOP[dtype])), dtype).reshape(2, -1)[:, 0]
    for w, (b, at) in enumerate(zip(bits, (co.key_at(d), co.value_at(d)))):
        for r, h, i, c in np.argwhere((b & 0x7FFF) == INF):
            p, t = divmod(int(slots[r, i]), PAGE)
            raw[p, h, w, at[t, c]] = top[int(b[r, h, i, c] >> 15)]
    c = ugbs.Cache.make(B, H, Hkv, d, x.n_pages, x.max_pages, rows=rows, dtype=dtype)
    cache, scales, table = x.device()
    ugbs.ugbs_cache_store(c, *(dev_bf16(b) for b in bits), dev(slots), cache, scales)
    assert np.array_equal(host(scales).view(np.uint32), sc.view(np.uint32))
    got = host(cache)
    if dtype == ugbs.E4M3:                               # a number's zero may have either sign
        got, raw = (np.where(y == 128, 0, y) for y in (got, raw))
    assert np.array_equal(got, raw)
    # and all that is read back is finite
    Kb, Vb = _load(c, cache, scales, table, [0] * B, [n + rows for n in lens], max(lens) + rows, fill=0.0)
    assert np.isfinite(Kb).all() and np.isfinite(Vb).all()
    x.raw, x.scales = host(cache), host(scales)
    Qb, _ = bf16(g.normal(0, 1, (B, H, rows, d)))
    assert np.isfinite(bf16_to_f64(host_bits(run_attend(c, x, Qb, [n + rows for n in lens], [rows] * B)))).all()
