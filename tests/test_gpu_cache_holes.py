"""Steps over tables and stacks with entries that are no page: what would lie there is left out, all else
is stored and attended as ever."""
import math

import numpy as np
import pytest
import torch

import cache_oracle as co
import paper_2607_07724_amd as ugbs

from gpu_helpers import bf16_to_f64, dev, dev_bf16, host, host_bits
from test_gpu_cache import I32, PAGE, Contents, bf16, pages, reference, run_attend

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need an MI355X (gfx950) visible to torch")
    ugbs.lib()


def store_past_holes(K, V, slots, raw, scales, dtype):
    """The oracle's store of each run of rows that have slots."""
    B, _, rows, _ = K.shape
    for b in range(B):
        i = 0
        while i < rows:
            n = 0
            while i + n < rows and slots[b, i + n] >= 0:
                n += 1
            if n:
                one = np.s_[b:b + 1, :, i:i + n]
                raw, scales = co.store(K[one], V[one], slots[b:b + 1, i:i + n], raw, scales, dtype)
            i += n + 1
    return raw, scales


@pytest.mark.parametrize("d,dtype", [(64, 0), (128, 0), (128, 1), (256, 1)])
@pytest.mark.parametrize("rows", [64, 65, 150, 300])
def test_pages_that_are_missing_take_nothing_from_the_others(rows, d, dtype):
    """plan, store and attend: requests whose first page, first pages, or a middle page is none."""
    g = np.random.default_rng(rows + d + dtype)
    H, Hkv = 4, 2
    ctx = [100, 0, 30, 0, 10, 0, 64, 200]
    new = [rows, rows, rows, rows, rows, 0, rows, min(rows, 70)]
    # new pages of a request, by place, that the stack has not
    gone = {1: (0,), 2: (0,), 3: (0, 1), 6: (0, 2), 7: (0,)}
    B = len(ctx)
    max_pages = max(pages(c + n) for c, n in zip(ctx, new)) + 1
    n_pages = B * max_pages
    x = Contents(g, ctx, Hkv, d, dtype, max_pages=max_pages, n_pages=n_pages)
    x.table[0, 1] = -1                                   # request 0 goes on inside a page that is none
    free = [p for p in g.permutation(n_pages) if p not in x.table]
    taken = []
    for b in range(B):
        for j in range(pages(ctx[b] + new[b]) - pages(ctx[b])):
            taken.append(int(g.choice([-1, n_pages, 2 ** 31 - 1])) if j in gone.get(b, ()) else int(free.pop()))
    stack = np.full(n_pages, -1, I32)
    stack[:len(taken)] = taken[::-1]
    want = co.plan(ctx, new, stack, len(taken), x.table, rows)
    c = ugbs.Cache.make(B, H, Hkv, d, n_pages, max_pages, rows=rows, dtype=dtype)
    cache, scales, table = x.device()
    kv, q, left = (torch.full((n,), -9, dtype=torch.int32, device="cuda") for n in (B, B, 1))
    slots = torch.full((B, rows), -9, dtype=torch.int32, device="cuda")
    ugbs.ugbs_cache_plan(c, dev(np.array(ctx, I32)), dev(np.array(new, I32)), dev(stack), dev(np.array([len(taken)], I32)),
                         table, kv, q, slots, left)
    for a, b in zip((table, kv, q, slots), want[1:5]):
        assert np.array_equal(host(a), b)
    Kb, K = bf16(g.normal(0, 1, (B, Hkv, rows, d)))
    Vb, V = bf16(g.normal(0, 1, (B, Hkv, rows, d)))
    ugbs.ugbs_cache_store(c, dev_bf16(Kb), dev_bf16(Vb), slots, cache, scales)
    x.table = want[1]
    x.raw, x.scales = store_past_holes(K, V, want[4], x.raw, x.scales, dtype)
    assert np.array_equal(host(scales).view(np.uint32), x.scales.view(np.uint32))
    got, raw = host(cache), x.raw
    if dtype == ugbs.E4M3:                               # a number's zero may have either sign
        got, raw = (np.where(y == 128, 0, y) for y in (got, raw))
    assert np.array_equal(got, raw)
    Qb, Qv = bf16(g.normal(0, 1, (B, H, rows, d)))
    O = bf16_to_f64(host_bits(run_attend(c, x, Qb, want[2], want[3])))
    for b in range(B):
        n = int(want[3][b])
        ref, tol = reference(x, b, Qv[b], int(want[2][b]), n, 1 / math.sqrt(d), True)
        assert (np.abs(O[b, :, :n] - ref[:, :n]) <= tol[:, :n]).all(), b
