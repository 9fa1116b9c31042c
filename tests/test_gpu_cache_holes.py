"""Steps over tables and stacks with entries that are no page: what would lie there is left out, all else
is stored and attended as ever."""
import math

import numpy as np
import pytest
import torch

import cache_oracle as co
import paper_2607_07724_amd as ugbs

from gpu_helpers import bf16_to_f64, dev, dev_bf16, host, host_bits
from test_gpu_cache import I32, PAGE, Contents, Mirror, _check_step, _plan_case, _run_plan, bf16, pages, reference, run_attend

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


# ---------------------------------------------------------------- what a released request gives back

def plan_past_holes(ctx, new, stack, count, table, rows):
    """The oracle's plan after the rows of released requests were closed up over what is no page."""
    closed, ctx = table.copy(), ctx.copy()
    gone = [b for b in range(len(ctx)) if new[b] == -1 and 0 <= ctx[b] <= PAGE * table.shape[1]]
    for b in gone:
        row = [p for p in table[b, :pages(int(ctx[b]))] if 0 <= p < len(stack)]
        closed[b, :len(row)], ctx[b] = row, PAGE * len(row)
    out = co.plan(ctx, new, stack, count, closed, rows)
    out[1][gone] = table[gone]
    return out


@pytest.mark.parametrize("B,max_pages,rows,stock,wild,room", [
    (1, 1, 1, 1, False, 50), (2, 300, 64, 1, False, 50), (5, 4, 100, 0.5, False, 1), (64, 6, 3, 1, False, 0), (65, 9, 65, 0, False, 50),
    (257, 5, 7, 0.3, True, 50), (1000, 3, 130, 0, True, 50), (4096, 2, 1, 0.5, True, 50), (30, 150, 2000, 0, False, 50)])
def test_entries_that_are_no_page_are_not_given_back(B, max_pages, rows, stock, wild, room):
    g = np.random.default_rng(B + max_pages)
    for share in (0.02, 0.3, 1.0):
        ctx, new, stack, count, table = _plan_case(g, B, max_pages, rows, stock, wild)
        new[g.random(B) < 0.3] = -1
        new[-1] = -1
        hole = (new == -1)[:, None] & (g.random(table.shape) < share) & (table >= 0)
        table[hole] = g.choice([-1, len(stack), 2 ** 31 - 1, -2 ** 31], hole.sum())
        stack = stack[:len(stack) - 50 + room]
        count = min(count, len(stack))
        if room == 0 and len(stack):                     # nearly full: what passes it is dropped
            stack, count = g.permutation(len(stack)).astype(I32), len(stack) - 1
        got = _run_plan(ctx, new, stack, count, table, rows)
        want = plan_past_holes(ctx, new, stack, count, table, rows)
        for name, a, b in zip(("free_pages", "table", "kv_lens", "q_lens", "slots", "free_left"), got, want):
            assert np.array_equal(a, b), (share, name)


def test_a_request_after_one_with_a_hole_gets_pages():
    """A request of two pages, of which one is none, is released; the next one takes the other and a free
    one, is stored, and attends to what is its own."""
    g = np.random.default_rng(70)
    d, rows = 128, 128
    x = Contents(g, [64, 0], 1, d, 0, max_pages=2, n_pages=8)
    page = int(x.table[0, 0])
    free = (page + 3) % 8
    ctx, new = np.array([128, 0], I32), np.array([-1, 128], I32)
    stack = np.full(8, -1, I32)
    stack[0] = free
    c = ugbs.Cache.make(2, 4, 1, d, 8, 2, rows=rows)
    cache, scales, table = x.device()
    kv, q, left = (torch.full((n,), -9, dtype=torch.int32, device="cuda") for n in (2, 2, 1))
    slots = torch.full((2, rows), -9, dtype=torch.int32, device="cuda")
    ugbs.ugbs_cache_plan(c, dev(ctx), dev(new), dev(stack), dev(np.array([1], I32)), table, kv, q, slots, left)
    assert host(table).tolist() == [[page, -1], [page, free]] and int(left.item()) == 0
    assert kv.tolist() == [0, 128] and q.tolist() == [0, 128]
    Kb, K = bf16(g.normal(0, 1, (2, 1, rows, d)))
    Vb, V = bf16(g.normal(0, 1, (2, 1, rows, d)))
    ugbs.ugbs_cache_store(c, dev_bf16(Kb), dev_bf16(Vb), slots, cache, scales)
    x.raw, x.scales = co.store(K, V, host(slots), x.raw, x.scales, 0)
    x.table = host(table)
    Qb, Qv = bf16(g.normal(0, 1, (2, 4, rows, d)))
    O = torch.zeros((2, 4, rows, d), dtype=torch.bfloat16, device="cuda")
    ugbs.ugbs_cache_attend(c, dev_bf16(Qb), cache, scales, table, kv, q, O,
                           torch.empty(max(256, ugbs.ugbs_cache_workspace_bytes(c)), dtype=torch.uint8, device="cuda"))
    got = bf16_to_f64(host_bits(O))
    want, tol = reference(x, 1, Qv[1], 128, 128, 1 / math.sqrt(d), True)
    assert (np.abs(got[1] - want) <= tol).all() and not got[0].any()


def test_a_common_prefix_is_given_back_once():
    """Request 1 lists the prompt's first page of request 0, and is released without it: request 0 goes on,
    request 2 takes what came back, and at the end every page is free once."""
    g = np.random.default_rng(80)
    B, H, Hkv, d, n_pages, max_pages = 3, 4, 2, 64, 9, 4
    c0 = ugbs.Cache.make(B, H, Hkv, d, n_pages, max_pages, rows=150)
    cbufs, step, mir = ugbs.CacheBuffers(c0), ugbs.CacheStep(c0), Mirror(c0)
    cbufs.cache.zero_()
    cbufs.scales.zero_()

    def one(rows, new):
        c = ugbs.Cache.make(B, H, Hkv, d, n_pages, max_pages, rows=rows)
        new = np.array(new, I32)
        (Qb, Qv), (Kb, K), (Vb, V) = (bf16(g.normal(0, 1, (B, h, rows, d))) for h in (H, Hkv, Hkv))
        O = torch.zeros((B, H, rows, d), dtype=torch.bfloat16, device="cuda")
        step.plan(c, dev(new))
        ugbs.cache_layer(c, dev_bf16(Qb), dev_bf16(Kb), dev_bf16(Vb), O, cbufs, step)
        mir.stack, mir.table, mir.kv, mir.q, slots, mir.count = plan_past_holes(mir.kv, new, mir.stack, mir.count, mir.table, rows)
        mir.raw, mir.scales = store_past_holes(K, V, slots, mir.raw, mir.scales, mir.dtype)
        assert np.array_equal(host(step.table), mir.table) and np.array_equal(host(step.kv_lens), mir.kv)
        assert int(step.free_left.item()) == mir.count and np.array_equal(host(step.free_pages), mir.stack)
        _check_step(mir, O, Qv, 1 / math.sqrt(d))

    one(128, [128, 0, 0])
    step.table[1, 0] = step.table[0, 0]
    step.kv_lens[1] = 64
    mir.table[1, 0], mir.kv[1] = mir.table[0, 0], 64
    one(90, [70, 90, 0])
    one(1, [1, 1, 0])
    step.table[1, 0] = -1
    mir.table[1, 0] = -1
    one(150, [5, -1, 150])
    one(1, [1, 0, 1])
    one(1, [-1, 0, -1])
    assert int(step.free_left.item()) == n_pages and sorted(step.free_pages.tolist()) == list(range(n_pages))
