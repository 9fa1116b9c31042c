"""The host's side of steps over the cache, without a GPU: forks, requests that leave pages, steps that are refused."""
import numpy as np
import pytest
import torch

import paper_2607_07724_amd as ugbs

B = 6


def made(kv, width=5):
    """A step whose requests have these lengths; request b lists pages 10 b, 10 b + 1, .. to the end of its row (as after a
    release: entries behind a request's tokens are left over)."""
    step = ugbs.CacheStep(ugbs.Cache.make(B, 4, 1, 64, 100, width), device="cpu", shared=True)
    step.table[:] = 10 * torch.arange(B)[:, None] + torch.arange(width)
    step.kv_lens[:] = torch.tensor(kv)
    return step


def row(b, n):
    return [10 * b + j for j in range(n)]


def test_forks_begin_with_the_pages_that_they_ask_for():
    step = made([200, 0, 0, 70, 0, 0])
    step.fork(0, [1, 4], 128)
    assert step.kv_lens.tolist() == [200, 128, 0, 70, 128, 0]
    assert step.table[1].tolist() == row(0, 2) + [12, 13, 14] and step.table[4, :2].tolist() == row(0, 2)
    assert step.table[0].tolist() == row(0, 5) and step.table[2].tolist() == row(2, 5)


@pytest.mark.parametrize("have,asked,full", [(200, 256, 3), (200, 320, 3), (63, 64, 0), (0, 128, 0), (128, 128, 2), (192, 0, 0)])
def test_a_fork_takes_no_more_than_the_full_pages_of_its_source(have, asked, full):
    step = made([have, 0, 0, 9, 9, 9])
    step.fork(0, [1, 2], asked)
    assert step.kv_lens.tolist() == [have, 64 * full, 64 * full, 9, 9, 9]
    for b in (1, 2):
        # (what lies behind may be another request's page by now)
        assert step.table[b, :asked // 64].tolist() == row(0, full) + [-1] * (asked // 64 - full)


def test_pages_that_the_source_no_longer_lists_are_not_forked():
    step = made([300, 0, 0, 0, 0, 0])
    for none in (-1, 100):
        step.table[0, 2] = none
        step.kv_lens[1] = 0
        step.fork(0, [1], 256)
        assert step.kv_lens.tolist() == [300, 128, 0, 0, 0, 0] and step.table[1, :4].tolist() == row(0, 2) + [-1, -1]


def test_requests_with_tokens_of_their_own_are_not_forked():
    step = made([200, 64, 0, 5, 0, 0])
    step.fork(0, [0, 1, 2, 3], 192)                       # the source among them
    assert step.kv_lens.tolist() == [200, 64, 192, 5, 0, 0]
    assert [step.table[b].tolist() for b in (0, 1, 3)] == [row(b, 5) for b in (0, 1, 3)]


@pytest.mark.parametrize("requests", [2, [2], (2,), (2, 2), range(2, 3), np.array([2]), [2, 2], [-4], torch.tensor([2, 2]), torch.arange(B) == 2, slice(2, 3)])
def test_requests_are_named_as_torch_takes_them(requests):
    step = made([200, 0, 0, 0, 0, 0])
    step.fork(0, requests, 64)
    assert step.kv_lens.tolist() == [200, 0, 64, 0, 0, 0]


def test_requests_that_are_none_are_refused():
    step = made([200, 0, 0, 0, 0, 0])
    for bad in ([6], [1, -7], torch.tensor([99])):
        with pytest.raises(IndexError):
            step.fork(0, bad, 64)
    for source in (6, -7):
        with pytest.raises(IndexError):
            step.fork(source, [1], 64)
    assert step.kv_lens.tolist() == [200, 0, 0, 0, 0, 0]


@pytest.mark.parametrize("tokens", [1, 63, 65, 200, -1, -64, -200, 64 * 6])
def test_requests_leave_whole_pages_of_their_rows(tokens):
    """A page that is left in part is the request's own: it would never come back to the free ones."""
    step = made([200, 200, 0, 0, 0, 0])
    before = step.table.clone()
    with pytest.raises(ValueError, match="whole pages"):
        step.leave([1], tokens)
    assert torch.equal(step.table, before)


@pytest.mark.parametrize("requests", [[1, 3], [3, 1, 3], torch.tensor([1, -3]), slice(1, 4, 2)])
def test_requests_leave_what_they_have_in_common(requests):
    step = made([200] * B)
    step.leave(requests, 128)
    for b in range(B):
        assert step.table[b].tolist() == ([-1, -1] + row(b, 5)[2:] if b in (1, 3) else row(b, 5))
    step.leave(requests, 0)
    step.leave(requests, 64 * 5)
    assert (step.table[[1, 3]] == -1).all() and step.table[0].tolist() == row(0, 5)


def test_leaving_requests_that_are_none_is_refused():
    step = made([200] * B)
    for bad in ([6], [1, -7]):
        with pytest.raises(IndexError):
            step.leave(bad, 64)
    assert (step.table >= 0).all()


def planned_calls(monkeypatch):
    calls = []
    monkeypatch.setattr(ugbs, "ugbs_cache_plan", lambda *a, **k: calls.append("plan"))
    monkeypatch.setattr(ugbs, "ugbs_cache_share", lambda *a, **k: calls.append("share"))
    return calls


@pytest.mark.parametrize("group,why", [
    (torch.zeros(B, dtype=torch.int64), "dtype"), (torch.zeros(B + 1, dtype=torch.int32), "shape"),
    (torch.zeros((B, 1), dtype=torch.int32), "shape"), (torch.zeros(B, dtype=torch.int32), "device tensor")])
def test_a_step_whose_groups_are_refused_is_not_planned(group, why, monkeypatch):
    """The tokens of a step that was planned and then refused would be counted again by the next one."""
    step, calls = made([200, 0, 64, 0, 0, 0]), planned_calls(monkeypatch)
    step._before.fill_(7)
    with pytest.raises(ValueError, match=why):
        step.plan(ugbs.Cache.make(B, 4, 1, 64, 100, 5), torch.ones(B, dtype=torch.int32), group=group)
    assert calls == [] and not step.grouped and (step._before == 7).all()


@pytest.mark.parametrize("H,d", [(16, 64), (4, 256)])
def test_a_step_whose_layout_does_not_fit_is_not_planned(H, d, monkeypatch):
    """Of more query heads than the step was made for (its layout is longer), or of more channels (its workspace is)."""
    step, calls = made([200, 0, 64, 0, 0, 0]), planned_calls(monkeypatch)
    monkeypatch.setattr(ugbs, "_check", lambda name, t, *a: t.data_ptr())          # (no device here)
    with pytest.raises(ValueError, match="made for"):
        step.plan(ugbs.Cache.make(B, H, 1, d, 100, 5), torch.ones(B, dtype=torch.int32), group=torch.zeros(B, dtype=torch.int32))
    assert calls == []
    step.plan(ugbs.Cache.make(B, 4, 1, 64, 100, 5), torch.ones(B, dtype=torch.int32), group=torch.zeros(B, dtype=torch.int32))
    assert calls == ["plan", "share"] and step.grouped
