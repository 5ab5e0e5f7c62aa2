"""The page pool where something goes wrong, or lies on another GPU than the current one: nothing it keeps changes, and copies go to its own."""
import contextlib

import pytest
import torch

import paper_2402_15319_amd as vq
from paper_2402_15319_amd import cache as vc


def _state(c):
    return ({s: (c.pages(s), c.length(s)) for s in c._pages}, c.free_pages, sorted(c._free), list(c._holders))


def _pool(pages=20, device="cpu"):
    return vc.PagedCache(2, 2, 1, 64, 16, pages, 6, device=device)


def test_a_fork_of_nothing_leaves_nothing():
    c = _pool()
    a = c.add()
    with pytest.raises(KeyError):
        c.fork(a + 7)
    assert list(c._pages) == list(c._length) == [a]
    assert c.fork(a) == a + 1


def test_a_copy_that_fails_changes_nothing(monkeypatch):
    def broken(*a, **k):
        raise vq.VQError(-5, "vq_cache_copy")
    c = _pool()
    a, other = c.add(), c.add()
    c.grow([other, a], [40, 20])
    c.fork(a)
    d = c.add()
    c.grow([d], [5])
    c.free(other)          # holes for a compaction
    before = _state(c)
    monkeypatch.setattr(vc, "vq_cache_copy", broken)
    with pytest.raises(vq.VQError):
        c.grow([d, a], [40, 30])
    assert _state(c) == before
    with pytest.raises(vq.VQError):
        c.compact()
    assert _state(c) == before
    monkeypatch.setattr(vc, "vq_cache_copy", lambda *a, **k: None)
    assert c.compact() > 0
    c.grow([d, a], [40, 30])
    assert c.length(a) == 50 and _state(c) != before


def test_copies_are_enqueued_on_the_pool_s_gpu(monkeypatch):
    current, at = [0], []

    @contextlib.contextmanager
    def device(d):
        before, current[0] = current[0], torch.device(d).index
        yield
        current[0] = before
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(vc, "vq_cache_copy", lambda *a, **k: at.append(current[0]))
    c = _pool()
    c.device = torch.device("cuda:1")     # the buffers stay on the host: nothing is copied here
    a = c.add()
    c.grow([a], [20])
    b = c.fork(a)
    c.grow([b], [1])
    assert at == [1] and current == [0]
    c.free(a)
    c.compact()
    assert set(at) == {1} and current == [0]


def test_a_workspace_lies_where_the_batch_does():
    desc = vq.make_attn_desc(8, 2, 128, 16, 5)
    batch = vq.AttnBatch(torch.ones(1, dtype=torch.int32), torch.zeros(1, 2, dtype=torch.int32), max_len=32)
    assert vq.attn_workspace(desc, batch).device == torch.device("cpu")
