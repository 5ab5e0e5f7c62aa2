"""The page pool's bookkeeping without a GPU: its copies are carried out on host tensors, and every sequence is checked to hold
exactly the tokens that were written into it."""
import random

import pytest
import torch

import paper_2402_15319_amd as vq
from paper_2402_15319_amd import cache as vc


def _copy(desc, buffers, pairs, stream=None):
    to, of = [b for _, b in pairs], [a for a, _ in pairs]
    assert len(set(to)) == len(to) and not set(to) & set(of)      # pairs that may share a launch
    assert all(0 <= p < desc.n_pages for p in to + of)
    for b in buffers:
        for x, y in pairs:
            b[y] = b[x].clone()


@pytest.fixture
def pool(monkeypatch):
    monkeypatch.setattr(vc, "vq_cache_copy", _copy)
    return lambda pages=20, width=6, page=16: vc.PagedCache(2, 2, 1, 64, page, pages, width, device="cpu")


class Model:
    """Writes a number for every token where the pool says that it lies, and knows what every sequence should read."""

    def __init__(self, c):
        self.c, self.want, self.count = c, {}, 0

    def write(self, s, n):
        c = self.c
        for pos in range(c.length(s) - n, c.length(s)):
            self.count = (self.count + 1) % 2000
            page, slot = c.pages(s)[pos // c.page_size], pos % c.page_size
            for layer in range(2):
                c.k[layer][page, :, slot], c.v[layer][page, :, :, slot] = self.count + layer * 0.5, -self.count
            self.want.setdefault(s, []).append(self.count)

    def check(self):
        c = self.c
        held = {}
        for s, want in self.want.items():
            assert c.length(s) == len(want) and len(c.pages(s)) == -(-len(want) // c.page_size)
            for pos, x in enumerate(want):
                page, slot = c.pages(s)[pos // c.page_size], pos % c.page_size
                assert float(c.k[0][page, 0, slot, 5]) == x and float(c.k[1][page, 0, slot, 9]) == x + 0.5
                assert float(c.v[1][page, 0, 3, slot]) == -x
            for p in c.pages(s):
                held[p] = held.get(p, 0) + 1
        assert c.free_pages == c.n_pages - len(held)
        assert [c._holders[p] for p in range(c.n_pages)] == [held.get(p, 0) for p in range(c.n_pages)]
        assert sorted(c._free) == [p for p in range(c.n_pages) if p not in held]


def test_a_fork_shares_pages_and_copies_the_last_one_when_it_is_written(pool):
    c = pool()
    m = Model(c)
    a = c.add()
    m.want[a] = []
    c.grow([a], [20])
    m.write(a, 20)
    b = c.fork(a)
    m.want[b] = list(m.want[a])
    assert c.pages(a) == c.pages(b) and c.free_pages == 18
    m.check()
    c.grow([a, b], [1, 1])                       # one of the two keeps the page, the other gets a copy
    m.write(a, 1)
    m.write(b, 1)
    assert c.pages(a)[0] == c.pages(b)[0] and c.pages(a)[1] != c.pages(b)[1] and c.free_pages == 17
    m.check()
    d = c.fork(b)
    m.want[d] = list(m.want[b])
    c.grow([d], [11])                            # the last page is full after this
    m.write(d, 11)
    e = c.fork(d)
    m.want[e] = list(m.want[d])
    c.grow([e], [1])                             # a full page stays shared
    m.write(e, 1)
    assert c.pages(e)[:2] == c.pages(d)
    m.check()
    for s in (a, b, d, e):
        c.free(s)
    assert c.free_pages == 20


def test_compaction_moves_pages_into_holes(pool):
    c = pool()
    m = Model(c)
    seqs = [c.add() for _ in range(4)]
    for s in seqs:
        m.want[s] = []
        c.grow([s], [40])
        m.write(s, 40)
    shared = c.fork(seqs[3])
    m.want[shared] = list(m.want[seqs[3]])
    for s in (seqs[0], seqs[2]):
        c.free(s)
        del m.want[s]
    assert c.compact() > 0
    assert max(p for s in m.want for p in c.pages(s)) == 5 and c.pages(shared) == c.pages(seqs[3])
    m.check()
    assert c.compact() == 0


def test_refusals_change_nothing(pool):
    c = pool(pages=4, width=4)
    a = c.add()
    c.grow([a], [40])
    before = c.pages(a), c.free_pages
    b = c.fork(a)
    with pytest.raises(vc.OutOfPages):
        c.grow([a, b], [8, 9])                   # a copy and a page more: two wanted, one free
    with pytest.raises(ValueError):
        c.grow([a], [25])                        # more than the table lists
    for bad in (([a], [1, 2]), ([a, a], [1, 1]), ([a], [-1])):
        with pytest.raises(ValueError):
            c.grow(*bad)
    assert (c.pages(a), c.free_pages) == before and c.length(a) == c.length(b) == 40
    with pytest.raises(KeyError):
        c.free(99)
    for bad in (dict(layers=0), dict(n_pages=0), dict(table_width=0), dict(dtype=vq.VQ_F32)):
        with pytest.raises(ValueError):
            vc.PagedCache(**{**dict(layers=1, heads=1, kv_heads=1, head_dim=64, page_size=16, n_pages=1, table_width=1, device="cpu"), **bad})


def test_batches(pool):
    c = pool()
    a, b = c.add(), c.add()
    c.grow([a, b], [33, 5])
    batch = c.batch([b, a], [5, 3])
    lens, table, start = batch._keep
    assert lens.tolist() == [5, 33] and start.tolist() == [0, 5, 8] and table.tolist() == [c.pages(b) + [-1, -1], c.pages(a)]
    assert (batch.struct.n_tokens, batch.struct.max_len, batch.struct.table_width) == (8, 33, 3)
    one = c.batch([a])
    assert one.struct.q_start is None and one.struct.n_tokens == 1


@pytest.mark.parametrize("seed", range(6))
def test_any_order_of_growing_forking_freeing_and_compacting(pool, seed):
    rng = random.Random(seed)
    c = pool(pages=14, width=5)
    m = Model(c)
    for _ in range(250):
        live = list(m.want)
        what = rng.random()
        if not live or what < 0.15:
            s = c.add()
            m.want[s] = []
        elif what < 0.65:
            some = rng.sample(live, rng.randint(1, min(3, len(live))))
            new = [rng.randint(0, 20) for _ in some]
            state = {s: (c.pages(s), c.length(s)) for s in live}
            try:
                c.grow(some, new)
            except (vc.OutOfPages, ValueError):
                assert state == {s: (c.pages(s), c.length(s)) for s in live}
                continue
            for s, n in zip(some, new):
                m.write(s, n)
        elif what < 0.8:
            s = rng.choice(live)
            t = c.fork(s)
            m.want[t] = list(m.want[s])
        elif what < 0.93:
            s = rng.choice(live)
            c.free(s)
            del m.want[s]
        else:
            c.compact()
        m.check()
