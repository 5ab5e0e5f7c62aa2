"""Prompts whose parts are longer than the 64 page numbers that a wave holds: it asks for the next ones on the way.  Many sequences with few new
tokens, whose tables name the same pages in different orders, so that a wrong page changes the result."""
import copy

import numpy as np
import pytest

from attn_cases import Problem, run

pytestmark = pytest.mark.gpu


class Shared(Problem):
    """Sequences of the same length on one pool of pages, each in an order of its own."""

    def __init__(self, heads, kv, dim, page, dtype, n_seqs, length, new, seed):
        import torch
        super().__init__(heads, kv, dim, page, dtype, [length], [new], seed=seed)
        rng = np.random.default_rng(seed + 1)
        width, rest = self.width - 1, length % page
        first = self.table[0, :width].copy()
        rows = []
        for _ in range(n_seqs):     # the last page stays the last: the others are full
            some = rng.permutation(first[:width - 1] if rest else first)
            rows.append(np.concatenate([some, first[width - 1:] if rest else some[:0], [-1]]))
        self.table = np.array(rows, dtype=np.int32)
        self.lens, self.new = [length] * n_seqs, [new] * n_seqs
        self.q_start = np.arange(n_seqs + 1, dtype=np.int32) * new
        self.total = n_seqs * new
        self.q_host = torch.from_numpy((rng.standard_normal((self.total, heads, dim)) * 1.5).astype(np.float32)).to(self.q_host.dtype)
        self.q = self.rows(self.q_host, heads)
        i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(self.dev)  # noqa: E731
        self.lens_d, self.table_d, self.start_d = i32(self.lens), i32(self.table), i32(self.q_start)


# The plans (a host check of the same sizes is in tests/test_attn_long_plans.py): whole, and in parts; with one team of waves and with two.
# (heads, kv, dim, page, sequences, length, new tokens of each)
LONG = [(2, 2, 64, 16, 260, 5000, 2), (2, 2, 64, 128, 260, 8300, 2), (2, 2, 128, 128, 260, 4500, 1), (1, 1, 256, 16, 500, 4400, 2),
        (8, 8, 128, 16, 20, 10000, 2), (8, 8, 128, 128, 20, 17000, 1), (8, 8, 96, 32, 20, 12001, 3), (8, 2, 64, 64, 70, 9000, 2)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("heads, kv, dim, page, n_seqs, length, new", LONG)
def test_page_numbers_are_asked_for_on_the_way(heads, kv, dim, page, n_seqs, length, new, dtype):
    import torch
    p = Shared(heads, kv, dim, page, dtype, n_seqs, length, new, seed=length)
    out, lse = run(p)
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())
    some = np.unique([0, n_seqs // 3, n_seqs - 2, n_seqs - 1])      # the oracle takes a sequence's tokens one by one
    rows = np.concatenate([np.arange(s * new, (s + 1) * new) for s in some])
    few = copy.copy(p)
    few.table, few.lens, few.new, few.total = p.table[some], [length] * len(some), [new] * len(some), len(some) * new
    few.q_start, few.q_host = np.arange(len(some) + 1, dtype=np.int32) * new, p.q_host[rows]
    few.check(out[rows], lse[rows])
