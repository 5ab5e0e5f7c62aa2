"""What vq_cache_copy makes of its lists (the library is a stand-in; no GPU needed)."""
import ctypes

import pytest
import torch

import paper_2402_15319_amd as vq


@pytest.mark.parametrize("of", [list, tuple, iter, lambda x: (b for b in x)])
@pytest.mark.parametrize("addresses", [False, True])
def test_every_buffer_is_passed_whatever_lists_them(monkeypatch, of, addresses):
    buffers = [torch.zeros(2, 16, dtype=torch.float16) for _ in range(3)]
    want = [b.data_ptr() for b in buffers]
    seen = []

    class Lib:
        def vq_cache_copy(self, desc, n, at, n_pairs, pairs, stream):
            seen.append((list((ctypes.c_uint64 * n).from_address(at)), list((ctypes.c_int32 * (2 * n_pairs)).from_address(pairs))))
            return 0
    monkeypatch.setattr(vq, "lib", Lib)
    vq.vq_cache_copy(vq.make_attn_desc(1, 1, 64, 16, 2), of(want if addresses else buffers), iter([(0, 1), (1, 0)]), stream=0)
    assert seen == [(want, [0, 1, 1, 0])]
