"""Alignment that the attention calls ask for, by the order of the rows (no GPU needed: every call here is refused)."""
import pytest

import paper_2402_15319_amd as vq
from test_attn_abi import A, ALIGN, ARG, S, _attn, _batch, _desc

WHOLE = [None, S(1024, 128, 1), S(128, 512, 1)]                 # read in whole vectors
SINGLE = [S(1, 128 * 8, 8), S(1027, 128, 1), S(3, 12 * 128, 12)]   # an element at a time


@pytest.mark.parametrize("name", ["vq_attn_decode", "vq_attn_prompt"])
def test_rows(name):
    d, b = _desc(), _batch()
    for s in WHOLE:
        for off in (2, 8):
            assert _attn(name, d, b, q=A + off, qs=s) == ALIGN and _attn(name, d, b, out=4 * A + off, os=s) == ALIGN
    for s in SINGLE:
        assert _attn(name, d, b, q=A + 1, qs=s) == ALIGN and _attn(name, d, b, out=4 * A + 1, os=s) == ALIGN
        assert _attn(name, d, b, q=A + 2, qs=s, n=0) == ARG and _attn(name, d, b, out=4 * A + 2, os=s, n=0) == ARG     # the workspace is looked at after them


def test_append():
    L, d, b = vq.lib(), _desc(), _batch()
    for s in WHOLE[:2]:
        assert L.vq_cache_append(d, b, A + 8, s, 2 * A, None, 3 * A, 4 * A, 0) == ALIGN and L.vq_cache_append(d, b, A, None, 2 * A + 8, s, 3 * A, 4 * A, 0) == ALIGN
    for s in SINGLE:
        assert L.vq_cache_append(d, b, A + 1, s, 2 * A, None, 3 * A, 4 * A, 0) == ALIGN and L.vq_cache_append(d, b, A, None, 2 * A + 1, s, 3 * A, 4 * A, 0) == ALIGN
        assert L.vq_cache_append(d, b, A + 2, s, 2 * A, None, A + 2, 4 * A, 0) == ALIGN     # the pages'
