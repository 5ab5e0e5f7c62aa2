"""The example of an attention block with its cache in 8 bits, with a window, and with both: append, attention, the pool's forks, copies, pages that
are given back and compaction, together.  Every call is compared with the definition, from the state that it found."""
import os
import sys

import numpy as np
import pytest

import oracle.attn_oracle as ao
from cache8_cases import split8

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits, window, sinks", [(8, None, 0), (16, 50, 3), (8, 40, 0), (8, 20, 17)])
def test_block_with_its_cache_in_8_bits_or_a_window(bits, window, sinks, monkeypatch):
    import torch
    import paper_2402_15319_amd as vq
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import attention_block as ab
    finally:
        sys.path.pop(0)
    H, KV, D, steps = 8, 4, 64, 40
    block = ab.AttentionBlock(H, KV, D, seed=3)
    gen = torch.Generator(device="cuda:0").manual_seed(5)
    prompts = [torch.randn(H * D, n, device="cuda:0", generator=gen).half() for n in (37, 150)]
    dense_o = torch.empty(H * D, H * D, dtype=torch.float16, device="cuda:0")
    vq.vq_decode_dense(*block.matrices["o"], dense_o)
    dense_o = dense_o.double().cpu().numpy()
    call = ab.AttentionBlock.__call__
    calls = []

    def pages(cache):
        if bits == 8:
            return [*split8(cache.desc, cache.k[0], True), *split8(cache.desc, cache.v[0], False)]
        return [cache.k[0].double().cpu().numpy(), cache.v[0].double().cpu().numpy()]

    def checked(self, x, cache, layer, batch, workspace, prompt, **kw):
        rows = lambda name, heads: self.by_heads(self.product(name, x), heads).double().cpu().numpy()  # noqa: E731
        q, k, v = rows("q", H), rows("k", KV), rows("v", KV)       # the same products as the block's own
        lens, table, start = ((t.tolist() if t is not None else None) for t in batch._keep)
        start = list(range(len(lens) + 1)) if start is None else start
        if bits == 8:
            want = ao.append8(k, v, *pages(cache), table, lens, start, "f16")
            kv = ao.values8(want[0], want[1], True), ao.values8(want[2], want[3], False)
        else:
            want = kv = ao.append(k, v, *pages(cache), table, lens, start)
        y = call(self, x, cache, layer, batch, workspace, prompt, **kw)
        torch.cuda.synchronize()
        for s, n in enumerate(lens):                               # this batch's tokens, as they should be
            for j in range(0 if window is None else max(0, n - window), n):
                page, slot = table[s][j // 16], j % 16
                got = pages(cache) if j == (0 if window is None else max(0, n - window)) else got  # noqa: F821
                for a, b, by_slot in ((got[0], want[0], True), (got[bits // 8 == 1 and 2 or 1], want[bits // 8 == 1 and 2 or 1], False)):
                    a, b = (t[page][:, slot] if by_slot else t[page][:, :, slot] for t in (a, b))
                    assert np.array_equal(a, b)
        out = ao.attention(q, *kv, table, lens, start, D ** -0.5, window, sinks)[0]
        ref = x.double().cpu().numpy() + dense_o @ out.reshape(out.shape[0], -1).T
        # q, the weights, out, the o product and the sum are each rounded to fp16 once (2^-11)
        assert np.linalg.norm(y.double().cpu().numpy() - ref) <= 2e-3 * np.linalg.norm(ref)
        calls.append(cache.n_pages - cache.free_pages)
        return y
    monkeypatch.setattr(ab.AttentionBlock, "__call__", checked)
    outputs, cache = ab.generate(block, prompts, steps, 3, bits=bits, window=None if window is None else vq.VQAttnWindow(window, sinks))
    assert [y.shape[1] for y in outputs] == [77, 190, 77, 77] and len(calls) == 1 + steps
    held = {p for s in cache._pages for p in cache.pages(s) if p >= 0}
    assert cache.n_pages - cache.free_pages == len(held) == max(held) + 1
    if window is not None:       # what the windows hold, a page more at each end, and the sinks' pages
        assert len(held) <= len(cache._pages) * (-(-window // 16) + 2 + -(-sinks // 16)) < 12 + 5 + 5 + 5
