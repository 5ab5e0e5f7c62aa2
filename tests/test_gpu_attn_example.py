"""The example of an attention block on quantised weights: products, cache and attention together, with a fork and compaction,
against the same block in 64 bits on the dense weights."""
import os
import sys

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu


def test_block_against_dense_weights():
    import torch
    import paper_2402_15319_amd as vq
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import attention_block as ab
    finally:
        sys.path.pop(0)
    H, KV, D, steps = 8, 4, 64, 20
    block = ab.AttentionBlock(H, KV, D, seed=3)
    gen = torch.Generator(device="cuda:0").manual_seed(5)
    prompts = [torch.randn(H * D, n, device="cuda:0", generator=gen).half() for n in (37, 150)]
    inputs = []
    call = block.__class__.__call__

    def recorded(self, x, *args, **kw):
        inputs.append(x.double().cpu().numpy())
        return call(self, x, *args, **kw)
    block.__class__.__call__ = recorded
    try:
        outputs, cache = ab.generate(block, prompts, steps, 3)
    finally:
        block.__class__.__call__ = call
    torch.cuda.synchronize()
    dense = {}
    for name, (desc, idx, cb) in block.matrices.items():
        w = torch.empty(desc.out_features, desc.in_features, dtype=torch.float16, device="cuda:0")
        vq.vq_decode_dense(desc, idx, cb, w)
        dense[name] = w.double().cpu().numpy()
    # sequence i's inputs: its prompt, then its column of every step
    first = np.split(inputs[0], [37], axis=1)
    seqs = [np.concatenate([first[p]] + [x[:, i:i + 1] for x in inputs[1:]], axis=1) for i, p in enumerate((0, 1, 0, 0))]
    assert [y.shape[1] for y in outputs] == [57, 170, 57, 57]
    for x, y in zip(seqs, outputs):
        n = x.shape[1]
        q, k, v = ((dense[m] @ x).reshape(-1, D, n) for m in "qkv")
        out = np.zeros((H, D, n))
        for h in range(H):
            t = q[h].T @ k[h // (H // KV)] / np.sqrt(D)
            t[np.triu_indices(n, 1)] = -np.inf
            p = np.exp(t - t.max(1, keepdims=True))
            out[h] = v[h // (H // KV)] @ (p / p.sum(1, keepdims=True)).T
        want = x + dense["o"] @ out.reshape(-1, n)
        # q, k, v, out, the weights and the result are each rounded to fp16 once (2^-11), logits of some units magnify those of q and k
        assert np.linalg.norm(y.double().cpu().numpy() - want) <= 2e-3 * np.linalg.norm(want)
    assert cache.n_pages - cache.free_pages == len({p for s in cache._pages for p in cache.pages(s)}) == max(p for s in cache._pages for p in cache.pages(s)) + 1
