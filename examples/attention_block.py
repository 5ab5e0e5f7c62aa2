"""The attention block of a decoder layer on vector-quantised weights: prompts, then tokens one at a time, with a fork.

    python examples/attention_block.py [--tokens 512] [--steps 16] [--continuations 3]

The q, k, v and o matrices are packed indices and codebooks; their products run straight into the paged cache and out of it:
vq_gemm_batched writes [features, tokens], whose strides vq_cache_append, vq_attn_prompt and vq_attn_decode take as they are, and
the next product reads what attention wrote.  One user's prompt is forked into several continuations, which share its pages.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2402_15319_amd as vq
from paper_2402_15319_amd.cache import PagedCache
from paper_2402_15319_amd.device import upload_and_pack

DEV = "cuda:0"


class AttentionBlock:
    """x + o(attention(q x, k x, v x)) with random vector-quantised weights (4-bit indices, fp16 codebooks)."""

    def __init__(self, heads: int, kv_heads: int, head_dim: int, seed: int = 0):
        import numpy as np
        rng = np.random.default_rng(seed)
        self.heads, self.kv_heads, self.head_dim, self.width = heads, kv_heads, head_dim, heads * head_dim
        self.matrices = {}
        for name, rows in (("q", self.width), ("k", kv_heads * head_dim), ("v", kv_heads * head_dim), ("o", self.width)):
            desc = vq.make_desc(rows, self.width, 16, 4)
            idx, cb = vq.vq_canonical_bytes(desc)
            values = (rng.standard_normal(cb // 2) * (2.0 if name in "qk" else 1.0) / self.width ** 0.5).astype(np.float16)
            self.matrices[name] = (desc, *upload_and_pack(desc, rng.integers(0, 256, idx, dtype=np.uint8), values, DEV))

    def product(self, name: str, x):
        """[rows, tokens] (token index contiguous, rows padded to 8) of a matrix and x [width, tokens], laid out the same."""
        desc, idx, cb = self.matrices[name]
        ld = x.stride(0)
        y = torch.empty(desc.out_features, ld, dtype=torch.float16, device=DEV)[:, :x.shape[1]]
        vq.vq_gemm_batched(desc, idx, cb, x, x.shape[1], ld, y, ld)
        return y

    def by_heads(self, y, heads: int):
        """The same values as [token][head][dim]."""
        return y.unflatten(0, (heads, self.head_dim)).permute(2, 0, 1)

    def __call__(self, x, cache: PagedCache, layer: int, batch, workspace, prompt: bool):
        q, k, v = self.product("q", x), self.product("k", x), self.product("v", x)
        vq.vq_cache_append(cache.desc, batch, self.by_heads(k, self.kv_heads), self.by_heads(v, self.kv_heads), cache.k[layer], cache.v[layer])
        out = torch.empty(self.width, x.stride(0), dtype=torch.float16, device=DEV)[:, :x.shape[1]]
        call = vq.vq_attn_prompt if prompt else vq.vq_attn_decode
        call(cache.desc, batch, self.by_heads(q, self.heads), cache.k[layer], cache.v[layer], self.by_heads(out, self.heads), workspace)
        return x + self.product("o", out)


def columns(x):
    """[width, tokens] on rows padded to 8 tokens, as the batched product takes it."""
    t = torch.zeros(x.shape[0], (x.shape[1] + 7) // 8 * 8, dtype=torch.float16, device=DEV)
    t[:, :x.shape[1]] = x
    return t[:, :x.shape[1]]


def generate(block: AttentionBlock, prompts, steps: int, continuations: int, page_size: int = 16):
    """prompts: [width, tokens] inputs of each user.  The first user's prompt is continued `continuations` times.  Returns every
    sequence's outputs, [width, its tokens], in the order of the users with the further continuations behind them."""
    longest = max(p.shape[1] for p in prompts) + steps
    per = -(-longest // page_size)
    cache = PagedCache(1, block.heads, block.kv_heads, block.head_dim, page_size, per * (len(prompts) + continuations), per)
    seqs, new = [cache.add() for _ in prompts], [p.shape[1] for p in prompts]
    users = len(prompts) + max(0, continuations - 1)
    ints = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=DEV)  # noqa: E731
    largest = vq.AttnBatch(ints(users), ints(users, per), n_tokens=max(sum(new), users), max_len=longest, q_start=ints(users + 1))
    workspace = vq.attn_workspace(cache.desc, largest, DEV)   # serves every smaller batch
    cache.grow(seqs, new)
    batch = cache.batch(seqs, new)
    y = block(columns(torch.cat(list(prompts), dim=1)), cache, 0, batch, workspace, prompt=True)
    outputs = [[part] for part in y.split(new, dim=1)]
    for _ in range(continuations - 1):
        seqs.append(cache.fork(seqs[0]))
        outputs.append([outputs[0][0]])
    gen = torch.Generator(device=DEV).manual_seed(1)
    for _ in range(steps):
        cache.grow(seqs, [1] * len(seqs))
        batch = cache.batch(seqs)
        # a real decoder goes on from a sampled token's embedding; here each sequence goes its way by some noise
        x = torch.stack([o[-1][:, -1] for o in outputs], dim=1)
        x = 0.5 * x + 0.5 * torch.randn(x.shape, device=DEV, dtype=x.dtype, generator=gen)
        y = block(columns(x), cache, 0, batch, workspace, prompt=False)
        for i, o in enumerate(outputs):
            o.append(y[:, i:i + 1])
    if len(seqs) > 2:       # a user leaves; what remains moves together
        cache.free(seqs[1])
        cache.compact()
    return [torch.cat(o, dim=1) for o in outputs], cache


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=512)
    ap.add_argument("--steps", type=int, default=16)
    ap.add_argument("--continuations", type=int, default=3)
    a = ap.parse_args()
    block = AttentionBlock(32, 32, 128)
    gen = torch.Generator(device=DEV).manual_seed(0)
    prompts = [torch.randn(block.width, n, device=DEV, generator=gen).half() for n in (a.tokens, max(1, a.tokens // 3))]
    outputs, cache = generate(block, prompts, a.steps, a.continuations)
    torch.cuda.synchronize()
    for i, y in enumerate(outputs):
        print(f"sequence {i}: {y.shape[1]} tokens, rms {y.float().square().mean().sqrt():.3f}")
    print(f"{cache.n_pages - cache.free_pages} of {cache.n_pages} pages in use")


if __name__ == "__main__":
    main()
