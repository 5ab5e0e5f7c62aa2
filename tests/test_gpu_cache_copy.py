"""Copies of more independent pairs than the 1,024 of a launch, and of both many pairs and many buffers: several launches, bit for bit."""
import numpy as np
import pytest

import oracle.attn_oracle as ao

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_buffers, n_pairs", [(1, 1025), (2, 2500), (130, 1100), (1, 64), (1, 65), (3, 1024)])
def test_pairs_over_several_launches(n_buffers, n_pairs):
    import torch
    import paper_2402_15319_amd as vq
    pages = 2 * n_pairs + 3
    order = np.random.default_rng(n_pairs).permutation(pages)
    pairs = [(int(a), int(b)) for a, b in zip(order[:n_pairs], order[n_pairs:2 * n_pairs])]
    gen = torch.Generator(device="cuda:0").manual_seed(1)
    caches = torch.randint(-32768, 32767, (n_buffers, pages, 64 * 16), generator=gen, device="cuda:0", dtype=torch.int16)
    want = ao.copy_pages(caches.cpu().numpy(), pairs)
    vq.vq_cache_copy(vq.make_attn_desc(1, 1, 64, 16, pages), list(caches.unbind(0)), pairs)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(caches.cpu().numpy(), want)
