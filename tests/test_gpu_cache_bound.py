"""New tokens of sequences whose length is more than the call's bound: positions from the bound on have no place and are left out, the
others lie where they belong, and every token that was there before stays."""
import numpy as np
import pytest

from attn_cases import Problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layout", ["tokens", "features", "odd"])
@pytest.mark.parametrize("dim, page", [(64, 16), (96, 32), (128, 128)])
@pytest.mark.parametrize("new, lens, max_len", [
    ([1, 1, 1, 1], [64, 33, 2 ** 31 - 1, 70], 64),               # one each: the last place, inside, far beyond, beyond
    ([1, 1, 1], [65, 129, -7], 128),
    ([2, 2, 2], [65, 66, 30], 64),                               # few each: one of two has a place, none has
    ([150, 300, 40, 200, 9], [400, 260, 100, 2 ** 31 - 1, 263], 256),   # blocks of eight by eight, cut inside a block and at its end
    ([600, 20], [500, 259], 250),                                # some before the first position, too
])
def test_positions_from_the_bound_on_are_left_out(new, lens, max_len, dim, page, layout):
    import torch
    import paper_2402_15319_amd as vq
    own = [max(0, min(n, max_len)) for n in lens]
    p = Problem(16, 16, dim, page, "f16", own, new, layout=layout, seed=sum(new) + dim)
    gen = torch.Generator().manual_seed(7)
    k_host, v_host = (torch.randint(-32768, 32768, (p.total, 16, dim), generator=gen, dtype=torch.int32).to(torch.int16) for _ in range(2))
    k, v = (p.rows(t.view(torch.float16), 16) for t in (k_host, v_host))
    k_host, v_host = k_host.numpy(), v_host.numpy()
    kp, vp = p.k_pages.clone(), p.v_pages.clone()
    bits = lambda t: t.contiguous().view(torch.int16).cpu().numpy()  # noqa: E731
    want_k, want_v = bits(kp).copy(), bits(vp).copy()
    for s, n in enumerate(lens):
        for i in range(new[s]):
            pos = max(n, 0) - new[s] + i
            if 0 <= pos < max_len:
                at, t = (int(p.table[s, pos // page]), pos % page), int(p.q_start[s]) + i
                want_k[at[0], :, at[1], :] = k_host[t]
                want_v[at[0], :, :, at[1]] = v_host[t]
    p.lens_d.copy_(torch.tensor(lens, dtype=torch.int32))
    vq.vq_cache_append(p.desc, p.batch(max_len=max_len, decode=all(n == 1 for n in new)), k, v, kp, vp)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(bits(kp), want_k)
    np.testing.assert_array_equal(bits(vp), want_v)
