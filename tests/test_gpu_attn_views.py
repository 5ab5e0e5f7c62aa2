"""Rows that begin anywhere in an array whose order is read and written an element at a time: a prompt's later tokens in what the batched product
wrote, [features, tokens], from a token on that is no multiple of 8."""
import numpy as np
import pytest

import oracle.attn_oracle as ao
from attn_cases import Problem, torch_type

pytestmark = pytest.mark.gpu


def _views(p, host, heads, skip, order):
    """The values as a [T, heads, dim] view `skip` elements behind an aligned address, and the array around it (NaN elsewhere)."""
    import torch
    T, D = host.shape[0], p.dim
    if order == "features":
        whole = torch.full((heads, D, (T + skip + 7) // 8 * 8), float("nan"), dtype=host.dtype, device=p.dev)
        view = whole.permute(2, 0, 1)[skip:skip + T]
    else:                                        # rows of an odd length
        whole = torch.full((skip + T * (heads * D + 3),), float("nan"), dtype=host.dtype, device=p.dev)
        view = whole.as_strided((T, heads, D), (heads * D + 3, D, 1), skip)
    view.copy_(host)
    return view, whole


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("order", ["features", "odd rows"])
@pytest.mark.parametrize("skip", [1, 3, 4, 7])
@pytest.mark.parametrize("lens, new", [([70, 3, 200, 33], None), ([70, 3, 200, 33], [9, 3, 130, 5]), ([300], [300])])
def test_attention_of_rows_that_begin_anywhere(lens, new, skip, order, dtype):
    import torch
    import paper_2402_15319_amd as vq
    p = Problem(6, 2, 64, 16, dtype, lens, new, seed=skip)
    q, _ = _views(p, p.q_host, 6, skip, order)
    out, whole = _views(p, torch.zeros_like(p.q_host), 6, skip, order)
    assert q.data_ptr() % 16 == 2 * skip and out.data_ptr() % 16 == 2 * skip
    rest = torch.isnan(whole)
    lse = torch.empty(p.total, 6, device=p.dev)
    batch = p.batch(decode=new is None)
    call = vq.vq_attn_decode if new is None else vq.vq_attn_prompt
    call(p.desc, batch, q, p.k_pages, p.v_pages, out, vq.attn_workspace(p.desc, batch), lse=lse)
    torch.cuda.synchronize()
    p.check(out, lse)
    assert bool(torch.isnan(whole[rest]).all())


@pytest.mark.parametrize("order", ["features", "odd rows"])
@pytest.mark.parametrize("skip", [1, 4, 7])
@pytest.mark.parametrize("lens, new", [([70, 3, 200, 33], None), ([170, 3, 200, 133], [99, 3, 130, 125])])
def test_new_tokens_that_begin_anywhere(lens, new, skip, order):
    import torch
    import paper_2402_15319_amd as vq
    p = Problem(8, 4, 64, 16, "f16", lens, new, seed=skip)
    gen = torch.Generator().manual_seed(7)
    hosts = [torch.randint(-32768, 32768, (p.total, 4, 64), generator=gen, dtype=torch.int32).to(torch.int16) for _ in range(2)]
    k, v = (_views(p, t.view(torch_type("f16")), 4, skip, order)[0] for t in hosts)
    kp, vp = p.k_pages.clone(), p.v_pages.clone()
    vq.vq_cache_append(p.desc, p.batch(decode=new is None), k, v, kp, vp)
    torch.cuda.synchronize()
    bits = lambda t: t.contiguous().view(torch.int16).cpu().numpy()  # noqa: E731
    want = ao.append(hosts[0].numpy(), hosts[1].numpy(), bits(p.k_pages), bits(p.v_pages), p.table, p.lens, p.q_start)
    np.testing.assert_array_equal(bits(kp), want[0])
    np.testing.assert_array_equal(bits(vp), want[1])
