"""New tokens into the cache's pages, and copies of pages: bit for bit."""
import numpy as np
import pytest

import oracle.attn_oracle as ao
from attn_cases import Problem, torch_type

pytestmark = pytest.mark.gpu


def _append(p, k, v):
    import torch
    import paper_2402_15319_amd as vq
    kp, vp = p.k_pages.clone(), p.v_pages.clone()
    vq.vq_cache_append(p.desc, p.batch(decode=all(n == 1 for n in p.new)), k, v, kp, vp)
    torch.cuda.synchronize()
    return kp, vp


def _bits(t):
    import torch
    return t.contiguous().view(torch.int16).cpu().numpy()


@pytest.mark.parametrize("layout, gap", [("tokens", 0), ("tokens", 2), ("heads", 1), ("features", 0), ("features", 1), ("odd", 1), ("odd features", 0)])
@pytest.mark.parametrize("heads, kv, dim, page, dtype, lens, new", [
    (4, 4, 128, 16, "f16", [1, 16, 17, 40, 300], None),
    (8, 2, 64, 32, "bf16", [1, 33, 90, 7], [1, 33, 50, 3]),
    (3, 3, 96, 64, "f16", [130, 0, 64, 200, 5], [130, 0, 1, 77, 9]),
    (2, 1, 256, 128, "bf16", [300, 129], [171, 129]),
    (4, 4, 128, 16, "f16", [700, 801], [700, 666]),
    (1, 1, 64, 16, "f16", [9], [1]),
])
def test_new_tokens_into_pages(heads, kv, dim, page, dtype, lens, new, layout, gap):
    import torch
    p = Problem(heads, kv, dim, page, dtype, lens, new, layout=layout, gap=gap, seed=dim)
    gen = torch.Generator().manual_seed(7)
    k_host = torch.randint(-32768, 32768, (p.total, kv, dim), generator=gen, dtype=torch.int32).to(torch.int16)   # every bit pattern
    v_host = torch.randint(-32768, 32768, (p.total, kv, dim), generator=gen, dtype=torch.int32).to(torch.int16)
    k, v = (p.rows(t.view(torch_type(dtype)), kv) for t in (k_host, v_host))
    kp, vp = _append(p, k, v)
    want = ao.append(k_host.numpy(), v_host.numpy(), _bits(p.k_pages), _bits(p.v_pages), p.table, p.lens, p.q_start)
    np.testing.assert_array_equal(_bits(kp), want[0])
    np.testing.assert_array_equal(_bits(vp), want[1])


def test_tokens_without_a_place_are_left_out():
    """Negative positions, pages outside the cache, and lengths beyond what the table lists write nothing."""
    import torch
    p = Problem(2, 2, 64, 16, "f16", [50, 3, 20], [50, 9, 20], seed=1)
    p.table[0, 1] = -1
    p.table[2, 0] = p.n_pages
    p.table_d.copy_(torch.from_numpy(p.table))
    k_host = torch.randn(p.total, 2, 64).half()
    kp, vp = _append(p, k_host.cuda(), k_host.cuda())
    want = ao.append(_bits(k_host), _bits(k_host), _bits(p.k_pages), _bits(p.v_pages), p.table, p.lens, p.q_start)
    np.testing.assert_array_equal(_bits(kp), want[0])
    np.testing.assert_array_equal(_bits(vp), want[1])


def test_append_then_attend():
    """What is appended is what attention reads: a prompt in two pieces, then single tokens."""
    import torch
    import paper_2402_15319_amd as vq
    n, H, kv, D, page = 150, 4, 2, 128, 16
    gen = torch.Generator().manual_seed(3)
    q, k, v = (torch.randn(n, h, D, generator=gen).half() for h in (H, kv, kv))
    pages = (n + page - 1) // page
    desc = vq.make_attn_desc(H, kv, D, page, pages + 1)
    kp = torch.full((pages + 1, kv, page, D), float("nan"), dtype=torch.float16, device="cuda:0")
    vp = torch.full((pages + 1, kv, D, page), float("nan"), dtype=torch.float16, device="cuda:0")
    table = torch.arange(pages, 0, -1, dtype=torch.int32, device="cuda:0")[None]
    out = torch.empty(n, H, D, dtype=torch.float16, device="cuda:0")
    at = 0
    for step in (100, 37, *[1] * (n - 137)):
        lens = torch.tensor([at + step], dtype=torch.int32, device="cuda:0")
        start = torch.tensor([0, step], dtype=torch.int32, device="cuda:0")
        batch = vq.AttnBatch(lens, table, n_tokens=step, max_len=at + step, q_start=None if step == 1 else start)
        ws = vq.attn_workspace(desc, batch)
        vq.vq_cache_append(desc, batch, k[at:at + step].cuda(), v[at:at + step].cuda(), kp, vp)
        call = vq.vq_attn_decode if step == 1 else vq.vq_attn_prompt
        call(desc, batch, q[at:at + step].cuda(), kp, vp, out[at:at + step], ws)
        torch.cuda.synchronize()
        at += step
    ref = ao.attention(q.double().numpy(), kp.cpu().double().numpy(), vp.cpu().double().numpy(), table.cpu().numpy(), [n], [0, n], D ** -0.5)
    u, f32 = 2.0 ** -11, 2.0 ** -24
    rel = u + 2 * (D + 8) * f32 * ref[3] + (n + 16) * f32
    assert (np.abs(out.cpu().double().numpy() - ref[0]) <= 1.01 * (rel[..., None] * ref[2] + u * np.abs(ref[0])) + 2.0 ** -25 * (1 + 8 * n)).all()


@pytest.mark.parametrize("n_buffers, pages, kv, dim, page, pairs", [
    (1, 4, 1, 64, 16, [(0, 3)]),
    (2, 9, 2, 96, 16, [(0, 1), (2, 3), (8, 4)]),
    (7, 30, 3, 128, 32, [(i, 15 + i) for i in range(15)]),
    (130, 6, 1, 64, 16, [(5, 0), (4, 1)]),                                       # more buffers than a launch takes
    (2, 1000, 1, 64, 16, [(i, 500 + i) for i in range(500)]),                    # more pairs than a launch takes
    (2, 12, 1, 128, 16, [(0, 1), (1, 2), (2, 3), (5, 5), (3, 0), (7, 3), (8, 3)]),   # each depends on the one before
    (1, 700, 1, 64, 16, [(i, i + 1) for i in range(699)]),
    (3, 5, 4, 256, 128, [(0, 4), (0, 3), (0, 2)]),                               # one page to several
])
def test_pages_are_copied_one_pair_after_another(n_buffers, pages, kv, dim, page, pairs):
    import torch
    import paper_2402_15319_amd as vq
    gen = torch.Generator(device="cuda:0").manual_seed(1)
    caches = torch.randint(-32768, 32767, (n_buffers, pages, kv * dim * page), generator=gen, device="cuda:0", dtype=torch.int16)
    want = ao.copy_pages(caches.cpu().numpy(), pairs)
    desc = vq.make_attn_desc(kv, kv, dim, page, pages)
    vq.vq_cache_copy(desc, list(caches.unbind(0)), pairs)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(caches.cpu().numpy(), want)


@pytest.mark.parametrize("layout", ["tokens", "features"])
@pytest.mark.parametrize("new", [1, 2, 3, 20])
def test_many_sequences(new, layout):
    """More than a wave looks at in one turn; few new tokens for each and more, some sequences without any."""
    import torch
    rng = np.random.default_rng(new)
    news = [0 if rng.random() < 0.1 else new for _ in range(150)]
    news[0] = new
    lens = [n + int(rng.integers(0, 30)) for n in news]
    p = Problem(8, 8, 64, 16, "f16", lens, news, layout=layout, seed=new)
    gen = torch.Generator().manual_seed(7)
    k_host = torch.randint(-32768, 32768, (p.total, 8, 64), generator=gen, dtype=torch.int32).to(torch.int16)
    k = p.rows(k_host.view(torch.float16), 8)
    kp, vp = _append(p, k, k)
    want = ao.append(k_host.numpy(), k_host.numpy(), _bits(p.k_pages), _bits(p.v_pages), p.table, p.lens, p.q_start)
    np.testing.assert_array_equal(_bits(kp), want[0])
    np.testing.assert_array_equal(_bits(vp), want[1])


def test_more_new_tokens_than_the_cache_counts():
    """The first of them have negative positions and are left out."""
    import torch
    p = Problem(2, 2, 96, 16, "f16", [70, 3, 0], [100, 40, 9], layout="features", seed=1)
    k_host = torch.randn(p.total, 2, 96).half()
    k = p.rows(k_host, 2)
    kp, vp = _append(p, k, k)
    want = ao.append(_bits(k_host), _bits(k_host), _bits(p.k_pages), _bits(p.v_pages), p.table, p.lens, p.q_start)
    np.testing.assert_array_equal(_bits(kp), want[0])
    np.testing.assert_array_equal(_bits(vp), want[1])


def test_offsets_beyond_32_bits():
    """Pages at the end of buffers of more than 2^32 bytes, as a place for tokens and as a copy's source and target."""
    import torch
    import paper_2402_15319_amd as vq
    pages = 2 ** 32 // (2 * 128 * 128 * 2) + 70
    k = torch.zeros(pages, 2, 128, 128, dtype=torch.float16, device="cuda:0")
    v = torch.zeros(pages, 2, 128, 128, dtype=torch.float16, device="cuda:0")
    desc = vq.make_attn_desc(2, 2, 128, 128, pages)
    table = torch.tensor([[pages - 1, pages - 5]], dtype=torch.int32, device="cuda:0")
    lens = torch.tensor([200], dtype=torch.int32, device="cuda:0")
    start = torch.tensor([0, 200], dtype=torch.int32, device="cuda:0")
    batch = vq.AttnBatch(lens, table, n_tokens=200, max_len=200, q_start=start)
    rows = torch.randn(200, 2, 128, device="cuda:0").half()
    vq.vq_cache_append(desc, batch, rows, rows, k, v)
    vq.vq_cache_copy(desc, [k, v], [(pages - 1, 3), (pages - 5, pages - 2)])
    torch.cuda.synchronize()
    for first, second in ((pages - 1, pages - 5), (3, pages - 2)):
        assert torch.equal(torch.cat([k[first].transpose(0, 1), k[second].transpose(0, 1)])[:200], rows)
        assert torch.equal(torch.cat([v[first].permute(2, 0, 1), v[second].permute(2, 0, 1)])[:200], rows)
    assert int(k.count_nonzero()) <= 2 * rows.numel() and not k[4:pages - 10].any()


def test_append_and_copy_in_a_captured_graph_and_on_another_stream():
    """A graph follows the lengths and the table when it is replayed."""
    import torch
    import paper_2402_15319_amd as vq
    p = Problem(4, 4, 64, 16, "f16", [40, 17], [1, 1], seed=3)
    rows = torch.randn(2, 4, 64, device="cuda:0").half()
    kp, vp = p.k_pages.clone(), p.v_pages.clone()
    batch = vq.AttnBatch(p.lens_d, p.table_d, max_len=p.width * 16)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        vq.vq_cache_append(p.desc, batch, rows, rows, kp, vp)
        vq.vq_cache_copy(p.desc, [kp], [(0, 1)])
    for lens in ([40, 17], [33, 2], [38, 16]):
        p.lens_d.copy_(torch.tensor(lens, dtype=torch.int32))
        kp.copy_(p.k_pages)
        vp.copy_(p.v_pages)
        rows.normal_()
        g.replay()
        torch.cuda.synchronize()
        want = ao.append(_bits(rows), _bits(rows), _bits(p.k_pages), _bits(p.v_pages), p.table, lens, p.q_start)
        np.testing.assert_array_equal(_bits(kp), ao.copy_pages(want[0][None], [(0, 1)])[0])
        np.testing.assert_array_equal(_bits(vp), want[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    kp.copy_(p.k_pages)
    side.wait_stream(torch.cuda.current_stream())
    vq.vq_cache_append(p.desc, batch, rows, rows, kp, vp, stream=side)
    vq.vq_cache_copy(p.desc, [kp], [(0, 1)], stream=side)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(_bits(kp), ao.copy_pages(want[0][None], [(0, 1)])[0])
