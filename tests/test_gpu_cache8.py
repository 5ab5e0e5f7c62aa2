"""New tokens into pages in 8 bits, and copies of such pages: codes and scales bit for bit."""
import numpy as np
import pytest

import oracle.attn_oracle as ao
from attn_cases import Problem, torch_type
from cache8_cases import into_8_bits, join8, split8

pytestmark = pytest.mark.gpu


class Pages:
    """A problem's pages in 8 bits before its new tokens come (only earlier ones are live; other slots and blocks hold anything)."""

    def __init__(self, p, seed=0, loud=1.0):
        import paper_2402_15319_amd as vq
        rng = np.random.default_rng(seed + 100)
        live = np.zeros_like(p.live)
        for s in range(len(p.lens)):
            for j in range(max(0, p.lens[s] - p.new[s])):
                page = p.table[s, j // p.page]
                if 0 <= page < p.n_pages:
                    live[page, j % p.page] = True
        tt = torch_type(p.dtype)
        import torch
        rand = lambda *shape: torch.from_numpy(rng.standard_normal(shape) * loud * 2.0 ** rng.integers(-6, 7, shape[:2])[..., None, None]).to(tt).double().numpy()  # noqa: E731
        self.k = into_8_bits(rand(p.n_pages, p.kv, p.page, p.dim), live, p.dtype, rng, True)
        self.v = into_8_bits(rand(p.n_pages, p.kv, p.dim, p.page), live, p.dtype, rng, False)
        self.p = p
        p.desc.cache_dtype = vq.VQ_E4M3

    def buffers(self):
        return join8(*self.k), join8(*self.v)

    def want(self, k_host, v_host, max_len=None):
        p = self.p
        return ao.append8(k_host.double().numpy(), v_host.double().numpy(), *self.k, *self.v, p.table, p.lens, p.q_start, p.dtype, max_len)

    def compare(self, kp, vp, want):
        for got, codes, scales, by_slot in ((kp, want[0], want[1], True), (vp, want[2], want[3], False)):
            c, s = split8(self.p.desc, got, by_slot)
            none = np.isnan(ao.CODE_VALUES[codes])
            assert np.array_equal(np.isnan(ao.CODE_VALUES[c]), none)   # a NaN's sign is anything
            np.testing.assert_array_equal(np.where(none, 127, c), np.where(none, 127, codes))
            np.testing.assert_array_equal(s.view(np.uint32), scales.view(np.uint32))


def _append(p, k, v, kp, vp, one_each=None, max_len=None):
    import torch
    import paper_2402_15319_amd as vq
    one_each = all(n == 1 for n in p.new) if one_each is None else one_each
    vq.vq_cache_append(p.desc, p.batch(max_len, decode=one_each), k, v, kp, vp)
    torch.cuda.synchronize()


def _values(p, seed, scale=1.0):
    import torch
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((p.total, p.kv, p.dim)) * scale * 2.0 ** rng.integers(-8, 9, (p.total, p.kv, 1))
    return torch.from_numpy(x).to(torch_type(p.dtype))


CASES = [
    (4, 4, 128, 16, "f16", [1, 16, 17, 40, 300], None),
    (8, 2, 64, 32, "bf16", [1, 33, 90, 7], [1, 33, 50, 3]),
    (3, 3, 96, 64, "f16", [130, 0, 64, 200, 5], [130, 0, 1, 77, 9]),
    (2, 1, 256, 128, "bf16", [300, 129], [171, 129]),
    (4, 4, 128, 16, "f16", [700, 801], [700, 666]),
    (1, 1, 64, 16, "f16", [9], [1]),
    (5, 5, 96, 16, "bf16", [1, 15, 16, 30, 31, 32, 33], None),
    (40, 40, 256, 32, "f16", [20, 50], None),
]


@pytest.mark.parametrize("layout, gap", [("tokens", 0), ("tokens", 2), ("heads", 1), ("features", 0), ("features", 1), ("odd", 1), ("odd features", 0)])
@pytest.mark.parametrize("heads, kv, dim, page, dtype, lens, new", CASES)
def test_new_tokens_into_pages(heads, kv, dim, page, dtype, lens, new, layout, gap):
    p = Problem(heads, kv, dim, page, dtype, lens, new, layout=layout, gap=gap, seed=dim)
    pages = Pages(p)
    k, v = _values(p, 1), _values(p, 2)
    kp, vp = pages.buffers()
    _append(p, p.rows(k, kv), p.rows(v, kv), kp, vp)
    want = pages.want(k, v)
    pages.compare(kp, vp, want)
    _append(p, p.rows(k, kv), p.rows(v, kv), kp, vp)   # once more: the scales stay, and so do the codes
    pages.compare(kp, vp, want)
    if new is None:                                     # the call for any number of tokens
        kp, vp = pages.buffers()
        _append(p, p.rows(k, kv), p.rows(v, kv), kp, vp, one_each=False)
        pages.compare(kp, vp, want)


@pytest.mark.parametrize("one_each", [True, False])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
def test_every_value_of_the_type(dim, dtype, one_each):
    """All 65,536 bit patterns, NaN, infinities and the largest numbers among them, in blocks of like and of unlike magnitudes."""
    import torch
    kv, n = 8, -(-65536 // (8 * dim))
    new = [1] * n if one_each else [n]
    lens = [17 + i % 40 for i in range(n)] if one_each else [n + 5]
    p = Problem(kv, kv, dim, 16, dtype, lens, new, seed=3)
    pages = Pages(p, loud=0.01)
    every = (torch.arange(n * kv * dim, dtype=torch.int32) % 65536).to(torch.int16).view(torch_type(dtype))
    k = every.view(n, kv, dim)                                             # neighbours: alike
    v = every.view(dim, n, kv).permute(1, 2, 0).contiguous()               # every magnitude in a row
    kp, vp = pages.buffers()
    _append(p, k.cuda(), v.cuda(), kp, vp, one_each=one_each)
    pages.compare(kp, vp, pages.want(k, v))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("value", [0.0, -0.0, 448.0, 449.0, 57344.0, 57376.0, 61440.0, 63488.0, 65504.0, 2.0 ** -24, 2.0 ** -14, float("inf"), float("nan")])
def test_one_value_everywhere(value, dtype):
    """The borders of a scale and of the type; a block of nothing but NaN has the least scale."""
    import torch
    for new in (None, [5, 33]):
        p = Problem(2, 2, 128, 32, dtype, [18, 40], new, seed=4)
        pages = Pages(p, loud=2.0 ** -9)
        k = torch.full((p.total, 2, 128), value).to(torch_type(dtype))
        v = -k
        kp, vp = pages.buffers()
        _append(p, k.cuda(), v.cuda(), kp, vp)
        pages.compare(kp, vp, pages.want(k, v))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_a_block_filled_one_token_at_a_time(dtype):
    """Louder tokens behind quieter ones: the codes of the earlier ones are rounded again where the scale grows, each time from what they are."""
    import torch
    lens = [1, 1, 1]
    p = Problem(2, 2, 96, 16, dtype, [40] * 3, [1] * 3, seed=5)
    pages = Pages(p)
    kp, vp = pages.buffers()
    rng = np.random.default_rng(1)
    for step in range(40):
        p.lens = lens = [step + 1, 39 - step, 17 + step // 2]
        p.lens_d.copy_(torch.tensor(lens, dtype=torch.int32))
        x = rng.standard_normal((2, 3, 2, 96)) * np.array([1.15 ** step, 0.9 ** step, 2.0 ** rng.integers(-9, 9)])[None, :, None, None]
        k, v = (torch.from_numpy(a).to(torch_type(dtype)) for a in x)
        want = pages.want(k, v)
        _append(p, k.cuda(), v.cuda(), kp, vp)
        pages.compare(kp, vp, want)
        pages.k, pages.v = want[:2], want[2:]


def test_codes_are_what_single_tokens_leave_where_no_scale_grows():
    """A prompt whose loudest token comes first in every block, whole and token by token."""
    import torch
    n, kv, dim = 50, 2, 64
    p = Problem(kv, kv, dim, 16, "f16", [n], [n], seed=6)
    pages = Pages(p)
    k, v = _values(p, 3), _values(p, 4)
    for t in (k, v):
        t.clamp_(-100, 100)
        t[::16] = 100.0
    kp, vp = pages.buffers()
    _append(p, k.cuda(), v.cuda(), kp, vp)
    k1, v1 = pages.buffers()
    import paper_2402_15319_amd as vq
    for t in range(n):
        batch = vq.AttnBatch(torch.tensor([t + 1], dtype=torch.int32, device="cuda:0"), p.table_d, max_len=t + 1)
        vq.vq_cache_append(p.desc, batch, k[t:t + 1].cuda(), v[t:t + 1].cuda(), k1, v1)
    torch.cuda.synchronize()
    assert torch.equal(kp, k1) and torch.equal(vp, v1)


@pytest.mark.parametrize("one_each", [True, False])
def test_tokens_without_a_place_are_left_out(one_each):
    """Negative positions, pages outside the cache, positions from max_len on: codes, scales and earlier tokens stay."""
    import torch
    lens = [50, 0, 20, 33, 34] if one_each else [50, 3, 20, 40, 34]
    p = Problem(2, 2, 64, 16, "f16", lens, [1] * 5 if one_each else [50, 9, 20, 7, 2], seed=1)
    p.table[0, 1] = p.table[0, 3] = -1
    p.table[2, 0] = p.table[2, 1] = p.n_pages
    p.table_d.copy_(torch.from_numpy(p.table))
    for max_len in (max(p.lens), 33, 38, 35, 16, 0):
        pages = Pages(p)
        k, v = _values(p, 5, 100.0), _values(p, 6, 100.0)
        kp, vp = pages.buffers()
        _append(p, k.cuda(), v.cuda(), kp, vp, one_each=one_each, max_len=max_len)
        pages.compare(kp, vp, pages.want(k, v, max_len))


@pytest.mark.parametrize("layout", ["tokens", "features"])
@pytest.mark.parametrize("new", [1, 2, 3, 20])
def test_many_sequences(new, layout):
    rng = np.random.default_rng(new)
    news = [0 if rng.random() < 0.1 else new for _ in range(150)]
    news[0] = new
    lens = [n + int(rng.integers(0, 30)) for n in news]
    p = Problem(8, 8, 64, 16, "f16", lens, news, layout=layout, seed=new)
    pages = Pages(p)
    k, v = _values(p, 7), _values(p, 8)
    kp, vp = pages.buffers()
    _append(p, p.rows(k, 8), p.rows(v, 8), kp, vp)
    pages.compare(kp, vp, pages.want(k, v))


@pytest.mark.parametrize("k_layout, v_layout", [("tokens", "features"), ("features", "tokens"), ("features", "odd"), ("odd features", "heads")])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
def test_keys_and_values_in_different_orders(dim, k_layout, v_layout):
    for page, lens, new in ((16, [100, 200, 7], [64, 200, 7]), (64, [300, 65], [177, 64]), (32, [20, 40, 9], [2, 1, 2])):
        p = Problem(3, 3, dim, page, "f16", lens, new, seed=dim)
        pages = Pages(p)
        k, v = _values(p, 11), _values(p, 12)
        kp, vp = pages.buffers()
        p.layout = k_layout
        k_rows = p.rows(k, 3)
        p.layout = v_layout
        _append(p, k_rows, p.rows(v, 3), kp, vp)
        pages.compare(kp, vp, pages.want(k, v))


@pytest.mark.parametrize("layout", ["tokens", "features"])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_one_long_sequence_among_many_without_new_tokens(dtype, layout):
    """Few tokens for each sequence on the average: those of the long one still make their blocks' scales together."""
    new = [0] * 150 + [301] + [1, 0, 3] * 10
    lens = [n + (5 * i) % 40 for i, n in enumerate(new)]
    p = Problem(2, 2, 128, 32, dtype, lens, new, layout=layout, seed=4)
    pages = Pages(p, loud=2.0 ** -4)
    k, v = _values(p, 13), _values(p, 14)
    kp, vp = pages.buffers()
    _append(p, p.rows(k, 2), p.rows(v, 2), kp, vp)
    pages.compare(kp, vp, pages.want(k, v))


@pytest.mark.parametrize("new", [[1, 2, 0], [70, 33, 2]])
@pytest.mark.parametrize("layout", ["tokens", "features"])
def test_rows_behind_the_last_sequence(layout, new):
    """A padded batch: q_start ends before n_tokens, and the rows from there on go nowhere."""
    import torch
    import paper_2402_15319_amd as vq
    p = Problem(2, 2, 128, 16, "f16", [70, 300, 9], new, layout=layout, seed=6)
    pages = Pages(p)
    k, v = _values(p, 15), _values(p, 16)
    want = pages.want(k, v)
    pad = lambda t: torch.cat([t, torch.full((2, *t.shape[1:]), float("nan"), dtype=t.dtype)])  # noqa: E731
    kp, vp = pages.buffers()
    batch = vq.AttnBatch(p.lens_d, p.table_d, n_tokens=p.total + 2, max_len=300, q_start=p.start_d)
    vq.vq_cache_append(p.desc, batch, p.rows(pad(k), 2), p.rows(pad(v), 2), kp, vp)
    torch.cuda.synchronize()
    pages.compare(kp, vp, want)


def test_a_captured_graph_and_another_stream():
    """A graph follows the lengths and the table when it is replayed."""
    import torch
    import paper_2402_15319_amd as vq
    p = Problem(4, 4, 64, 16, "f16", [40, 17], [1, 1], seed=3)
    pages = Pages(p)
    kp, vp = pages.buffers()
    k, v = torch.zeros(2, 4, 64, device="cuda:0").half(), torch.zeros(2, 4, 64, device="cuda:0").half()
    batch = vq.AttnBatch(p.lens_d, p.table_d, max_len=p.width * 16)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        vq.vq_cache_append(p.desc, batch, k, v, kp, vp)
    for lens in ([40, 17], [33, 2], [38, 16]):
        p.lens = lens
        p.lens_d.copy_(torch.tensor(lens, dtype=torch.int32))
        for got, start in ((kp, pages.buffers()[0]), (vp, pages.buffers()[1])):
            got.copy_(start)
        k.normal_()
        v.normal_(std=30.0)
        g.replay()
        torch.cuda.synchronize()
        want = pages.want(k.cpu(), v.cpu())
        pages.compare(kp, vp, want)
    side = torch.cuda.Stream()
    for got, start in ((kp, pages.buffers()[0]), (vp, pages.buffers()[1])):
        got.copy_(start)
    side.wait_stream(torch.cuda.current_stream())
    vq.vq_cache_append(p.desc, batch, k, v, kp, vp, stream=side)
    torch.cuda.synchronize()
    pages.compare(kp, vp, want)


@pytest.mark.parametrize("n_buffers, pages, kv, dim, page, pairs", [
    (1, 4, 1, 64, 16, [(0, 3)]),
    (2, 9, 2, 96, 16, [(0, 1), (2, 3), (8, 4)]),
    (7, 30, 3, 128, 32, [(i, 15 + i) for i in range(15)]),
    (130, 6, 1, 64, 16, [(5, 0), (4, 1)]),
    (2, 1000, 1, 64, 16, [(i, 500 + i) for i in range(500)]),
    (2, 12, 1, 128, 16, [(0, 1), (1, 2), (2, 3), (5, 5), (3, 0), (7, 3), (8, 3)]),
    (3, 5, 40, 256, 128, [(0, 4), (0, 3), (0, 2)]),                              # 320 scales to a page
])
def test_pages_are_copied_with_their_scales(n_buffers, pages, kv, dim, page, pairs):
    import torch
    import paper_2402_15319_amd as vq
    desc = vq.make_attn_desc(kv, kv, dim, page, pages, cache_dtype=vq.VQ_E4M3)
    size, codes = vq.vq_cache_bytes(desc), pages * kv * dim * page
    assert size == codes + codes // dim // 4
    gen = torch.Generator(device="cuda:0").manual_seed(1)
    caches = torch.randint(0, 256, (n_buffers, (size + 79) // 16 * 16), generator=gen, device="cuda:0", dtype=torch.uint8)
    before = caches.cpu().numpy()
    want = before.copy()
    want[:, :codes] = ao.copy_pages(before[:, :codes].reshape(n_buffers, pages, -1), pairs).reshape(n_buffers, -1)
    want[:, codes:size] = ao.copy_pages(before[:, codes:size].reshape(n_buffers, pages, -1), pairs).reshape(n_buffers, -1)
    vq.vq_cache_copy(desc, list(caches.unbind(0)), pairs)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(caches.cpu().numpy(), want)


def test_offsets_beyond_32_bits():
    """Pages and scales at the end of buffers of more than 2^32 bytes, as places for tokens, for attention and for copies."""
    import torch
    import paper_2402_15319_amd as vq
    pages = 2 ** 32 // (2 * 128 * 128) + 70
    desc = vq.make_attn_desc(2, 2, 128, 128, pages, cache_dtype=vq.VQ_E4M3)
    k, v = (torch.zeros(vq.vq_cache_bytes(desc), dtype=torch.uint8, device="cuda:0") for _ in "kv")
    n = 200
    start = torch.tensor([0, n], dtype=torch.int32, device="cuda:0")
    lens = torch.tensor([n], dtype=torch.int32, device="cuda:0")
    rows, q = torch.randn(n, 2, 128, device="cuda:0").half(), torch.randn(n, 2, 128, device="cuda:0").half()

    def attend(*table):
        t = torch.tensor([table], dtype=torch.int32, device="cuda:0")
        batch = vq.AttnBatch(lens, t, n_tokens=n, max_len=n, q_start=start)
        out = torch.empty_like(q)
        vq.vq_attn_prompt(desc, batch, q, k, v, out, vq.attn_workspace(desc, batch))
        one = torch.empty_like(q[:1])
        last = vq.AttnBatch(lens, t, max_len=n)
        vq.vq_attn_decode(desc, last, q[-1:], k, v, one, vq.attn_workspace(desc, last))
        return out, one, batch
    _, _, low = attend(3, 4)
    vq.vq_cache_append(desc, low, rows, rows, k, v)
    want = attend(3, 4)
    k.zero_()
    v.zero_()
    _, _, high = attend(pages - 1, pages - 5)
    vq.vq_cache_append(desc, high, rows, rows, k, v)
    got = attend(pages - 1, pages - 5)
    vq.vq_cache_copy(desc, [k, v], [(pages - 1, 7), (pages - 5, pages - 2)])
    moved = attend(7, pages - 2)
    torch.cuda.synchronize()
    assert bool(want[0].any())
    for x in (got, moved):
        assert torch.equal(x[0], want[0]) and torch.equal(x[1], want[1])
