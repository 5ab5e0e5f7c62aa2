"""Attention over pages in 8 bits, and attention with a window and sinks over pages of both kinds, against the definition in 64
bits.  A cache in 8 bits stands for numbers of the 16-bit type, so the bounds are those of attention over a cache of these."""
import numpy as np
import pytest

from attn_cases import torch_type
from cache8_cases import Windowed, run_window

pytestmark = pytest.mark.gpu

LENS = [1, 0, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 255, 257, 500]


def check(p, call, **kw):
    out, lse = run_window(p, call, **kw)
    p.check(out, lse)
    return out, lse


# ------------------------------------------------------------------------------------------ 8 bits, every token
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_one_new_token(dim, page, dtype):
    check(Windowed(8, 4, dim, page, dtype, LENS, seed=dim + page, bits=8), "decode")


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_prompts(dim, page, dtype):
    check(Windowed(4, 2, dim, page, dtype, [1, 2, 17, 40, 64, 365, 0, 130], [1, 2, 17, 33, 64, 65, 0, 130], seed=dim + page, bits=8), "prompt")


@pytest.mark.parametrize("heads, kv", [(1, 1), (3, 3), (32, 8), (28, 4), (16, 1), (17, 1), (48, 1), (100, 2), (5, 5)])
def test_every_head_layout(heads, kv):
    check(Windowed(heads, kv, 128, 32, "f16", [1, 70, 0, 129, 33], seed=heads, bits=8), "decode")
    check(Windowed(heads, kv, 64, 16, "bf16", [129, 300, 31], [129, 45, 7], seed=heads, bits=8), "prompt")


@pytest.mark.parametrize("dim", [64, 96, 128, 256])
@pytest.mark.parametrize("heads, kv", [(32, 1), (40, 1), (48, 1), (96, 2)])
def test_many_heads_to_one(heads, kv, dim):
    """Several tiles of heads to a workgroup, with one part and with several; the last tile is not full."""
    for lens in ([70, 0, 300, 1] * 6, [1300, 2] * 10):
        check(Windowed(heads, kv, dim, 64, "f16", lens, seed=heads, bits=8, layout="features" if dim == 96 else "tokens"), "decode")


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("seqs, n", [(1, 5000), (2, 3001), (1, 9999), (3, 1025)])
def test_one_new_token_behind_many(seqs, n, dtype):
    check(Windowed(4, 2, 128, 16, dtype, [n - 13 * i for i in range(seqs)], seed=n, bits=8), "decode")


@pytest.mark.parametrize("layout, gap", [("tokens", 3), ("heads", 2), ("features", 1), ("odd", 1), ("odd features", 1)])
@pytest.mark.parametrize("call", ["decode", "prompt"])
@pytest.mark.parametrize("dim", [64, 96])
def test_strides(dim, call, layout, gap):
    check(Windowed(6, 2, dim, 16, "f16", [70, 3, 0, 200, 33], None if call == "decode" else [9, 3, 0, 130, 5], layout=layout, gap=gap, seed=gap, bits=8), call)


@pytest.mark.parametrize("dim, page, dtype", [(64, 16, "f16"), (96, 32, "bf16"), (128, 64, "f16"), (128, 16, "bf16"), (256, 32, "f16")])
@pytest.mark.parametrize("lens, new", [([449], [449]), ([1000], [777]), ([0, 700, 1, 450], [0, 700, 1, 450]), ([1500, 30, 0, 640], [130, 30, 3, 1]),
                                       ([5000], [40]), ([2040, 500], [1, 520])])
def test_middling_prompts(dim, page, dtype, lens, new):
    """Odd and even numbers of steps, two teams, parts and their join; the same bits every time."""
    p = Windowed(4, 2, dim, page, dtype, lens, new, layout="features" if page == 16 else "tokens", seed=sum(lens), bits=8)
    out, _ = check(p, "prompt")
    assert bool((run_window(p, "prompt")[0] == out).all())


def test_a_part_of_more_steps_than_page_numbers_are_fetched_for():
    p = Windowed(1, 1, 64, 16, "f16", [20000], [300], seed=2, bits=8)
    check(p, "prompt")


@pytest.mark.parametrize("call", ["decode", "prompt"])
def test_the_same_as_over_16_bits_of_these_values(call):
    """The values that the codes stand for, in a cache of 16 bits: within the two calls' roundings of one another."""
    import torch
    p = Windowed(8, 2, 128, 32, "bf16", [900, 64, 333], None if call == "decode" else [200, 64, 1], seed=3, bits=8)
    out, lse = run_window(p, call)
    ref = p.reference()
    b_out, b_lse = p.bounds(ref)
    p.desc.cache_dtype = 0
    p.k_pages, p.v_pages = p.k_host.to(p.dev), p.v_host.to(p.dev)
    other, other_lse = run_window(p, call)
    assert (np.abs((out.double() - other.double()).cpu().numpy()) <= 2 * b_out).all()
    assert (np.abs((lse - other_lse).double().cpu().numpy()) <= 2 * b_lse).all() and torch.isfinite(lse).all()


@pytest.mark.parametrize("call", ["decode", "prompt"])
@pytest.mark.parametrize("window", [None, 50])
def test_loud_and_quiet_blocks(call, window):
    """Blocks whose scales are the type's extremes, side by side."""
    import torch
    import oracle.attn_oracle as ao
    from cache8_cases import join8, split8
    for dtype, scales in (("f16", [2.0 ** -15, 1.0, 2.0 ** 8]), ("bf16", [2.0 ** -117, 2.0 ** -60, 1.0, 2.0 ** 100])):
        p = Windowed(2, 2, 64, 16, dtype, [200], None if call == "decode" else [70], seed=3, bits=8, window=window, sinks=3)
        rng = np.random.default_rng(2)
        c, s = split8(p.desc, p.v_pages, False)
        s = rng.choice(scales, s.shape).astype(np.float32)
        c = c.copy()
        c[(c & 0x7f) > 0x70] &= 0x8f     # up to 120: within the type at the largest scale
        p.v_pages = join8(c, s)
        p.v_host = torch.from_numpy(ao.values8(c, s, False)).to(torch_type(dtype))
        out, _ = run_window(p, call)
        ref = p.reference()
        unit = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}[dtype]
        # A weight is off by its rounding and by that of its logit (p.bounds); what it rounds to below 2^-24 of the largest is off by that.
        largest = np.abs(p.v_host.double().numpy()[p.table[0, :13]]).max()
        tiny = 2.0 ** -24 * largest * 200 if dtype == "f16" else 0
        b_out = p.bounds(ref)[0] + tiny
        assert (np.abs(out.double().cpu().numpy() - ref[0]) <= b_out).all() and unit


@pytest.mark.parametrize("call", ["decode", "prompt"])
@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("window, sinks", [(None, 0), (40, 0), (40, 75), (64, 3)])
@pytest.mark.parametrize("where", ["k", "v"])
def test_nan_goes_to_the_rows_that_see_it(where, window, sinks, bits, call):
    """From the sinks, from a window's two ends and from between, to the heads that read it and no other."""
    import torch
    from cache8_cases import join8, split8
    for token in (0, 2, 70, 109, 110, 149):
        p = Windowed(4, 2, 64, 16, "f16", [150, 60], None if call == "decode" else [100, 20], seed=5, bits=bits, window=window, sinks=sinks)
        page, slot = int(p.table[0, token // 16]), token % 16
        host, at = (p.k_host, (page, 1, slot, 9)) if where == "k" else (p.v_host, (page, 1, 9, slot))
        host[at] = float("nan")
        if bits == 8:
            buffer = p.k_pages if where == "k" else p.v_pages
            c, s = split8(p.desc, buffer, where == "k")
            c = c.copy()
            c[at] = 0xff
            buffer.copy_(join8(c, s))
        else:
            p.k_pages, p.v_pages = p.k_host.to(p.dev), p.v_host.to(p.dev)
        out, lse = run_window(p, call)
        ref = p.reference()
        got = out.double().cpu().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(ref[0])) and np.array_equal(np.isnan(lse.cpu().numpy()), np.isnan(ref[1]))
        over = np.abs(got - ref[0]) - p.bounds(ref)[0]
        assert not (over > 0).any() and torch.is_tensor(out)


@pytest.mark.parametrize("call", ["decode", "prompt"])
@pytest.mark.parametrize("value", [float("inf"), float("-inf")])
def test_infinite_values_within_and_outside_a_window(value, call):
    """Pages in 16 bits: infinity for the rows whose window or sinks hold it, whatever its weight rounds to; the others do not feel it."""
    for token in (1, 5, 109, 110, 140):
        p = Windowed(4, 2, 64, 16, "f16", [150], None if call == "decode" else [100], seed=6, window=40, sinks=4, spread=20.0)
        p.v_host[int(p.table[0, token // 16]), 1, 3, token % 16] = value
        p.v_pages = p.v_host.to(p.dev)
        got = run_window(p, call)[0].double().cpu().numpy()
        ref = p.reference()
        assert np.array_equal(np.isfinite(got), np.isfinite(ref[0]))
        assert np.array_equal(got[np.isinf(ref[0])], ref[0][np.isinf(ref[0])])
        b_out, _ = p.bounds(ref)
        with np.errstate(invalid="ignore"):
            over = (np.abs(got - ref[0]) > b_out) & np.isfinite(ref[0]) & np.isfinite(b_out)
        assert not over.any()


# ------------------------------------------------------------------------------------------ windows
WINDOWS = [(1, 0), (1, 1), (2, 0), (15, 4), (16, 16), (17, 1), (31, 33), (32, 0), (33, 64), (64, 65), (65, 3), (100, 0), (128, 128), (300, 20), (2 ** 29, 0), (3, 2 ** 29)]


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("window, sinks", WINDOWS)
def test_one_new_token_with_a_window(window, sinks, bits):
    for i, (dim, page, dtype) in enumerate(((128, 16, "f16"), (64, 64, "bf16"), (96, 32, "f16"), (256, 128, "bf16"))):
        p = Windowed(8, 4, dim, page, dtype, LENS, seed=window % 1000 + i, bits=bits, window=window, sinks=sinks, give_back=True)
        check(p, "decode")


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("window, sinks", WINDOWS)
def test_prompts_with_a_window(window, sinks, bits):
    for i, (heads, kv, dim, page, dtype) in enumerate(((4, 2, 128, 16, "f16"), (7, 1, 64, 64, "bf16"), (3, 3, 96, 32, "f16"), (2, 1, 256, 128, "bf16"))):
        p = Windowed(heads, kv, dim, page, dtype, [1, 2, 17, 40, 64, 365, 0, 290], [1, 2, 17, 33, 64, 65, 0, 290], seed=window % 1000 + i, bits=bits, window=window,
                     sinks=sinks, give_back=True)
        check(p, "prompt")


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("window, sinks", [(700, 0), (1000, 4), (2000, 100), (4000, 1)])
def test_long_windows_in_parts(window, sinks, bits):
    """Windows that are split over their length: one new token, and few rows behind many tokens."""
    for heads, kv in ((4, 4), (6, 2), (40, 1)):
        check(Windowed(heads, kv, 128, 16, "f16", [5000, 3, 2500], seed=heads, bits=bits, window=window, sinks=sinks, give_back=True), "decode")
    for heads, kv in ((4, 4), (6, 2)):
        check(Windowed(heads, kv, 64, 16, "bf16", [5000, 70, 2500], [5, 0, 130], seed=heads, bits=bits, window=window, sinks=sinks, give_back=True), "prompt")


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("dim, heads, kv", [(64, 4, 2), (96, 4, 4), (128, 8, 2), (256, 2, 2)])
def test_long_prompts_with_a_window(dim, heads, kv, bits):
    """Several tiles, each with steps that are passed over, of one team and of two; the token index contiguous."""
    for window, sinks in ((60, 4), (200, 0), (513, 70)):
        p = Windowed(heads, kv, dim, 16, "f16", [900, 1300], [900, 700], seed=dim, bits=bits, window=window, sinks=sinks, give_back=True, layout="features")
        out, _ = check(p, "prompt")
        assert bool((run_window(p, "prompt")[0] == out).all())


@pytest.mark.parametrize("bits", [16, 8])
def test_a_wide_window_is_no_window(bits):
    """Windows that reach the first token: the same bits as the call without one, or the same within the roundings where the split is another."""
    for call in ("decode", "prompt"):
        p = Windowed(4, 2, 128, 32, "f16", [700, 0, 90], None if call == "decode" else [300, 0, 90], seed=1, bits=bits)
        out, lse = check(p, call)
        p.window, p.sinks = 2 ** 29, 5
        again, lse2 = check(p, call)
        if bits == 8:
            assert bool((out == again).all()) and bool((lse == lse2).all())


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("call", ["decode", "prompt"])
def test_rows_before_the_first_token_and_lengths_beyond_the_bound(call, bits):
    import torch
    if call == "prompt":
        p = Windowed(4, 2, 64, 16, "bf16", [3, 0, 200, 1], [10, 5, 210, 90], seed=3, bits=bits, window=20, sinks=2)
        out, lse = check(p, call)
        for s in range(4):
            a, b = int(p.q_start[s]), int(p.q_start[s + 1])
            none = b - a - p.lens[s]
            assert not out[a:a + none].any() and bool((lse[a:a + none] == -np.inf).all())
    p = Windowed(4, 4, 64, 16, "f16", [100, 40, 61], seed=1, bits=bits, window=30, sinks=5)
    p.lens_d.copy_(torch.tensor([2 ** 31 - 1, 40, -5], dtype=torch.int32))
    out, lse = run_window(p, call, max_len=50)
    p.lens = [50, 40, 0]
    p.check(out, lse)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("call", ["decode", "prompt"])
def test_another_stream_and_captured_graphs(call, bits):
    """A graph follows what the arrays hold when it is replayed; two graphs share a workspace, one after the other."""
    import torch
    import paper_2402_15319_amd as vq
    p = Windowed(8, 2, 128, 16, "f16", [2000, 37, 900], None if call == "decode" else [40, 37, 3], seed=9, bits=bits, window=700, sinks=4)
    p.check(*run_window(p, call, stream=torch.cuda.Stream()))
    batch = p.batch(max_len=p.width * 16, decode=call == "decode")
    ws = vq.attn_workspace(p.desc, batch)
    f = vq.vq_attn_decode_window if call == "decode" else vq.vq_attn_prompt_window
    graphs = []
    for window in (700, 90):
        out, lse = torch.empty_like(p.q), torch.empty(p.total, p.heads, device="cuda:0")
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            f(p.desc, batch, vq.VQAttnWindow(window, 4), p.q, p.k_pages, p.v_pages, out, ws, lse=lse)
        graphs.append((window, g, out, lse))
    for lens in ([2000, 37, 900], [70, 37, 333], [1999, 37, 64]):
        p.lens = lens
        p.lens_d.copy_(torch.tensor(lens, dtype=torch.int32))
        for _, g, out, _ in graphs:
            out.fill_(float("nan"))
            g.replay()
        torch.cuda.synchronize()
        for window, _, out, lse in graphs:
            p.window = window
            p.check(out, lse)


@pytest.mark.parametrize("bits", [16, 8])
def test_a_prompt_is_what_its_tokens_are_one_at_a_time(bits):
    import torch
    import paper_2402_15319_amd as vq
    p = Windowed(4, 2, 128, 16, "f16", [200], [200], seed=4, bits=bits, window=37, sinks=3)
    out, lse = run_window(p, "prompt")
    b_out, b_lse = p.bounds(p.reference())
    got, got_lse = torch.empty_like(out), torch.empty_like(lse)
    for t in range(200):
        batch = vq.AttnBatch(torch.tensor([t + 1], dtype=torch.int32, device="cuda:0"), p.table_d, max_len=t + 1)
        vq.vq_attn_decode_window(p.desc, batch, vq.VQAttnWindow(37, 3), p.q[t:t + 1], p.k_pages, p.v_pages, got[t:t + 1], vq.attn_workspace(p.desc, batch),
                                 lse=got_lse[t:t + 1])
    torch.cuda.synchronize()
    assert (np.abs((got - out).double().cpu().numpy()) <= 2 * b_out).all()
    assert (np.abs((got_lse - lse).double().cpu().numpy()) <= 2 * b_lse).all()


@pytest.mark.parametrize("bits, value", [(16, float("nan")), (16, float("inf")), (8, float("nan"))])
@pytest.mark.parametrize("heads, kv, dim", [(2, 2, 64), (4, 1, 128), (2, 1, 96), (1, 1, 256)])
def test_what_is_no_number_in_long_prompts_with_a_window(heads, kv, dim, bits, value):
    """Steps that some waves' rows see whole and others in part, or not at all: it goes to the rows that see it, and every other row is what it is
    without it, bit for bit."""
    import torch
    from cache8_cases import join8, split8
    for window, sinks in ((150, 0), (70, 100)):
        p = Windowed(heads, kv, dim, 16, "f16", [420], [420], seed=8, bits=bits, window=window, sinks=sinks)
        clean = run_window(p, "prompt")
        for token in (3, 99, 130, 200, 319, 419):
            page, slot = int(p.table[0, token // 16]), token % 16
            if bits == 8:
                c, s = split8(p.desc, p.v_pages, False)
                c = c.copy()
                was = p.v_pages
                c[page, 0, 5, slot] = 0x7f
                p.v_pages = join8(c, s)
            else:
                was = p.v_pages.clone()
                p.v_pages[page, 0, 5, slot] = value
            out, lse = run_window(p, "prompt")
            p.v_pages = was
            rows = torch.arange(420, device=out.device)
            sees = (rows >= token) & ((rows < token + window) | (token < sinks))
            reads = torch.arange(heads, device=out.device) < heads // kv
            hit = (sees[:, None] & reads)[..., None] & (torch.arange(dim, device=out.device) == 5)
            assert bool((torch.isnan(out[hit]) if value != value else out[hit] == value).all())
            assert torch.equal(out[~hit], clean[0][~hit]) and torch.equal(lse, clean[1])


@pytest.mark.parametrize("call", ["decode", "prompt"])
@pytest.mark.parametrize("bits, dim, page", [(8, 128, 64), (16, 256, 128), (8, 256, 16), (16, 64, 16)])
def test_pages_beyond_4_gib(bits, dim, page, call):
    """The last pages of a large cache: bit for bit what the same tokens give in a small one."""
    import torch
    from cache8_cases import split8
    p = Windowed(16, 16, dim, page, "f16", [400, 33], None if call == "decode" else [70, 33], seed=2, bits=bits, window=150, sinks=20)
    out, lse = check(p, call)
    few, by_page = p.n_pages, 16 * page * dim * bits // 8
    many = 2 ** 32 // by_page + few + 3

    def put(small, by_slot):
        if bits == 16:
            big = torch.zeros(many, *small.shape[1:], dtype=small.dtype, device=small.device)
            big[many - few:] = small
            return big
        codes, scales = (torch.from_numpy(np.ascontiguousarray(x)).to(small.device).view(torch.uint8).flatten() for x in split8(p.desc, small, by_slot))
        big = torch.zeros(many * (by_page + page * 4), dtype=torch.uint8, device=small.device)
        big[(many - few) * by_page:many * by_page] = codes
        big[len(big) - len(scales):] = scales
        return big

    p.k_pages, p.v_pages = put(p.k_pages, True), put(p.v_pages, False)
    p.desc.n_pages = many
    p.table_d.add_(many - few)
    far, far_lse = run_window(p, call)
    assert torch.equal(far, out) and torch.equal(far_lse, lse)


@pytest.mark.parametrize("bits, window", [(8, None), (8, 40), (16, 40)])
@pytest.mark.parametrize("dim", [64, 128])
def test_rows_behind_the_last_sequence(dim, bits, window):
    """A padded batch: q_start ends before n_tokens, and the rows from there on stay as they were."""
    import torch
    import paper_2402_15319_amd as vq
    p = Windowed(4, 2, dim, 16, "f16", [70, 300, 9], [70, 33, 2], seed=6, bits=bits, window=window, sinks=3)
    out, lse = check(p, "prompt")
    for more in (1, 200):
        pad = lambda t, x: torch.cat([t, torch.full((more, *t.shape[1:]), x, dtype=t.dtype, device=t.device)])  # noqa: E731
        batch = vq.AttnBatch(p.lens_d, p.table_d, n_tokens=p.total + more, max_len=300, q_start=p.start_d)
        o, e = pad(torch.empty_like(out), 55.0), pad(torch.empty_like(lse), 55.0)
        args = pad(p.q, float("nan")), p.k_pages, p.v_pages, o, vq.attn_workspace(p.desc, batch)
        if window is None:
            vq.vq_attn_prompt(p.desc, batch, *args, lse=e)
        else:
            vq.vq_attn_prompt_window(p.desc, batch, vq.VQAttnWindow(window, 3), *args, lse=e)
        torch.cuda.synchronize()
        p.check(o[:p.total], e[:p.total])
        assert bool((o[p.total:] == 55).all()) and bool((e[p.total:] == 55).all())
