"""Attention over the paged cache against the definition in 64 bits: every head layout, type and page size, lengths from none
to thousands, rows that attend nothing, NaN and infinities where no token is, strides."""
import numpy as np
import pytest

from attn_cases import Problem, run, torch_type

pytestmark = pytest.mark.gpu

LENS = [1, 0, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 255, 257, 500]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_one_new_token(dim, page, dtype):
    p = Problem(8, 4, dim, page, dtype, LENS, seed=dim + page)
    p.check(*run(p, "decode"))


@pytest.mark.parametrize("heads, kv", [(1, 1), (3, 3), (32, 8), (28, 4), (16, 1), (17, 1), (48, 1), (100, 2), (5, 5)])
def test_one_new_token_of_every_head_layout(heads, kv):
    p = Problem(heads, kv, 128, 32, "f16", [1, 70, 0, 129, 33], seed=heads)
    p.check(*run(p, "decode"))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("seqs, n", [(1, 5000), (2, 3001), (1, 9999), (3, 1025)])
def test_one_new_token_behind_many(seqs, n, dtype):
    p = Problem(4, 2, 128, 16, dtype, [n - 13 * i for i in range(seqs)], seed=n)
    p.check(*run(p, "decode"))


@pytest.mark.parametrize("layout, gap", [("tokens", 0), ("tokens", 3), ("heads", 0), ("heads", 2), ("features", 0), ("features", 1),
                                         ("odd", 0), ("odd", 1), ("odd features", 0), ("odd features", 1)])
@pytest.mark.parametrize("call", ["decode", "prompt"])
def test_strides(call, layout, gap):
    lens = [70, 3, 0, 200, 33]
    p = Problem(6, 2, 64, 16, "f16", lens, new=None if call == "decode" else [9, 3, 0, 130, 5], layout=layout, gap=gap, seed=gap)
    p.check(*run(p, call))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_prompts(dim, page, dtype):
    new = [1, 2, 17, 33, 64, 65, 0, 130]
    lens = [1, 2, 17, 40, 64, 365, 0, 130]
    p = Problem(4, 2, dim, page, dtype, lens, new, seed=dim + page)
    p.check(*run(p))


@pytest.mark.parametrize("heads, kv", [(1, 1), (3, 3), (8, 2), (7, 1), (20, 1)])
def test_prompts_of_every_head_layout(heads, kv):
    p = Problem(heads, kv, 128, 32, "f16", [129, 300, 31], [129, 45, 7], seed=heads)
    p.check(*run(p))


@pytest.mark.parametrize("n, prefix", [(127, 0), (128, 0), (129, 0), (255, 1), (300, 500), (1, 700), (700, 0), (3, 1500), (16, 2000)])
def test_one_prompt(n, prefix):
    p = Problem(4, 2, 128, 16, "f16", [n + prefix], [n], layout="features", seed=n)
    p.check(*run(p))


def test_rows_before_the_first_token_attend_nothing():
    """More new tokens than the cache counts: the first of them have negative positions."""
    p = Problem(4, 2, 64, 16, "bf16", [3, 0, 200, 1], [10, 5, 210, 90], seed=3)
    out, lse = run(p)
    p.check(out, lse)
    for s in range(4):
        a, b = int(p.q_start[s]), int(p.q_start[s + 1])
        none = b - a - p.lens[s]
        assert not out[a:a + none].any() and bool((lse[a:a + none] == -np.inf).all())


@pytest.mark.parametrize("call", ["decode", "prompt"])
def test_lengths_beyond_the_bound_are_cut(call):
    import torch
    p = Problem(4, 4, 64, 16, "f16", [100, 40, 61], seed=1)
    p.lens_d.copy_(torch.tensor([2 ** 31 - 1, 40, -5], dtype=torch.int32))
    out, lse = run(p, call, max_len=50)
    p.lens = [50, 40, 0]
    p.check(out, lse)


@pytest.mark.parametrize("call", ["decode", "prompt"])
def test_page_numbers_outside_the_cache_stay_harmless(call):
    """What such a sequence gets is not specified; nothing is read outside, and the others are right."""
    p = Problem(4, 4, 64, 16, "f16", [100, 40, 61], seed=1)
    import torch
    p.table_d[0, :3] = torch.tensor([-7, 2 ** 31 - 1, p.n_pages], dtype=torch.int32)
    out, _ = run(p, call)
    ref = p.reference()
    b_out, _ = p.bounds(ref)
    got = out.double().cpu().numpy()
    assert (np.abs(got - ref[0])[1:] <= b_out[1:]).all()


@pytest.mark.parametrize("call", ["decode", "prompt"])
@pytest.mark.parametrize("where, value", [("k", np.inf), ("v", np.nan), ("v", -np.inf), ("q", np.nan), ("q", 0.0), ("k", 60000.0)])
def test_infinities_and_nan_among_the_attended(call, where, value):
    """They go through the formula, to the rows and heads that attend them and no other."""
    import torch
    p = Problem(4, 2, 64, 16, "f16", [150, 60], new=None if call == "decode" else [100, 20], seed=5)
    at = int(p.table[0, 70 // 16]), 70 % 16
    if where == "k":
        p.k_host[at[0], 1, at[1], :] = value
    elif where == "v":
        p.v_host[at[0], 1, 3, at[1]] = value
    else:
        p.q_host[0, 2] = value
    p.k_pages, p.v_pages, p.q = p.k_host.to(p.dev), p.v_host.to(p.dev), p.rows(p.q_host, p.heads)
    out, lse = run(p, call)
    ref = p.reference()
    got = out.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(ref[0]))
    assert np.array_equal(np.isinf(got), np.isinf(ref[0])) and np.array_equal(np.sign(got[np.isinf(got)]), np.sign(ref[0][np.isinf(got)]))
    assert np.array_equal(np.isnan(lse.cpu().numpy()), np.isnan(ref[1]))
    b_out, _ = p.bounds(ref)
    with np.errstate(invalid="ignore"):
        over = (np.abs(got - ref[0]) > b_out) & np.isfinite(ref[0]) & np.isfinite(b_out)
    assert not over.any()


@pytest.mark.parametrize("call", ["decode", "prompt"])
@pytest.mark.parametrize("spread", [0.0, 30.0])
def test_flat_and_peaked_weights(call, spread):
    p = Problem(4, 2, 128, 32, "f16", [700, 300], new=None if call == "decode" else [200, 3], seed=6, spread=spread)
    p.check(*run(p, call))


def test_same_bits_every_time_and_whatever_the_split():
    """Two calls give the same bits; other bounds on the lengths split the work elsewhere, and stay within the rounding."""
    import torch
    p = Problem(8, 2, 128, 16, "f16", [4000, 37, 900], seed=8)
    ref = p.reference()
    first = run(p, "decode")
    again = run(p, "decode")
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    for max_len in (4000 + 16, p.width * 16):
        p.check(*run(p, "decode", max_len=max_len), ref=ref)


def test_a_workspace_serves_calls_of_other_sizes():
    """One workspace, as large as the largest needs, through calls of different shapes, one after another."""
    import torch
    import paper_2402_15319_amd as vq
    ps = [Problem(8, 2, 128, 16, "f16", [3000, 10], seed=1), Problem(4, 4, 64, 32, "bf16", [50] * 9, seed=2),
          Problem(8, 1, 128, 64, "f16", [2500], [20], seed=3)]
    calls = ["decode", "decode", "prompt"]
    need = max(vq.vq_attn_workspace_bytes(p.desc, p.batch(decode=c == "decode")) for p, c in zip(ps, calls))
    ws = torch.zeros(need, dtype=torch.uint8, device="cuda:0")
    refs = [p.reference() for p in ps]
    for i in (0, 1, 2, 0, 2, 1, 0):
        p = ps[i]
        out = torch.empty_like(p.q)
        lse = torch.empty(p.total, p.heads, device="cuda:0")
        f = vq.vq_attn_decode if calls[i] == "decode" else vq.vq_attn_prompt
        f(p.desc, p.batch(decode=calls[i] == "decode"), p.q, p.k_pages, p.v_pages, out, ws, lse=lse)
        torch.cuda.synchronize()
        p.check(out, lse, ref=refs[i])


@pytest.mark.parametrize("call", ["decode", "prompt"])
def test_another_stream_and_a_captured_graph(call):
    """A graph follows what the arrays hold when it is replayed."""
    import torch
    import paper_2402_15319_amd as vq
    p = Problem(8, 2, 128, 16, "f16", [2000, 37, 900], new=None if call == "decode" else [40, 37, 3], seed=9)
    p.check(*run(p, call, stream=torch.cuda.Stream()))
    batch = p.batch(max_len=p.width * 16, decode=call == "decode")
    ws = vq.attn_workspace(p.desc, batch)
    out = torch.empty_like(p.q)
    lse = torch.empty(p.total, p.heads, device="cuda:0")
    f = vq.vq_attn_decode if call == "decode" else vq.vq_attn_prompt
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        f(p.desc, batch, p.q, p.k_pages, p.v_pages, out, ws, lse=lse)
    for lens in ([2000, 37, 900], [70, 37, 333], [1999, 37, 64]):
        p.lens = lens
        p.lens_d.copy_(torch.tensor(lens, dtype=torch.int32))
        out.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        p.check(out, lse)


def test_offsets_beyond_32_bits():
    """Pages at the end of buffers of more than 2^32 bytes."""
    import torch
    import paper_2402_15319_amd as vq
    small = Problem(2, 2, 128, 128, "f16", [300, 200], seed=4)
    pages = 2 ** 32 // (2 * 128 * 128 * 2) + 70
    free, _ = torch.cuda.mem_get_info()
    assert free > 4 * pages * 2 * 128 * 128 * 2
    k = torch.zeros(pages, 2, 128, 128, dtype=torch.float16, device="cuda:0")
    v = torch.zeros(pages, 2, 128, 128, dtype=torch.float16, device="cuda:0")
    shift = pages - small.n_pages
    k[shift:], v[shift:] = small.k_pages, small.v_pages
    small.k_pages, small.v_pages = k, v
    small.table_d += shift
    small.desc = vq.make_attn_desc(2, 2, 128, 128, pages, vq.VQ_F16, small.scale)
    small.check(*run(small, "decode"))
    small.check(*run(small, "prompt"))
    assert torch_type("f16") == torch.float16


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("heads, kv", [(4, 4), (4, 2), (8, 2), (7, 1), (12, 1)])
@pytest.mark.parametrize("layout, gap", [("tokens", 1), ("heads", 0), ("features", 0), ("odd", 0), ("odd features", 0)])
def test_long_prompts_in_every_order(layout, gap, heads, kv, dtype):
    """Prompts long enough that a wave takes successive tokens of one head, some of them with an end inside a wave, some empty."""
    p = Problem(heads, kv, 64, 32, dtype, [290, 0, 410, 33, 127], [257, 0, 128, 33, 127], layout=layout, gap=gap, seed=heads)
    p.check(*run(p))


@pytest.mark.parametrize("dim, page", [(96, 16), (128, 64), (256, 32), (256, 128)])
def test_long_prompts_of_every_size_of_head(dim, page):
    p = Problem(4, 1, dim, page, "f16", [400, 333], [300, 333], seed=dim)
    p.check(*run(p))


@pytest.mark.parametrize("call", ["decode", "prompt"])
def test_many_sequences(call):
    """More than a wave looks at in one turn, with none, one or a few tokens."""
    rng = np.random.default_rng(1)
    lens = rng.integers(0, 40, 200).tolist()
    new = None if call == "decode" else [int(rng.integers(0, n + 1)) for n in lens]
    p = Problem(4, 2, 64, 16, "bf16", lens, new, seed=2)
    p.check(*run(p, call))


@pytest.mark.parametrize("call", ["decode", "prompt"])
def test_nothing_in_any_cache(call):
    import torch
    p = Problem(4, 2, 64, 16, "f16", [0, 0, 0], [1, 1, 1], seed=2)
    out, lse = run(p, call, max_len=0)
    assert not out.any() and bool(torch.isneginf(lse).all())


@pytest.mark.parametrize("new", [1, 5, 40])
def test_prompts_of_few_rows_behind_many_tokens(new):
    """Split over the length and joined, with every layout of heads that a tile can have."""
    for heads, kv in ((4, 4), (6, 2), (4, 1), (20, 1)):
        p = Problem(heads, kv, 64, 16, "f16", [3000, 2500 - new, 70], [new, 2, 0], seed=heads)
        p.check(*run(p))


def test_a_prompt_is_what_its_tokens_are_one_at_a_time():
    """Every row of a prompt against the call for one new token with that many tokens in the cache: two roundings apart."""
    import torch
    import paper_2402_15319_amd as vq
    p = Problem(4, 2, 128, 16, "f16", [200], [200], seed=4)
    out, lse = run(p)
    ref = p.reference()
    b_out, b_lse = p.bounds(ref)
    got = torch.empty_like(out)
    got_lse = torch.empty_like(lse)
    for t in range(200):
        lens = torch.tensor([t + 1], dtype=torch.int32, device="cuda:0")
        batch = vq.AttnBatch(lens, p.table_d, max_len=t + 1)
        vq.vq_attn_decode(p.desc, batch, p.q[t:t + 1], p.k_pages, p.v_pages, got[t:t + 1], vq.attn_workspace(p.desc, batch), lse=got_lse[t:t + 1])
    torch.cuda.synchronize()
    assert (np.abs((got - out).double().cpu().numpy()) <= 2 * b_out).all()
    assert (np.abs((got_lse - lse).double().cpu().numpy()) <= 2 * b_lse).all()


@pytest.mark.parametrize("dim", [64, 96, 128, 256])
@pytest.mark.parametrize("heads, kv", [(17, 1), (32, 1), (40, 1), (48, 1), (64, 1), (100, 1), (96, 2)])
def test_many_heads_to_one(heads, kv, dim):
    """Several tiles of heads to a workgroup, with one part and with several; the last tile is not full."""
    for lens in ([70, 0, 300, 1] * 6, [1300, 2] * 10):
        p = Problem(heads, kv, dim, 64, "f16", lens, seed=heads, layout="features" if dim == 96 else "tokens")
        p.check(*run(p, "decode"))


@pytest.mark.parametrize("dim, page, dtype", [(64, 16, "f16"), (64, 128, "bf16"), (96, 32, "f16"), (96, 16, "bf16"), (128, 64, "f16"), (128, 16, "bf16"), (256, 32, "f16")])
@pytest.mark.parametrize("lens, new", [([449], [449]), ([513], [513]), ([1000], [777]), ([1600], [1600]), ([0, 700, 1, 450], [0, 700, 1, 450]),
                                       ([1500, 30, 0, 640], [130, 30, 3, 1]), ([5000], [40]), ([2040, 500], [1, 520])])
def test_middling_prompts_on_few_heads(dim, page, dtype, lens, new):
    """Few tiles of 8 to 80 steps each: odd and even numbers of steps, rows without tokens, sequences that are much shorter than the longest."""
    p = Problem(4, 2, dim, page, dtype, lens, new=new, layout="features" if page == 16 else "tokens", seed=sum(lens))
    out, lse = run(p)
    p.check(out, lse)
    again, _ = run(p)
    assert bool((out == again).all())


@pytest.mark.parametrize("where, value", [("k", np.inf), ("v", np.nan), ("v", -np.inf)])
def test_what_is_no_number_in_middling_prompts(where, value):
    """It goes to the rows that attend it and no other, from whichever half of the steps."""
    p = Problem(4, 2, 128, 16, "f16", [700], new=[700], seed=9)
    for token in (70, 330, 699):
        at = int(p.table[0, token // 16]), token % 16
        if where == "k":
            p.k_host[at[0], 1, at[1], :] = value
        else:
            p.v_host[at[0], 1, 3, at[1]] = value
    p.k_pages, p.v_pages = p.k_host.to(p.dev), p.v_host.to(p.dev)
    got = run(p)[0].double().cpu().numpy()
    ref = p.reference()
    assert np.array_equal(np.isfinite(got), np.isfinite(ref[0]))
    b_out, _ = p.bounds(ref)
    with np.errstate(invalid="ignore"):
        over = (np.abs(got - ref[0]) > b_out) & np.isfinite(ref[0]) & np.isfinite(b_out)
    assert not over.any()
