"""Pages in 8 bits and windows without a GPU: what the entry points refuse, sizes, the binding's own checks, and the pool's pages that are
given back."""
import ctypes
import random

import pytest
import torch

import paper_2402_15319_amd as vq
from paper_2402_15319_amd import cache as vc
from test_attn_abi import A, ALIGN, ARG, DESC, NULL, S, UNSUPPORTED, _batch
from test_attn_binding import On, reached  # noqa: F401


def _desc(**change):
    return vq.make_attn_desc(**{**dict(heads=8, kv_heads=2, head_dim=128, page_size=16, n_pages=100, dtype=vq.VQ_F16, scale=0.1), **change})


def _window(name, desc, batch, window=None, q=A, qs=None, k=2 * A, v=3 * A, out=4 * A, os=None, lse=5 * A, ws=6 * A, n=1 << 40):
    window = vq.VQAttnWindow(100, 4) if window is None else window
    return getattr(vq.lib(), name)(desc, batch, window if window != "none" else None, q, qs, k, v, out, os, lse, ws, n, 0)


NAMES = ("vq_attn_decode_window", "vq_attn_prompt_window")


@pytest.mark.parametrize("cache_dtype", [1, vq.VQ_F16, vq.VQ_BF16, vq.VQ_I8, 7, -1])
def test_cache_types_that_are_refused(cache_dtype):
    d, size, L = _desc(), ctypes.c_size_t(), vq.lib()
    d.cache_dtype = cache_dtype
    assert d.reserved == cache_dtype
    assert [_window(n, d, _batch()) for n in NAMES] == [DESC] * 2
    assert L.vq_cache_append(d, _batch(), A, None, 2 * A, None, 3 * A, 4 * A, 0) == DESC
    assert L.vq_cache_bytes(d, ctypes.byref(size)) == DESC
    assert L.vq_cache_copy(d, 1, (ctypes.c_void_p * 1)(A), 1, (ctypes.c_int32 * 2)(0, 1), 0) == DESC


@pytest.mark.parametrize("change, status", [(dict(heads=9), DESC), (dict(head_dim=80), UNSUPPORTED), (dict(page_size=8), UNSUPPORTED), (dict(dtype=vq.VQ_F32), UNSUPPORTED),
                                            (dict(dtype=vq.VQ_E4M3), UNSUPPORTED), (dict(scale=0.0), ARG), (dict(scale=float("nan")), ARG)])
def test_bad_descriptors(change, status):
    for cache_dtype in (None, vq.VQ_E4M3):
        d = _desc(**change, cache_dtype=cache_dtype)
        assert [_window(n, d, _batch()) for n in NAMES] == [status] * 2


@pytest.mark.parametrize("window, sinks", [(0, 0), (-1, 4), (2 ** 29 + 1, 0), (-2 ** 31, 0), (5, -1), (5, 2 ** 29 + 1), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_bad_windows(window, sinks):
    for cache_dtype in (None, vq.VQ_E4M3):
        for n in NAMES:
            assert _window(n, _desc(cache_dtype=cache_dtype), _batch(), vq.VQAttnWindow(window, sinks)) == ARG
    assert ctypes.sizeof(vq.VQAttnWindow) == 8


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("cache_dtype", [None, vq.VQ_E4M3])
def test_everything_else_is_refused_as_without_a_window(name, cache_dtype):
    d, b = _desc(cache_dtype=cache_dtype), _batch()
    assert _window(name, d, b, "none") == NULL and _window(name, None, b) == NULL and _window(name, d, None) == NULL
    for what in ("q", "k", "v", "out", "ws"):
        assert _window(name, d, b, **{what: None}) == NULL
        assert _window(name, d, b, **{what: A + 8}) == ALIGN
    assert _window(name, d, b, lse=A + 2) == ALIGN
    for same in ("q", "k", "v"):
        assert _window(name, d, b, **{same: 4 * A}) == ARG
    assert _window(name, d, b, n=0) == ARG
    assert _window(name, d, b, os=S(1000, 128, 1)) == ARG and _window(name, d, b, qs=S(-1024, 128, 1)) == ARG
    for change in (dict(n_seqs=0), dict(n_tokens=0), dict(max_len=161), dict(max_len=-1)):
        assert _window(name, d, _batch(**change)) == ARG
    if "decode" in name:
        assert _window(name, d, _batch(n_tokens=5)) == ARG


def test_append_and_copy_refusals_in_8_bits():
    d, b, L = _desc(cache_dtype=vq.VQ_E4M3), _batch(), vq.lib()
    for i in range(4):
        for bad, status in ((None, NULL), (A + 2, ALIGN)):
            p = [A, 2 * A, 3 * A, 4 * A]
            p[i] = bad
            assert L.vq_cache_append(d, b, p[0], None, p[1], None, p[2], p[3], 0) == status
    assert L.vq_cache_append(d, b, A, None, 2 * A, None, 3 * A, 3 * A, 0) == ARG
    assert L.vq_cache_copy(d, 1, (ctypes.c_void_p * 1)(A + 8), 1, (ctypes.c_int32 * 2)(0, 1), 0) == ALIGN
    assert L.vq_cache_copy(d, 1, (ctypes.c_void_p * 1)(A), 1, (ctypes.c_int32 * 2)(0, 100), 0) == ARG


def test_sizes():
    """A byte a value, and four for the 16 tokens of a head."""
    d = _desc(cache_dtype=vq.VQ_E4M3)
    assert vq.vq_cache_bytes(d) == 100 * 2 * 16 * 128 + 100 * 2 * 4
    assert vq.vq_cache_bytes(_desc(cache_dtype=vq.VQ_E4M3, n_pages=2 ** 31 - 1, page_size=128)) == (2 ** 31 - 1) * 2 * (128 * 128 + 8 * 4)
    assert vq.make_attn_desc(8, 2, 128, 16, 5).cache_dtype == 0 and vq.make_attn_desc(8, 2, 128, 16, 5, cache_dtype=vq.VQ_E4M3).cache_dtype == 6


def _case(cache_dtype=vq.VQ_E4M3, n=4):
    d = vq.make_attn_desc(8, 2, 128, 16, 5, cache_dtype=cache_dtype)
    batch = vq.AttnBatch(On(torch.ones(n, dtype=torch.int32)), On(torch.zeros(n, 2, dtype=torch.int32)), max_len=32)
    size = 5 * 2 * 16 * 128
    pages = lambda: torch.zeros(size + size // 512, dtype=torch.uint8) if cache_dtype else torch.zeros(5, 2, 16, 128).half()  # noqa: E731
    t = dict(q=torch.zeros(n, 8, 128).half(), k_pages=pages(), v_pages=pages(), out=torch.zeros(n, 8, 128).half(),
             workspace=torch.zeros(1 << 20, dtype=torch.uint8), lse=torch.zeros(n, 8))
    return d, batch, {a: On(b) for a, b in t.items()}


def _attend(d, batch, t, call):
    call(d, batch, vq.VQAttnWindow(9, 1), t["q"], t["k_pages"], t["v_pages"], t["out"], t["workspace"], lse=t["lse"], stream=0)


@pytest.mark.parametrize("cache_dtype", [None, vq.VQ_E4M3])
def test_the_binding_checks_buffers_types_and_devices(reached, cache_dtype):  # noqa: F811
    d, batch, t = _case(cache_dtype)
    for call in (vq.vq_attn_decode_window, vq.vq_attn_prompt_window):
        _attend(d, batch, t, call)
        for name in t:
            with pytest.raises(ValueError):
                _attend(d, batch, {**t, name: t[name].as_subclass(torch.Tensor)}, call)      # on the host
        for name in ("k_pages", "v_pages"):
            for bad in (t[name].reshape(-1)[:-1], t[name].view(torch.int8), t[name].reshape(-1).repeat(2)[::2]):
                with pytest.raises(ValueError):
                    _attend(d, batch, {**t, name: On(bad)}, call)
        for bad in (t["q"][:3], t["q"].bfloat16(), t["q"][..., :64]):
            with pytest.raises(ValueError):
                _attend(d, batch, {**t, "q": On(bad)}, call)
    assert reached == ["vq_attn_decode_window", "vq_attn_prompt_window"]
    new = On(torch.zeros(4, 2, 128).half())
    vq.vq_cache_append(d, batch, new, new, t["k_pages"], t["v_pages"], stream=0)
    with pytest.raises(ValueError):
        vq.vq_cache_append(d, batch, new, new, t["k_pages"], On(t["v_pages"].view(torch.int8)), stream=0)
    assert reached[2:] == ["vq_cache_append"]


# --------------------------------------------------------------------------------------------- the pool
def _copy(desc, buffers, pairs, stream=None):
    for b in buffers:
        for x, y in pairs:
            b[y] = b[x].clone()


@pytest.fixture
def pool(monkeypatch):
    monkeypatch.setattr(vc, "vq_cache_copy", _copy)
    return lambda pages=20, width=9: vc.PagedCache(1, 2, 1, 64, 16, pages, width, device="cpu")


def test_buffers_in_8_bits():
    c = vc.PagedCache(3, 8, 2, 64, 32, 7, 4, device="cpu", cache_dtype=vq.VQ_E4M3)
    assert len(c.k) == len(c.v) == 3 and all(b.dtype == torch.uint8 and b.nbytes == vq.vq_cache_bytes(c.desc) for b in c.k + c.v)
    for bad in (0, vq.VQ_F16, vq.VQ_I8):
        with pytest.raises(ValueError):
            vc.PagedCache(1, 2, 1, 64, 16, 5, 2, device="cpu", cache_dtype=bad)


def test_pages_behind_the_window_are_given_back(pool):
    c = pool()
    a = c.add()
    c.grow([a], [100])                                   # pages of tokens 0-15, .. 96-99
    assert c.slide([a], 200) == 0 and c.slide([a], 101) == 0 and c.slide([a], 86) == 0
    assert c.slide([a], 85) == 1 and c.pages(a)[0] == -1  # token 100 sees 16 ..
    assert c.slide([a], 85) == 0
    before = c.free_pages
    assert c.slide([a], 20, sinks=17) == 3               # token 100 sees 81 ..: pages 2, 3 and 4; page 1 holds sink 16
    assert [p >= 0 for p in c.pages(a)] == [False, True, False, False, False, True, True] and c.free_pages == before + 3
    b = c.fork(a)
    assert c.slide([b], 1, sinks=0) == 2                 # of a shared pair: they stay a's
    assert c.free_pages == before + 3
    c.grow([b], [12])
    assert c.slide([b], 1) == 1 and c.pages(b) == [-1] * 7   # all full: the next token sees itself alone
    c.grow([b], [1])
    assert c.pages(b)[:7] == [-1] * 7 and c.pages(b)[7] >= 0
    batch = c.batch([a, b])
    assert batch._keep[1][0].tolist()[:7] == c.pages(a) and batch._keep[0].tolist() == [100, 113]
    c.free(a)
    c.free(b)
    assert c.free_pages == 20 and not any(c._holders)
    for bad in ((0, 0), (-3, 0), (5, -1)):
        with pytest.raises(ValueError):
            c.slide([], *bad)
    d = c.add()
    c.grow([d], [50])
    with pytest.raises(KeyError):
        c.slide([d, 99], 1)
    assert min(c.pages(d)) >= 0                          # nothing has changed


def test_slides_among_everything_else(pool):
    """Random growth, forks, slides, frees and compaction: every token that may still be seen reads what was written."""
    rng = random.Random(4)
    for window, sinks in ((1, 0), (20, 0), (33, 5), (16, 16), (47, 33)):
        c = pool(pages=60)
        want, kept_from = {}, {}
        count = 0
        for step in range(300):
            what = rng.random()
            if what < 0.1 or not want:
                s = c.add()
                want[s], kept_from[s] = [], 0
            elif what < 0.6:
                chosen = rng.sample(sorted(want), rng.randint(1, min(3, len(want))))
                new = [min(rng.randint(0, 25), 9 * 16 - c.length(s)) for s in chosen]
                try:
                    c.grow(chosen, new)
                except vc.OutOfPages:
                    c.free(chosen[0])
                    del want[chosen[0]]
                    continue
                for s, n in zip(chosen, new):
                    for pos in range(c.length(s) - n, c.length(s)):
                        count = (count + 1) % 2000
                        c.k[0][c.pages(s)[pos // 16], :, pos % 16] = count
                        want[s].append(count)
            elif what < 0.7:
                s = rng.choice(sorted(want))
                t = c.fork(s)
                want[t], kept_from[t] = list(want[s]), kept_from[s]
            elif what < 0.9:
                s = rng.choice(sorted(want))
                c.slide([s], window, sinks)
                kept_from[s] = max(kept_from[s], c.length(s) - window + 1)
            elif what < 0.95:
                s = rng.choice(sorted(want))
                c.free(s)
                del want[s]
            else:
                c.compact()
            held = {}
            for s, tokens in want.items():
                assert c.length(s) == len(tokens)
                for pos, x in enumerate(tokens):
                    if pos < sinks or pos >= kept_from[s]:
                        assert float(c.k[0][c.pages(s)[pos // 16], 0, pos % 16, 5]) == x
                for p in c.pages(s):
                    if p >= 0:
                        held[p] = held.get(p, 0) + 1
            assert [c._holders[p] for p in range(c.n_pages)] == [held.get(p, 0) for p in range(c.n_pages)]
            assert sorted(c._free) == [p for p in range(c.n_pages) if p not in held]
