"""Attention over the paged cache without a GPU: what the entry points refuse, sizes, and the binding's own checks."""
import ctypes

import pytest

import paper_2402_15319_amd as vq

A = 0x10000   # a fake, aligned address: validation fails before any launch
OK, NULL, DESC, UNSUPPORTED, ALIGN, ARG = 0, -1, -2, -3, -4, -6


def _desc(**change):
    d = dict(heads=8, kv_heads=2, head_dim=128, page_size=16, n_pages=100, dtype=vq.VQ_F16, scale=0.1)
    d.update(change)
    reserved = d.pop("reserved", 0)
    x = vq.make_attn_desc(**d)
    x.reserved = reserved
    return x


def _batch(**change):
    b = dict(n_seqs=4, n_tokens=4, table_width=10, max_len=160, q_start=A, kv_len=A, page_table=A)
    b.update(change)
    return vq.VQAttnBatch(*b.values())


def _attn(name, desc, batch, q=A, qs=None, k=2 * A, v=3 * A, out=4 * A, os=None, lse=5 * A, ws=6 * A, n=1 << 40):
    return getattr(vq.lib(), name)(desc, batch, q, qs, k, v, out, os, lse, ws, n, 0)


def _all(desc, batch):
    """Statuses of the entry points that take a descriptor and a batch."""
    size = ctypes.c_size_t()
    L = vq.lib()
    return [_attn("vq_attn_decode", desc, batch), _attn("vq_attn_prompt", desc, batch),
            L.vq_cache_append(desc, batch, A, None, 2 * A, None, 3 * A, 4 * A, 0), L.vq_attn_workspace_bytes(desc, batch, ctypes.byref(size))]


@pytest.mark.parametrize("change, status", [
    (dict(heads=0), DESC), (dict(kv_heads=0), DESC), (dict(heads=9), DESC), (dict(kv_heads=-2), DESC), (dict(n_pages=0), DESC),
    (dict(page_size=0), DESC), (dict(head_dim=-128), DESC), (dict(reserved=1), DESC),
    (dict(head_dim=80), UNSUPPORTED), (dict(head_dim=512), UNSUPPORTED), (dict(page_size=24), UNSUPPORTED), (dict(page_size=8), UNSUPPORTED),
    (dict(page_size=256), UNSUPPORTED), (dict(dtype=vq.VQ_F32), UNSUPPORTED), (dict(dtype=vq.VQ_I8), UNSUPPORTED), (dict(heads=2048, kv_heads=1), UNSUPPORTED),
])
def test_bad_descriptors(change, status):
    d = _desc(**change)
    assert _all(d, _batch()) == [status] * 4
    size = ctypes.c_size_t()
    assert vq.lib().vq_cache_bytes(d, ctypes.byref(size)) == status
    assert vq.lib().vq_cache_copy(d, 1, (ctypes.c_void_p * 1)(A), 1, (ctypes.c_int32 * 2)(0, 1), 0) == status


@pytest.mark.parametrize("scale", [0.0, -1.0, float("nan"), float("inf")])
def test_bad_scales(scale):
    for name in ("vq_attn_decode", "vq_attn_prompt"):
        assert _attn(name, _desc(scale=scale), _batch()) == ARG


@pytest.mark.parametrize("change", [dict(n_seqs=0), dict(n_seqs=65536), dict(n_tokens=0), dict(table_width=0), dict(max_len=-1), dict(max_len=161),
                                    dict(max_len=2 ** 29 + 1, table_width=2 ** 27)])
def test_bad_batches(change):
    assert _all(_desc(), _batch(**change)) == [ARG] * 4


def test_other_bad_batches():
    d = _desc()
    assert _attn("vq_attn_decode", d, _batch(n_tokens=5)) == ARG                      # one new token a sequence
    assert _attn("vq_attn_prompt", d, _batch(n_tokens=5, q_start=None)) == ARG
    for name in ("vq_attn_decode", "vq_attn_prompt"):
        for what in ("kv_len", "page_table"):
            assert _attn(name, d, _batch(**{what: None})) == NULL
            assert _attn(name, d, _batch(**{what: A + 2})) == ALIGN
        assert _attn(name, d, None) == NULL and _attn(name, None, _batch()) == NULL


@pytest.mark.parametrize("name", ["vq_attn_decode", "vq_attn_prompt"])
def test_bad_pointers(name):
    d, b = _desc(), _batch()
    for what in ("q", "k", "v", "out", "ws"):
        assert _attn(name, d, b, **{what: None}) == NULL
        assert _attn(name, d, b, **{what: A + 8}) == ALIGN
    assert _attn(name, d, b, lse=A + 2) == ALIGN
    for same in ("q", "k", "v"):
        assert _attn(name, d, b, **{same: 4 * A}) == ARG      # the output
    assert _attn(name, d, b, n=0) == ARG                      # a workspace that is too small


S = vq.VQStrides


@pytest.mark.parametrize("strides, input_too", [
    (S(-1024, 128, 1), True), (S(1024, -128, 1), True), (S(1024, 128, 0), True), (S(1024, 128, -1), True),
    (S(1 << 60, 128, 1), True), (S(1024, 1 << 60, 1), True), (S(1, 8, 1 << 62), True),
    (S(0, 128, 1), False), (S(1024, 0, 1), False), (S(1024, 64, 1), False), (S(1000, 128, 1), False), (S(1, 128 * 3, 3), False),
])
def test_strides_that_are_refused(strides, input_too):
    """Negative or far too large ones everywhere, elements that share a place in an output."""
    for name in ("vq_attn_decode", "vq_attn_prompt"):
        assert _attn(name, _desc(), _batch(), os=strides) == ARG
        if input_too:
            assert _attn(name, _desc(), _batch(), qs=strides) == ARG
    if input_too:
        assert vq.lib().vq_cache_append(_desc(), _batch(), A, strides, 2 * A, None, 3 * A, 4 * A, 0) == ARG
        assert vq.lib().vq_cache_append(_desc(), _batch(), A, None, 2 * A, strides, 3 * A, 4 * A, 0) == ARG


def test_append_refusals():
    d, b, L = _desc(), _batch(), vq.lib()
    good = [A, 2 * A, 3 * A, 4 * A]
    for i in range(4):
        for bad, status in ((None, NULL), (A + 2, ALIGN)):
            p = list(good)
            p[i] = bad
            assert L.vq_cache_append(d, b, p[0], None, p[1], None, p[2], p[3], 0) == status
    assert L.vq_cache_append(d, b, A, None, 2 * A, None, 3 * A, 3 * A, 0) == ARG
    assert L.vq_cache_append(d, b, A, None, 2 * A, None, A, 3 * A, 0) == ARG
    assert L.vq_cache_append(d, b, A, None, 2 * A, None, 3 * A, 2 * A, 0) == ARG


def test_copy_refusals():
    d, L = _desc(), vq.lib()
    buffers, pairs = (ctypes.c_void_p * 2)(A, 2 * A), (ctypes.c_int32 * 4)(0, 1, 2, 3)
    assert L.vq_cache_copy(d, 0, buffers, 2, pairs, 0) == ARG and L.vq_cache_copy(d, 65537, buffers, 2, pairs, 0) == ARG
    assert L.vq_cache_copy(d, 2, buffers, 0, pairs, 0) == ARG and L.vq_cache_copy(d, 2, buffers, -1, pairs, 0) == ARG
    assert L.vq_cache_copy(d, 2, None, 2, pairs, 0) == NULL and L.vq_cache_copy(d, 2, buffers, 2, None, 0) == NULL
    assert L.vq_cache_copy(d, 2, (ctypes.c_void_p * 2)(A, None), 2, pairs, 0) == NULL
    assert L.vq_cache_copy(d, 2, (ctypes.c_void_p * 2)(A, A + 8), 2, pairs, 0) == ALIGN
    for bad in (-1, 100, 2 ** 31 - 1):
        for at in range(4):
            p = (ctypes.c_int32 * 4)(0, 1, 2, 3)
            p[at] = bad
            assert L.vq_cache_copy(d, 2, buffers, 2, p, 0) == ARG
    assert L.vq_cache_copy(d, 2, buffers, 2, (ctypes.c_int32 * 4)(7, 7, 9, 9), 0) == OK    # onto themselves: nothing is launched


def test_sizes():
    d = _desc()
    assert vq.vq_cache_bytes(d) == 100 * 2 * 16 * 128 * 2
    assert vq.vq_cache_bytes(_desc(n_pages=2 ** 31 - 1)) == (2 ** 31 - 1) * 8192
    assert vq.lib().vq_cache_bytes(d, None) == NULL and vq.lib().vq_attn_workspace_bytes(d, _batch(), None) == NULL
    assert ctypes.sizeof(vq.VQAttnDesc) == 32 and ctypes.sizeof(vq.VQAttnBatch) == 40 and ctypes.sizeof(vq.VQStrides) == 24


def test_weight_products_do_not_take_the_attention_type():
    d = vq.make_desc(4096, 4096, 16, 4, codebook_dtype=vq.VQ_BF16)
    assert vq.lib().vq_gemv(ctypes.byref(d), A, A, A, 2 * A, vq.VQ_F16, 0) == UNSUPPORTED
    d = vq.make_desc(4096, 4096, 16, 4)
    assert vq.lib().vq_gemv(ctypes.byref(d), A, A, A, 2 * A, vq.VQ_BF16, 0) == ARG


def test_the_binding_checks_shapes_and_types():
    import torch
    d = _desc()
    lens, table = torch.zeros(4, dtype=torch.int32), torch.zeros(4, 10, dtype=torch.int32)
    batch = vq.AttnBatch(lens, table, max_len=160)
    assert (batch.struct.n_seqs, batch.struct.n_tokens, batch.struct.table_width, batch.struct.q_start) == (4, 4, 10, None)
    assert vq.AttnBatch(lens, table, page_size=16).struct.max_len == 160
    for bad in (dict(kv_len=lens.long()), dict(kv_len=lens[:3]), dict(page_table=table[:, ::2]), dict(page_table=table[0]),
                dict(q_start=torch.zeros(4, dtype=torch.int32)), dict(max_len=None), dict(q_start=torch.zeros(5, dtype=torch.int32))):
        with pytest.raises(ValueError):
            vq.AttnBatch(**{"kv_len": lens, "page_table": table, "max_len": 160, **bad})
    q = torch.zeros(4, 8, 128, dtype=torch.float16)
    kp = torch.zeros(16)
    for bad in (q[:3], q[:, :7], q[..., :64], q.float(), q[0]):
        with pytest.raises(ValueError):
            vq.vq_attn_decode(d, batch, bad, kp, kp, q, kp, stream=0)
        with pytest.raises(ValueError):
            vq.vq_attn_prompt(d, batch, q, kp, kp, bad, kp, stream=0)
        with pytest.raises(ValueError):
            vq.vq_cache_append(d, batch, bad, q[:, :2], kp, kp, stream=0)
    for bad in (torch.zeros(4, 7), torch.zeros(8, 4).T, torch.zeros(4, 8, dtype=torch.float16)):
        with pytest.raises(ValueError):
            vq.vq_attn_decode(d, batch, q, kp, kp, q, kp, lse=bad, stream=0)
    with pytest.raises(ValueError):
        vq.vq_cache_copy(d, [kp], [(1, 2, 3)], stream=0)
