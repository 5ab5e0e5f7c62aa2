"""What the binding of the attention calls takes: tensors of the descriptor's type, on the GPU that the batch's arrays are on, and whole K
and V buffers.  None of these calls gets as far as the library, so no GPU is needed: tensors on a device of their own stand for those on a GPU."""
import pytest
import torch

import paper_2402_15319_amd as vq


class On(torch.Tensor):
    """A tensor that says it is on GPU 0 (or another one)."""
    gpu = 0

    def get_device(self):
        return self.gpu

    def __new__(cls, t):
        return torch.Tensor._make_subclass(cls, t)


class OnOther(On):
    gpu = 1


def _case(dtype=torch.float16, n=4, kind=On):
    d = vq.make_attn_desc(8, 2, 128, 16, 5, vq.VQ_F16 if dtype == torch.float16 else vq.VQ_BF16)
    batch = vq.AttnBatch(kind(torch.ones(n, dtype=torch.int32)), kind(torch.zeros(n, 2, dtype=torch.int32)), max_len=32)
    t = dict(q=torch.zeros(n, 8, 128, dtype=dtype), k_pages=torch.zeros(5, 2, 16, 128, dtype=dtype), v_pages=torch.zeros(5, 2, 128, 16, dtype=dtype),
             out=torch.zeros(n, 8, 128, dtype=dtype), workspace=torch.zeros(1 << 20, dtype=torch.uint8), lse=torch.zeros(n, 8))
    new = dict(k=torch.zeros(n, 2, 128, dtype=dtype), v=torch.zeros(n, 2, 128, dtype=dtype))
    return d, batch, {a: kind(b) for a, b in t.items()}, {a: kind(b) for a, b in new.items()}


@pytest.fixture
def reached(monkeypatch):
    """Stands for the library: what it was called with."""
    calls = []

    class Lib:
        def __getattr__(self, name):
            return lambda *a: calls.append(name) or 0
    monkeypatch.setattr(vq, "lib", Lib)
    return calls


def _attend(d, batch, t, call=vq.vq_attn_decode):
    call(d, batch, t["q"], t["k_pages"], t["v_pages"], t["out"], t["workspace"], lse=t["lse"], stream=0)


def _append(d, batch, t, new):
    vq.vq_cache_append(d, batch, new["k"], new["v"], t["k_pages"], t["v_pages"], stream=0)


@pytest.mark.parametrize("dtype, other", [(torch.float16, torch.bfloat16), (torch.bfloat16, torch.float16)])
def test_other_types_are_refused(reached, dtype, other):
    d, batch, t, new = _case(dtype)
    for call in (vq.vq_attn_decode, vq.vq_attn_prompt):
        _attend(d, batch, t, call)
    _append(d, batch, t, new)
    assert reached == ["vq_attn_decode", "vq_attn_prompt", "vq_cache_append"]
    for name in ("q", "k_pages", "v_pages", "out"):
        for kind in (other, torch.int16):
            for call in (vq.vq_attn_decode, vq.vq_attn_prompt):
                with pytest.raises(ValueError):
                    _attend(d, batch, {**t, name: On(t[name].to(kind))}, call)
    with pytest.raises(ValueError):
        _attend(d, batch, {**t, "lse": On(t["lse"].to(torch.int32))})
    for name in ("k", "v"):
        with pytest.raises(ValueError):
            _append(d, batch, t, {**new, name: On(new[name].to(other))})
    with pytest.raises(ValueError):
        _append(d, batch, {**t, "v_pages": On(t["v_pages"].to(other))}, new)
    assert len(reached) == 3


def test_buffers_that_are_not_whole_are_refused(reached):
    d, batch, t, new = _case()
    for name in ("k_pages", "v_pages"):
        for bad in (t[name][:4], t[name][..., :8], torch.zeros(5, 2, 16, 256, dtype=torch.float16)[..., ::2]):
            with pytest.raises(ValueError):
                _attend(d, batch, {**t, name: On(bad)})
            with pytest.raises(ValueError):
                _append(d, batch, {**t, name: On(bad)}, new)
    assert reached == []
    _attend(d, batch, {**t, "k_pages": On(torch.zeros(7, 2, 16, 128, dtype=torch.float16)), "v_pages": 1 << 20})   # a larger one, an address
    assert len(reached) == 1


def test_tensors_elsewhere_are_refused(reached):
    d, batch, t, new = _case()
    for elsewhere in (lambda x: x.as_subclass(torch.Tensor), OnOther):
        for name in t:
            with pytest.raises(ValueError):
                _attend(d, batch, {**t, name: elsewhere(t[name])})
        for name in new:
            with pytest.raises(ValueError):
                _append(d, batch, t, {**new, name: elsewhere(new[name])})
        for name in ("k_pages", "v_pages"):
            with pytest.raises(ValueError):
                _append(d, batch, {**t, name: elsewhere(t[name])}, new)
    d, batch, t, new = _case(kind=lambda x: x)     # all of it on the host
    with pytest.raises(ValueError):
        _attend(d, batch, t)
    with pytest.raises(ValueError):
        _append(d, batch, t, new)
    lens, table = torch.ones(4, dtype=torch.int32), torch.zeros(4, 2, dtype=torch.int32)
    with pytest.raises(ValueError):
        vq.AttnBatch(On(lens), OnOther(table), max_len=32)
    with pytest.raises(ValueError):
        vq.AttnBatch(lens, table, n_tokens=4, max_len=32, q_start=On(torch.zeros(5, dtype=torch.int32)))
    assert reached == []
