"""What the binding of the attention calls does on the host (no GPU needed): its own Python calls and the descriptor's fields that it reads for each, every one a
tenth of a microsecond or less of calls that take six."""
import collections
import sys

import pytest

import paper_2402_15319_amd as vq
from test_attn_binding import _append, _attend, _case, reached  # noqa: F401


def _on_the_host(f, *args):
    """({Python function of the binding: calls}, fields of the descriptor that are read)"""
    calls, fields = collections.Counter(), 0

    class Desc(vq.VQAttnDesc):
        def __getattribute__(self, name):
            nonlocal fields
            fields += name in {n for n, _ in vq.VQAttnDesc._fields_}
            return super().__getattribute__(name)
    desc = Desc(*(getattr(args[0], n) for n, _ in vq.VQAttnDesc._fields_))

    def look(frame, event, _):
        if event == "call" and frame.f_code.co_filename == vq.__file__:
            calls[frame.f_code.co_name] += 1
    sys.setprofile(look)
    try:
        f(desc, *args[1:])
    finally:
        sys.setprofile(None)
    return calls, fields


@pytest.mark.parametrize("call", [vq.vq_attn_decode, vq.vq_attn_prompt])
def test_attention(reached, call):  # noqa: F811
    d, batch, t, _ = _case()
    calls, fields = _on_the_host(_attend, d, batch, t, call)
    assert calls == {call.__name__: 1, "_attn": 1, "_rows": 2, "_pages": 2, "_ptr": 2, "_stream": 1, "_check": 1}
    assert fields == 7   # all but the scale, once


def test_append(reached):  # noqa: F811
    d, batch, t, new = _case()
    calls, fields = _on_the_host(_append, d, batch, t, new)
    assert calls == {"vq_cache_append": 1, "_rows": 2, "_pages": 2, "_stream": 1, "_check": 1}
    assert fields == 6   # nor the query heads
