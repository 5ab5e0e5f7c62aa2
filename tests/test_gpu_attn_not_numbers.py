"""Attended values that are no numbers, behind weights too small for the type that the weights are rounded to: such a weight is not
zero, so an infinite value gives an infinite output (one of each sign: NaN), as the formula says.  A logit of -infinity is a weight
of zero, and zero times infinity is NaN.  Rows and heads that do not attend the token stay as they were."""
import numpy as np
import pytest

from attn_cases import Problem, run

pytestmark = pytest.mark.gpu

# (call, heads, kv, lens, new): one part and several (joined by few and by many threads), waves with and without tokens, tiles that share
# a workgroup; prompts with one team and with two, whole and in parts, masked steps and others
SHAPES = [("decode", 4, 2, [150, 71], None), ("decode", 2, 1, [9, 200], None), ("decode", 4, 2, [3000, 71], None), ("decode", 2, 1, [30001], None),
          ("decode", 48, 1, [130, 71] * 8, None), ("decode", 20, 1, [1400, 100] * 8, None),
          ("prompt", 4, 2, [150, 71], [100, 20]), ("prompt", 4, 2, [700], [700]), ("prompt", 4, 1, [5000], [7]), ("prompt", 32, 32, [330], [330]),
          ("prompt", 6, 2, [1500, 90], [130, 90])]


def _problem(call, heads, kv, lens, new, dim, dtype, falls, rise):
    """Every query has 1 / scale in dimension 0, so a key's dimension 0 is a term of its logit.  falls: that term and the value of
    some tokens; rise: the term of a later token, or None.  Returns the problem and, for each
    sequence, where the values that are no numbers are: (token, dimension, value, logit -infinity)."""
    import torch
    p = Problem(heads, kv, dim, 16, dtype, lens, new, seed=dim + len(lens))
    p.q_host[:, :, 0] = 1.0 / p.scale
    p.k_host[..., 0] = torch.where(torch.isfinite(p.k_host[..., 0]), torch.zeros_like(p.k_host[..., 0]), p.k_host[..., 0])
    odd = {}
    for i, (term, value) in enumerate(falls):
        for s, n in enumerate(lens):
            at = (5 + 11 * i) % n if i % 2 else max(0, n - 3 - 7 * i) % n     # early and late tokens
            where = int(p.table[s, at // 16]), at % 16
            p.k_host[where[0], kv - 1, where[1], 0] = term
            p.v_host[where[0], kv - 1, 3 + i // 2, where[1]] = value
            if not np.isfinite(value):
                odd.setdefault(s, []).append((at, 3 + i // 2, value, term == -np.inf))
    if rise is not None:
        for s, n in enumerate(lens):
            taken = {o[0] for o in odd[s]}
            at = next(t for t in range(2 * n // 3, n) if t not in taken)
            p.k_host[int(p.table[s, at // 16]), kv - 1, at % 16, 0] = rise
    p.k_pages, p.v_pages, p.q = p.k_host.to(p.dev), p.v_host.to(p.dev), p.rows(p.q_host, p.heads)
    return p, odd


def _expected(p, odd):
    """The definition: finite values by the oracle, then what the others make of every row that attends them."""
    v = p.v_host.clone()
    for s, marks in odd.items():
        for at, d, _, _ in marks:
            p.v_host[int(p.table[s, at // 16]), p.kv - 1, d, at % 16] = 0
    ref = p.reference()
    p.v_host = v
    out = ref[0].copy()
    with np.errstate(invalid="ignore"):
        for s, marks in odd.items():
            for t in range(p.q_start[s], p.q_start[s + 1]):
                pos = p.lens[s] - p.q_start[s + 1] + t
                for at, d, value, none in marks:
                    if at <= pos:
                        out[t, p.heads - p.heads // p.kv:, d] += np.nan if none else value
    return ref, out


@pytest.mark.parametrize("shape, dim, dtype", [(s, *t) for i, s in enumerate(SHAPES) for t in ((128, "f16"), (64, "bf16"), (96, "f16"), (256, "bf16"))
                                               if t[0] in (64, 128) or i in (0, 2, 6, 8)], ids=lambda x: "-".join(map(str, x[:4])).replace(" ", "") if isinstance(x, tuple) else str(x))
@pytest.mark.parametrize("falls, rise", [
    ([(-30.0, np.inf), (-30.0, np.inf), (-40.0, -np.inf)], None),                       # below the smallest weight of fp16
    ([(-200.0, np.inf), (-150.0, -np.inf), (-300.0, np.nan)], None),                    # below the smallest of fp32
    ([(0.0, np.inf), (-1.0, -np.inf), (0.0, -np.inf)], 250.0),                          # first a weight of one, then next to none
    ([(-np.inf, np.inf), (-60.0, 1.0), (-60.0, -np.inf)], None),                        # no weight at all
], ids=["small", "smaller", "rise", "none"])
def test_infinite_values_with_next_to_no_weight(shape, dim, dtype, falls, rise):
    p, odd = _problem(*shape, dim, dtype, falls, rise)
    out, _ = run(p, shape[0])
    ref, want = _expected(p, odd)
    got = out.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(np.isposinf(got), np.isposinf(want)) and np.array_equal(np.isneginf(got), np.isneginf(want))
    b_out, _ = p.bounds(ref)
    with np.errstate(invalid="ignore"):
        over = (np.abs(got - want) > b_out) & np.isfinite(want)
    assert not over.any()


@pytest.mark.parametrize("call, lens, new", [("decode", [700] * 128, None), ("decode", [700], None), ("prompt", [300], [300]), ("prompt", [3000], [5])])
def test_sums_beyond_the_range_stay_visible(call, lens, new):
    """Values close to bf16's largest: their sum is infinite, and no number once a later token leaves it next to no weight.  Neither
    may come out as a finite value made up for it."""
    p = Problem(4, 2, 64, 16, "bf16", lens, new, seed=1)
    p.q_host[:, :, 0] = 1.0 / p.scale
    rise = lens[0] - 100
    for t in range(lens[0]):
        pages, slot = p.table[:, t // 16], t % 16
        p.k_host[pages, :, slot, 0] = 250.0 if t == rise else 0.0
        p.v_host[pages, 1, 3, slot] = 3.3e38 if t < 100 else 1.0
    p.k_pages, p.v_pages, p.q = p.k_host.to(p.dev), p.v_host.to(p.dev), p.rows(p.q_host, p.heads)
    out, _ = run(p, call)
    got = out.double().cpu().numpy()
    above = got[-1, 2:, 3]
    assert (~np.isfinite(above) | (np.abs(above - 1.0) < 0.02)).all(), above
    finite = np.delete(got, 3, axis=2)
    assert np.isfinite(finite).all()
