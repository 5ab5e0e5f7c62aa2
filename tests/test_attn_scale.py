"""Scales that the kernels cannot hold: they work with powers of two, on scale * log2(e)."""
import pytest

from test_attn_abi import ARG, NULL, _attn, _desc


@pytest.mark.parametrize("scale", [2.4e38, 3.0e38, 3.4028234e38])
def test_scales_whose_product_with_log2_e_is_infinite(scale):
    """Infinity times a logit of 0 would be NaN."""
    for name in ("vq_attn_decode", "vq_attn_prompt"):
        assert _scale_is_refused(name, scale)
        assert not _scale_is_refused(name, 2.3e38) and not _scale_is_refused(name, 1e-38)


def _scale_is_refused(name, scale):
    """The batch is looked at next, and there is none: nothing is launched."""
    status = _attn(name, _desc(scale=scale), None)
    assert status in (ARG, NULL)
    return status == ARG
