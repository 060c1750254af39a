"""Attention with a relative position bias: how large a scale its entry points take (no GPU needed: the calls are refused)."""
import pytest

from test_rel_attention_host import BAD, _call


@pytest.mark.parametrize("back", [False, True])
def test_scales_whose_product_with_log2_e_is_infinite_are_refused(back):
    """The kernels multiply scores by scale * log2(e) in fp32: where that is infinite a score of 0 would be NaN."""
    for scale in (2.37e38, 3e38, 3.4028234e38):
        assert _call(back, scale=scale) == BAD, scale
