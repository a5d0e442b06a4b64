"""Calls of the 8-bit cache's operators that their results could not be right for, without a GPU: refused, nothing launched."""
import pytest

from tests.test_kv8_plan import _call


@pytest.mark.parametrize("scale", [2.4e38, 3.4e38])
def test_scales_that_overflow_as_the_kernels_take_them(scale):
    """scale * log2(e) beyond fp32: scores of zero would become NaN."""
    from paper_2602_16603_amd import binding as B
    with pytest.raises(B.FlowPrefillError) as e:
        _call("attention", scale=scale)
    assert e.value.status == B.FP_ERR_INVALID and "scale" in str(e.value)


def test_the_largest_scale_is_taken():
    _call("attention", scale=2.3e38, n_tokens=0)
