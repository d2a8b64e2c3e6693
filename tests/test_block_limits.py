"""Operators around a block: what lies past a limit is refused, and what lies just before it is not (no GPU needed)."""
import pytest

from paper_2505_00315_amd import mosa, ops
from test_block_refusals import A, INV, linear_back, mat, status


@pytest.mark.parametrize("scale", [2.36e38, 3e38, 3.4028234e38])
def test_scales_past_the_exponents(scale):
    """A scale whose product with log2(e) passes fp32 would make every exponent NaN."""
    with pytest.raises(mosa.MosaError) as e:
        ops.logprob_scratch_size(ops.make_logprob_shape(2, 1000, scale=scale))
    assert e.value.status == mosa.MOSA_ERR_UNSUPPORTED


@pytest.mark.parametrize("scale", [2.35e38, 1e30, 1.0, 1e-45])
def test_scales_that_are_taken(scale):
    ops.logprob_scratch_size(ops.make_logprob_shape(2, 1000, scale=scale))


def test_product_gradients_need_what_they_read():
    """x is read for dw, w for dx; one that is given is checked, read or not."""
    assert status(*linear_back(x=None, dx=None)) == INV and status(*linear_back(w=None, dw=None)) == INV
    bad = mat(64, A + 40)
    assert status(*linear_back(x=bad, dw=None)) == INV and status(*linear_back(w=bad, dx=None)) == INV
