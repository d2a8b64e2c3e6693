"""Operators around a block: what lies past a limit is refused, and what lies just before it is not (no GPU needed)."""
import pytest

from paper_2505_00315_amd import mosa, ops


@pytest.mark.parametrize("scale", [2.36e38, 3e38, 3.4028234e38])
def test_scales_past_the_exponents(scale):
    """A scale whose product with log2(e) passes fp32 would make every exponent NaN."""
    with pytest.raises(mosa.MosaError) as e:
        ops.logprob_scratch_size(ops.make_logprob_shape(2, 1000, scale=scale))
    assert e.value.status == mosa.MOSA_ERR_UNSUPPORTED


@pytest.mark.parametrize("scale", [2.35e38, 1e30, 1.0, 1e-45])
def test_scales_that_are_taken(scale):
    ops.logprob_scratch_size(ops.make_logprob_shape(2, 1000, scale=scale))
