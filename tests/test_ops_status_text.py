"""A refusal of an operator names the operators' limits, not the layer's alone (no GPU needed)."""
import pytest

from paper_2505_00315_amd import mosa, ops


def test_unsupported_head_size_names_the_sizes_there_are():
    with pytest.raises(mosa.MosaError, match="d_head 32, 64 or 128"):
        ops.attn_scratch_size(ops.make_attn_shape(1, 1, 1, 1, 1, 96))


def test_small_scratch_is_not_called_the_layers_workspace():
    with pytest.raises(mosa.MosaError) as e:
        mosa._check(mosa.MOSA_ERR_WORKSPACE, "mosa_window_attention")
    assert "size function" in str(e.value)
