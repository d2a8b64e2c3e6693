"""Extents of rows are limited in bytes, whatever the type (no GPU needed)."""
import pytest

from paper_2505_00315_amd import ops
from test_ops_refusals import INV, rows, status


@pytest.mark.parametrize("dtype,stride", [("f32", (1 << 27) + 4), ("bf16", (1 << 28) + 8)])
def test_rows_over_more_than_2_46_bytes(dtype, stride):
    T = (1 << 17) + 1
    s = ops.make_norm_shape(1, T, 1, 1, 64, dtype)
    k, far = rows(1, 1, T, 64), rows(1, 1, T, 64, row_stride=stride)
    for at in range(4):
        assert status("mosa_qk_norm_rope", s, *[far if i == at else k for i in range(2)], None, None, None,
                      *[far if i == at - 2 else k for i in range(2)], None) == INV
