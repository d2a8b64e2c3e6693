"""The weights' gradients of norm and rotation: sums over all rows, rounded once (fp32 storage)."""
import pytest
import torch

from ops_util import HALF, within
from paper_2505_00315_amd import ops

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("B,T,Hq,Hkv", [(1, 3, 2, 1), (2, 777, 4, 4), (3, 2500, 6, 2)])
def test_sums_over_rows_are_rounded_once(B, T, Hq, Hkv, dh):
    """Rows of +-1 are their own norm, so every product is a gradient's value: multiples of 2^-10 of at most 2^23, which
    64 bits add up exactly in any order.  The two largest cancel, and what is left has half a step of its own size."""
    g = torch.Generator().manual_seed(1)
    shape = ops.make_norm_shape(B, T, Hq, Hkv, dh, "f32", rope_dim=0, eps=0.0)
    x, d = {}, {}
    for n, H in (("q", Hq), ("k", Hkv)):
        x[n] = (2.0 * torch.randint(0, 2, (B, H, T, dh), generator=g) - 1).cuda()
        d[n] = (torch.randint(-4096, 4097, (B, H, T, dh), generator=g) / 1024.0).cuda()
        d[n][0, 0, 0] = 2.0 ** 23 * x[n][0, 0, 0]
        d[n][B - 1, H - 1, T - 1] = -2.0 ** 23 * x[n][B - 1, H - 1, T - 1]
    one = torch.ones(dh, device="cuda")
    dq, dk, dwq, dwk = ops.qk_norm_rope_backward(shape, x["q"], x["k"], one, one, d["q"], d["k"])
    for n, got in (("q", dwq), ("k", dwk)):
        want = (d[n].double() * x[n].double()).sum((0, 1, 2))
        within(got, want, HALF[torch.float32] * want.abs(), n)
