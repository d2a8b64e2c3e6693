"""Operators around a block: values and calls at the edges of what they allow."""
import math

import pytest
import torch

from block_util import U32, logprobs64, slope64, within
from paper_2505_00315_amd import mosa, ops
from test_gpu_block_linear import make as make_linear
from test_gpu_block_logprob import check as check_logprobs
from test_gpu_block_residual import check as check_stream
from test_gpu_block_residual import make as make_stream

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
# NaN whose first bit of the fraction is 0, as no arithmetic makes them
SIGNALING = {"bf16": (torch.int16, 0x7F81), "f32": (torch.int32, 0x7F800001)}


def signaling(x, dtype, at):
    """Signaling NaN in x at these indices of its flat values (set as bits: a copy of values may quiet them)."""
    kind, bits = SIGNALING[dtype]
    x.view(kind).view(-1)[torch.as_tensor(at, device=x.device)] = bits


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,V", [(9, 12), (9, 700), (9, 3000), (9, 40001), (9, 140002), (300, 3000), (300, 66003), (1100, 12),
                                 (1100, 700), (1100, 9001)])
def test_signaling_nan(R, V, dtype):
    """A row with a signaling NaN is NaN throughout and its alternatives are in order, NaN as -inf, wherever in the row
    the NaN lies and whatever the lane that meets it has seen before."""
    g = torch.Generator().manual_seed(V)
    x = (torch.randn(R, V, generator=g) * 3).to(DT[dtype]).cuda()
    x[0] = -torch.arange(V) / 64  # falling: every lane's largest value is its first
    x[1] = torch.arange(V) / 64
    most = [0, V // 2, V - 1, min(V - 1, 7), min(V - 1, 3), V // 3]
    for r in range(min(R, 8)):
        at = {0: [0], 1: [V - 1], 2: most, 3: list(range(0, V, 2)), 4: list(range(7, V, 8)), 5: [],
              6: list(range(V)), 7: most[1:2]}[r]
        if at:
            signaling(x, dtype, [r * V + i for i in at])
    for r in range(8, R):
        signaling(x, dtype, [r * V + int(i) for i in torch.randint(0, V, (3,), generator=g)])
    assert bool(torch.isnan(x[4:5, 7::8]).all()) and not bool(torch.isnan(x[5]).any())
    top = min(V, 8)
    shape = ops.make_logprob_shape(R, V, dtype, top=top)
    t = torch.randint(0, V, (R,), generator=g, dtype=torch.int32).cuda()
    stats, ent = torch.empty(R, 2, device="cuda"), torch.empty(R, device="cuda")
    ones = torch.ones(R, device="cuda")
    # (the 64-bit form's conversion quiets NaN)
    want = logprobs64(x, t, 1.0, top, d_logp=ones, d_entropy=ones)
    logp, lse, top_logp, top_index = ops.token_logprobs(shape, x, t, stats=stats, entropy=ent)
    for name, got in (("logp", logp), ("lse", lse), ("entropy", ent), ("top_logp", top_logp)):
        within(got, *want[name], name)
    assert torch.equal(top_index.long(), want["top_index"])
    dx = ops.token_logprobs_backward(shape, x, t, stats, entropy=ent, d_logp=ones, d_entropy=ones)
    within(dx, *want["dx"], "gradient")


@pytest.mark.parametrize("V", [60, 3001, 20001, 140002])
@pytest.mark.parametrize("scale", [1.0, 0.3])
@pytest.mark.parametrize("spread", [0.5, 40.0])
def test_bases_at_their_limit(spread, scale, V):
    """Rows whose largest exponent, in log2 units, lies just below, across and just above 2^20 (of either sign), with
    weights of one size in all lanes and other maxima in each: the roundings of the lanes' bases, up to 2^-5 here,
    leave the sums, whichever bases they are brought to."""
    at = 2.0 ** 20 * math.log(2.0) / scale
    g = torch.Generator().manual_seed(V)
    shift = torch.tensor([at * f for f in (0.9, 0.999, 1.0, 1.001, 1.1, -0.9, -1.0, -1.1, 0.6)])
    x = (torch.randn(9, V, generator=g) * spread + shift[:, None]).cuda()
    t = torch.randint(0, V, (9,), generator=g, dtype=torch.int32).cuda()
    check_logprobs(x, t, scale=scale, top=min(V, 5))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_extreme_scales(dtype):
    """The largest scale that is taken, and one below the normal numbers."""
    x = torch.zeros(4, 3000, dtype=DT[dtype], device="cuda")
    x[1, 7] = 1.0
    x[2] = torch.linspace(-1.0, 1.0, 3000).to(DT[dtype])
    x[3] = (torch.arange(3000) % 7 * 2.0 ** -126).to(DT[dtype])
    t = torch.tensor([0, 7, 2999, 6], dtype=torch.int32, device="cuda")
    check_logprobs(x, t, scale=1e-40, top=3)
    shape = ops.make_logprob_shape(4, 3000, dtype, top=3, scale=2.35e38)
    want = logprobs64(x, t, shape.scale, 3)
    ent = torch.empty(4, device="cuda")
    logp, lse, top_logp, top_index = ops.token_logprobs(shape, x, t, entropy=ent)
    assert torch.equal(top_index.long(), want["top_index"])
    for name, got in (("logp", logp), ("lse", lse), ("entropy", ent), ("top_logp", top_logp)):
        ref, bound = want[name]
        if "logp" in name:
            # The form's bound takes differences z - m up to 1e30 only (masked places are infinitely far).  Here they are up
            # to 4.7e38 in 32 bits: a difference, a product and a difference, each off by 2^-24 of itself at most, so 3 2^-24
            # (1.8e-7) of a log p that is all but z - m.
            bound = bound + 3 * 2.0 ** -24 * ref.abs().clamp(max=1e39)
        within(got, ref, bound, name)


@pytest.mark.parametrize("order", ["in_out", "out_in"])
@pytest.mark.parametrize("M", [3, 200])
def test_product_gradients_without_what_they_do_not_read(M, order):
    """dx needs no x (a frozen weight's product keeps no activations), dw no w, db neither; a missing one that is
    read is refused."""
    shape = ops.make_linear_shape(M, 136, 264, act="gelu", w_order=order)
    t = make_linear(21, M, 136, 264, "bf16", order)
    z = torch.empty_like(t["dy"])
    ops.linear(shape, t["x"], t["w"], bias=t["bias"], z=z)
    every = ops.linear_backward(shape, t["x"], t["w"], t["dy"], z=z, grads="xwb")
    for grads, x, w in (("x", None, t["w"]), ("xb", None, t["w"]), ("w", t["x"], None), ("wb", t["x"], None),
                        ("b", None, None)):
        got = ops.linear_backward(shape, x, w, t["dy"], z=z, grads=grads)
        for letter, a, b in zip("xwb", got, every):
            assert (a is None) if letter not in grads else torch.equal(a, b)
    for grads, x, w in (("w", None, t["w"]), ("xw", None, t["w"]), ("x", t["x"], None), ("xb", None, None)):
        with pytest.raises(mosa.MosaError) as e:
            ops.linear_backward(shape, x, w, t["dy"], z=z, grads=grads)
        assert e.value.status == mosa.MOSA_ERR_INVALID_ARG


def padded(rows, cols, dtype):
    """A store of 7s and its middle [rows, cols], and whether what is around the middle is as it was."""
    store = torch.full((rows + 2, cols + 16), 7.0, dtype=dtype, device="cuda")
    around = torch.ones_like(store, dtype=torch.bool)
    around[1:rows + 1, 8:cols + 8] = False
    return store[1:rows + 1, 8:cols + 8], lambda: bool((store[around] == 7.0).all())


@pytest.mark.parametrize("order", ["in_out", "out_in"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M", [1, 3, 9, 70, 400, 2100])
def test_product_gradients_keep_to_themselves(M, dtype, order):
    """NaN in a row of dy or of z reaches that row of dx only, and infinities there too; dw and db are NaN in that
    column; memory around z, dx, dw and y stays as it is."""
    K, N = 328, 456
    shape = ops.make_linear_shape(M, K, N, dtype, act="silu", w_order=order)
    t = make_linear(22, M, K, N, dtype, order)
    (y, y_ok), (z, z_ok), (dx, dx_ok), (dw, dw_ok) = (padded(*s, DT[dtype]) for s in ((M, N), (M, N), (M, K), t["w"].shape))
    plain = torch.empty_like(t["dy"])
    want_y = ops.linear(shape, t["x"], t["w"], bias=t["bias"], z=plain)
    want = ops.linear_backward(shape, t["x"], t["w"], t["dy"], z=plain, grads="xwb")
    ops.linear(shape, t["x"], t["w"], bias=t["bias"], y=y, z=z)
    assert torch.equal(y, want_y) and torch.equal(z, plain)
    db = torch.empty_like(want[2])
    ops.linear_backward(shape, t["x"], t["w"], t["dy"], z=z, grads="xwb", dx=dx, dw=dw, db=db)
    assert torch.equal(dx, want[0]) and torch.equal(dw, want[1]) and torch.equal(db, want[2])
    r, col = M // 2, 5
    others = torch.arange(M, device="cuda") != r
    rest = torch.arange(N, device="cuda") != col
    for what, bad in (("dy", float("nan")), ("z", float("nan")), ("dy", float("inf"))):
        d = {"dy": t["dy"].clone(), "z": plain.clone()}
        d[what][r, col] = bad
        ops.linear_backward(shape, t["x"], t["w"], d["dy"], z=d["z"], grads="xwb", dx=dx, dw=dw, db=db)
        assert torch.equal(dx[others], want[0][others]) and not bool(dx[r].isfinite().any())
        by_output = dw.t() if order == "in_out" else dw  # [N, K]
        want_dw = want[1].t() if order == "in_out" else want[1]
        assert torch.equal(by_output[rest], want_dw[rest]) and not bool(by_output[col].isfinite().any())
        assert torch.equal(db[rest], want[2][rest]) and not bool(db[col].isfinite())
    assert y_ok() and z_ok() and dx_ok() and dw_ok()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,T,d", [(7, 23, 1032), (7, 24, 1032), (7, 25, 1032), (2, 97, 8), (5, 767, 64), (5, 768, 64),
                                   (5, 773, 64), (3, 333, 200), (1, 2500, 1024), (40, 130, 264), (1, 24, 8192)])
def test_gate_of_a_long_sequence(B, T, d, dtype):
    """Sequences over few and over many workgroups' rows, that start with one and inside one: both ways of adding up
    their parts."""
    shape = ops.make_residual_shape(B, T, d, dtype, post_norm=True, pre_norm=True, gate="sequence")
    check_stream(shape, "sequence", make_stream(B + T, B, T, d, dtype, True, True, "sequence"))


@pytest.mark.parametrize("order", ["in_out", "out_in"])
@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("M,K,N", [(33, 264, 1032), (1000, 520, 1304), (2048, 1024, 512)])
def test_bf16_product_gradients_lose_one_rounding(M, K, N, act, order):
    """With bf16 storage dx and dw are those of dy act'(z) rounded to bf16 once, and of nothing else that was rounded:
    against the products of the rounded values they are off by 32-bit sums and their own rounding only."""
    shape = ops.make_linear_shape(M, K, N, act=act, w_order=order)
    t = make_linear(23, M, K, N, "bf16", order)
    z = torch.empty_like(t["dy"])
    ops.linear(shape, t["x"], t["w"], bias=t["bias"], z=z)
    dx, dw, _ = ops.linear_backward(shape, t["x"], t["w"], t["dy"], z=z)
    X, W = t["x"].double(), t["w"].double() if order == "in_out" else t["w"].double().t()
    dy = t["dy"].double()
    D = dy * slope64(z.double(), act)
    # what 32 bits leave open of it (as in the bounds of all gradients), and of its rounding where that is near a tie
    e = dy.abs() * 16 * U32 * (1 + z.double().abs()) + 9e-8 * dy.abs()
    lo, hi, D = ((D + s * e).to(torch.bfloat16).double() for s in (-1, 1, 0))
    open_ = torch.maximum((hi - D).abs(), (lo - D).abs())
    for name, got, a, b, mag, gap in (
            ("dx", dx, D, W.t(), D.abs() @ W.abs().t(), open_ @ W.abs().t()),
            ("dw", dw if order == "in_out" else dw.t(), X.t(), D, X.abs().t() @ D.abs(), X.abs().t() @ open_)):
        ref = a @ b
        n = a.shape[1]
        within(got, ref, 2.0 ** -8 * ref.abs() + gap + (n + 2) * U32 * mag, name)
