"""Log probabilities of tokens, their entropy, alternatives and gradients, against 64-bit forms."""
import math

import pytest
import torch

from block_util import logprobs64, within
from paper_2505_00315_amd import ops

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def check(x, targets, scale=1.0, top=0, entropy=True, backward=True, seed=0, dtype=None):
    R, V = x.shape
    dtype = "bf16" if x.dtype == torch.bfloat16 else "f32"
    shape = ops.make_logprob_shape(R, V, dtype, top=top, scale=scale)
    g = torch.Generator().manual_seed(seed)
    d = {n: torch.randn(R, generator=g).cuda() for n in ("d_logp", "d_lse", "d_entropy")} if backward else {}
    if targets is None:
        d.pop("d_logp", None)
    if not entropy:
        d.pop("d_entropy", None)
    want = logprobs64(x, targets, shape.scale, top, **d)
    stats = torch.empty(R, 2, device="cuda")
    ent = torch.empty(R, device="cuda") if entropy else None
    logp, lse, top_logp, top_index = ops.token_logprobs(shape, x, targets, stats=stats, entropy=ent)
    what = f"{R} x {V} {dtype} top {top}"
    within(lse, *want["lse"], "lse " + what)
    if targets is not None:
        within(logp, *want["logp"], "logp " + what)
    if entropy:
        within(ent, *want["entropy"], "entropy " + what)
    if top:
        assert torch.equal(top_index.long(), want["top_index"]), "alternatives " + what
        within(top_logp, *want["top_logp"], "log p of alternatives " + what)
    if backward and d:
        dx = ops.token_logprobs_backward(shape, x, targets, stats, entropy=ent, **d)
        within(dx, *want["dx"], "gradient " + what)
        inplace = x.clone() if x.is_contiguous() else x
        ops.token_logprobs_backward(shape, inplace, targets, stats, entropy=ent, **d, d_logits=inplace)
        assert torch.equal(*(v.view(torch.int16 if dtype == "bf16" else torch.int32) for v in (inplace, dx)))  # (NaN too)
    return logp, lse, ent, top_logp, top_index


def logits(seed, R, V, dtype, spread=3.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(R, V, generator=g) * spread).to(DT[dtype]).cuda()


def targets_of(seed, R, V, none=True):
    g = torch.Generator().manual_seed(seed + 100)
    t = torch.randint(0, V, (R,), generator=g, dtype=torch.int32)
    if none and R > 2:
        t[1], t[2] = -1, V
    return t.cuda()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 17, 63, 64, 255, 1000, 2049, 8191, 32000, 50001, 131075])
@pytest.mark.parametrize("R", [1, 5, 37])
def test_sizes(R, V, dtype):
    check(logits(V + R, R, V, dtype), targets_of(V, R, V), top=min(V, 20))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,V", [(1, 300007), (3, 140001), (130, 9001), (300, 66003), (600, 5000), (1500, 9), (1100, 3001),
                                 (2000, 517)])
def test_parts_of_rows(R, V, dtype):
    """Rows in parts that are joined, and one workgroup's."""
    check(logits(R, R, V, dtype), targets_of(R, R, V), top=7)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("top,entropy", [(0, False), (0, True), (1, False), (32, True), (5, True)])
def test_parts(top, entropy, dtype):
    for R, V in ((3, 40), (70, 3001), (2, 40000)):
        check(logits(R, R, V, dtype), targets_of(R, R, V), scale=0.7, top=top, entropy=entropy)
    check(logits(1, 3, 500, dtype), None, top=top, entropy=entropy)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [33, 5000, 70001, 262147])
def test_equal_values(V, dtype):
    """Ties go to the lower index: rows of few different values, of one value, rising and falling; many such rows."""
    g = torch.Generator().manual_seed(V)
    if V < 100000:
        check(torch.randint(-1, 2, (1100, min(V, 3000)), generator=g).to(DT[dtype]).cuda(), None, top=32, backward=False)
    x = torch.randint(-2, 3, (6, V), generator=g).float()
    x[1] = 1.5
    x[2] = torch.arange(V) / 64
    x[3] = -torch.arange(V) / 64
    x[4] = torch.where(torch.arange(V) % 2 == 0, 0.0, -0.0)
    x[5] = -3.0
    x[5, V // 2:] = 2.0
    check(x.to(DT[dtype]).cuda(), targets_of(V, 6, V), top=32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [9, 700, 33333, 150001])
def test_masked(V, dtype):
    """-inf in places, in all but one, everywhere; the type's lowest value in places and everywhere; masked targets."""
    x = logits(V, 9, V, dtype)
    g = torch.Generator().manual_seed(V)
    x[0][(torch.rand(V, generator=g) < 0.6).cuda()] = -math.inf
    x[1] = -math.inf
    x[1, V // 3] = 2.0
    x[2] = -math.inf
    low = torch.finfo(x.dtype).min
    x[3] = low
    x[4, : V // 2] = low
    x[5, : V - 1] = -math.inf
    x[6, 1:] = -math.inf
    t = targets_of(V, 9, V, none=False)
    t[4], t[5], t[6], t[2] = 0, 0, 0, 1
    check(x, t, top=min(9, V))
    check(x, t, scale=0.5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [12, 3000, 40001, 140002])
def test_not_finite(V, dtype):
    """A row with NaN or +inf is NaN throughout; the others are as without it; alternatives stay in order."""
    x = logits(V, 7, V, dtype)
    x[1, V // 2] = math.nan
    x[2, V - 1] = math.inf
    x[3] = math.nan
    x[4, :] = -math.inf
    x[4, 0] = math.nan
    x[5, ::2] = math.inf
    check(x, targets_of(V, 7, V, none=False), top=min(V, 8))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_far_from_zero(dtype):
    """Rows shifted far from 0 lose what their storage loses, and no more."""
    x = (logits(1, 4, 3000, dtype).float() * 8 + torch.tensor([[3e4], [-3e4], [1e30], [0.0]]).cuda()).to(DT[dtype])
    check(x, targets_of(1, 4, 3000, none=False), top=4)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1, 5, 250, 5001, 40003])
@pytest.mark.parametrize("lead,pad", [(0, 0), (1, 0), (3, 5), (8, 3)])
def test_rows_anywhere(lead, pad, V, dtype):
    """Rows that start at any element, NaN around them; the gradient leaves what is around it as it is."""
    R = 6
    width = lead + V + pad
    store = torch.full((R * width + 16,), math.nan, dtype=DT[dtype], device="cuda")
    x = store.as_strided((R, V), (width, 1), lead)
    x.copy_(logits(V, R, V, dtype))
    t = targets_of(V, R, V)
    check(x.clone(), t, top=min(V, 3))
    shape = ops.make_logprob_shape(R, V, dtype, top=min(V, 3))
    stats, ent = torch.empty(R, 2, device="cuda"), torch.empty(R, device="cuda")
    got = ops.token_logprobs(shape, x, t, stats=stats, entropy=ent)
    ref_stats, ref_ent = torch.empty_like(stats), torch.empty_like(ent)
    want = logprobs64(x, t, 1.0, min(V, 3), d_logp=torch.ones(R, device="cuda"), d_entropy=torch.ones(R, device="cuda"))
    within(got[0], *want["logp"], "logp")
    within(got[1], *want["lse"], "lse")
    assert torch.equal(got[3].long(), want["top_index"])
    place = torch.full((R * width + 16,), 4.0, dtype=DT[dtype], device="cuda")
    dx = place.as_strided((R, V), (width, 1), lead)
    ones = torch.ones(R, device="cuda")
    ops.token_logprobs_backward(shape, x, t, stats, entropy=ent, d_logp=ones, d_entropy=ones, d_logits=dx)
    within(dx, *want["dx"], "gradient")
    other = ops.token_logprobs_backward(shape, x, t, stats, entropy=ent, d_logp=ones, d_entropy=ones)
    assert torch.equal(other, dx)
    inside = torch.zeros(R * width + 16, dtype=torch.bool, device="cuda")
    inside.as_strided((R, V), (width, 1), lead).fill_(True)
    assert bool((place[~inside] == 4.0).all())


def test_one_row_for_all():
    x = logits(3, 1, 3000, "bf16").expand(40, 3000)
    t = torch.arange(40, dtype=torch.int32, device="cuda")
    shape = ops.make_logprob_shape(40, 3000, top=2)
    logp, lse, tl, ti = ops.token_logprobs(shape, x, t)
    want = logprobs64(x, t, 1.0, 2)
    within(logp, *want["logp"], "logp")
    assert torch.equal(ti.long(), want["top_index"])


def test_gradient_parts():
    """Each gradient alone, and none."""
    R, V = 9, 1003
    x, t = logits(4, R, V, "f32"), targets_of(4, R, V)
    shape = ops.make_logprob_shape(R, V, "f32", scale=1.3)
    stats, ent = torch.empty(R, 2, device="cuda"), torch.empty(R, device="cuda")
    ops.token_logprobs(shape, x, t, stats=stats, entropy=ent)
    g = torch.linspace(-1, 1, R, device="cuda")
    for name in ("d_logp", "d_lse", "d_entropy"):
        dx = ops.token_logprobs_backward(shape, x, t, stats, entropy=ent, **{name: g})
        within(dx, *logprobs64(x, t, shape.scale, **{name: g})["dx"], name)
    assert bool((ops.token_logprobs_backward(shape, x, t, stats) == 0).all())


def test_differences():
    """The gradient is that of the forward: central differences along random directions."""
    R, V = 5, 77
    x, t = logits(5, R, V, "f32", 1.0), targets_of(5, R, V)
    shape = ops.make_logprob_shape(R, V, "f32", scale=0.8)
    g = torch.Generator().manual_seed(6)
    d = [torch.randn(R, generator=g).cuda() for _ in range(3)]
    stats, ent = torch.empty(R, 2, device="cuda"), torch.empty(R, device="cuda")
    ops.token_logprobs(shape, x, t, stats=stats, entropy=ent)
    dx = ops.token_logprobs_backward(shape, x, t, stats, entropy=ent, d_logp=d[0], d_lse=d[1], d_entropy=d[2])

    def loss(v):
        e = torch.empty(R, device="cuda")
        logp, lse, _, _ = ops.token_logprobs(shape, v, t, entropy=e)
        return float(sum((a.double() * b.double()).sum() for a, b in zip((logp, lse, e), d)))
    for k in range(4):
        step, eps = torch.randn(R, V, generator=g).cuda(), 2.0 ** -6
        num = (loss(x + eps * step) - loss(x - eps * step)) / (2 * eps)
        part = dx.double() * step.double()
        # third derivatives of size 1 times eps^2, and 2^-24 / eps of values of size 5
        assert abs(num - float(part.sum())) < 0.005 * float(part.abs().sum()) + 1e-3


@pytest.mark.parametrize("R,V,top", [(1, 32000, 20), (200, 5000, 3)])
def test_captured(R, V, top):
    x, t = logits(7, R, V, "bf16"), targets_of(7, R, V)
    shape = ops.make_logprob_shape(R, V, top=top)
    new = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731
    o = {"logp": new(R), "lse": new(R), "stats": new(R, 2), "entropy": new(R), "top_logp": new(R, top),
         "top_index": new(R, top, dtype=torch.int32)}
    dx, ones, scratch = torch.zeros_like(x), torch.ones(R, device="cuda"), ops.alloc_logprob_scratch(shape)

    def step():
        ops.token_logprobs(shape, x, t, **o, scratch=scratch)
        ops.token_logprobs_backward(shape, x, t, o["stats"], entropy=o["entropy"], d_logp=ones, d_entropy=ones, d_logits=dx)
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        x.copy_(x.roll(17, 1))
        s, e = torch.empty_like(o["stats"]), torch.empty_like(o["entropy"])
        want = ops.token_logprobs(shape, x, t, stats=s, entropy=e)
        grad = ops.token_logprobs_backward(shape, x, t, s, entropy=e, d_logp=ones, d_entropy=ones)
        for v in (*o.values(), dx):
            v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((o["logp"], o["lse"], o["top_logp"], o["top_index"], o["stats"], o["entropy"], dx), (*want, s, e, grad)):
            assert torch.equal(a, b), k


def test_far_rows():
    """Rows whose offsets pass 32 bits."""
    R, V = 70000, 40000
    x = torch.zeros(R, V, dtype=torch.bfloat16, device="cuda")
    last = logits(8, 3, V, "bf16")
    x[-3:] = last
    t = torch.zeros(R, dtype=torch.int32, device="cuda")
    shape = ops.make_logprob_shape(R, V, top=2)
    stats = torch.empty(R, 2, device="cuda")
    logp, lse, tl, ti = ops.token_logprobs(shape, x, t, stats=stats)
    one = ops.make_logprob_shape(3, V, top=2)
    want = logprobs64(last, t[:3], 1.0, 2, d_logp=torch.ones(3, device="cuda"))
    within(logp[-3:], *want["logp"], "logp")
    assert torch.equal(ti[-3:].long(), want["top_index"])
    ops.token_logprobs_backward(shape, x, t, stats, d_logp=torch.ones(R, device="cuda"), d_logits=x)
    within(x[-3:], *want["dx"], "gradient")
    within(x[40000:40001, 1:], torch.full((1, V - 1), -1.0 / V).cuda(), torch.tensor(2 ** -8 / V).cuda(), "gradient of a flat row")
