"""The residual stream with norms and gate, forward and backward, against 64-bit forms."""
import pytest
import torch

from block_util import residual64, within
from paper_2505_00315_amd import ops

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def stream(g, B, T, d, dtype, layout="btd", scale=1.0):
    def normal(*s):
        return (torch.randn(s, generator=g) * scale).to(dtype).cuda()
    if layout == "btd":
        return normal(B, T, d)
    if layout == "tbd":
        return normal(T, B, d).transpose(0, 1)
    if layout == "part":  # columns of wider rows
        return normal(B, T, d + 24)[..., 8:d + 8]
    if layout == "one":  # one row for every token
        return normal(d).expand(B, T, d)
    raise ValueError(layout)


def make(seed, B, T, d, dtype, post, pre, gate, layouts="btd btd btd btd btd", weights=True):
    g, dt = torch.Generator().manual_seed(seed), DT[dtype]
    lx, ly, lg, lh, ln = layouts.split()
    t = {"x": stream(g, B, T, d, dt, lx, 3.0), "y": stream(g, B, T, d, dt, ly)}
    if gate != "none":
        t["gate"] = {"vector": lambda: stream(g, 1, 1, d, dt)[0, 0], "sequence": lambda: stream(g, B, 1, d, dt)[:, 0],
                     "token": lambda: stream(g, B, T, d, dt, lg)}[gate]()
    if post and weights:
        t["w_post"] = (1 + 0.3 * torch.randn(d, generator=g)).to(dt).cuda()
    if pre and weights:
        t["w_pre"] = (1 + 0.3 * torch.randn(d, generator=g)).to(dt).cuda()
    t["dh"] = stream(g, B, T, d, dt, lh)
    if pre:
        t["dn"] = stream(g, B, T, d, dt, ln)
    return t


def check(shape, gate, t, **kw):
    """Forward and backward of the operator against the 64-bit form."""
    ins = {n: t.get(n) for n in ("x", "y", "w_post", "gate", "w_pre")}
    want = residual64(shape, gate, **ins, dh=t.get("dh"), dn=t.get("dn"), grads=True)
    h, n = ops.residual_norm(shape, **ins)
    got = dict(zip(("dx", "dy", "dw_post", "dgate", "dw_pre"),
                   ops.residual_norm_backward(shape, **ins, dh=t.get("dh"), dn=t.get("dn"), **kw)))
    got.update(h=h, n=n)
    for name, (ref, bound) in want.items():
        if got.get(name) is not None:
            within(got[name], ref, bound, name)
    return got


SIZES = [(1, 1, 8), (1, 3, 64), (2, 5, 72), (3, 33, 136), (2, 7, 264), (1, 9, 520), (2, 3, 1032), (1, 5, 2056),
         (1, 3, 4104), (2, 2, 8192)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", SIZES)
def test_widths(size, dtype):
    """Every width of a team of lanes, at its edges; all parts of the operator."""
    B, T, d = size
    shape = ops.make_residual_shape(B, T, d, dtype, post_norm=True, pre_norm=True, gate="vector", residual_scale=0.9,
                                    branch_scale=-0.5)
    check(shape, "vector", make(d, B, T, d, dtype, True, True, "vector"))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gate", ["none", "vector", "sequence", "token"])
@pytest.mark.parametrize("post,pre", [(True, True), (True, False), (False, True), (False, False)])
def test_parts(post, pre, gate, dtype):
    shape = ops.make_residual_shape(3, 21, 200, dtype, post_norm=post, pre_norm=pre, gate=gate, branch_scale=0.7)
    check(shape, gate, make(5, 3, 21, 200, dtype, post, pre, gate))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,T", [(2, 5000), (700, 3), (3000, 1), (1, 4099), (37, 111)])
@pytest.mark.parametrize("d", [64, 1024])
def test_gate_of_a_sequence(B, T, d, dtype):
    """Sequences that end inside a workgroup's rows, fill several workgroups, or are many in one."""
    shape = ops.make_residual_shape(B, T, d, dtype, post_norm=True, pre_norm=True, gate="sequence")
    check(shape, "sequence", make(B + T, B, T, d, dtype, True, True, "sequence"))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layouts", ["tbd part tbd part tbd", "part tbd part tbd btd", "one btd one one btd",
                                     "btd one tbd btd one"])
def test_strides(layouts, dtype):
    shape = ops.make_residual_shape(4, 9, 328, dtype, post_norm=True, pre_norm=True, gate="token")
    check(shape, "token", make(3, 4, 9, 328, dtype, True, True, "token", layouts))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_without_weights_or_gradient_of_the_stream(dtype):
    shape = ops.make_residual_shape(2, 17, 96, dtype, post_norm=True, pre_norm=True)
    t = make(8, 2, 17, 96, dtype, True, True, "none", weights=False)
    t["dh"] = None
    got = check(shape, "none", t)
    assert got["dw_post"] is None and got["dw_pre"] is None


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_first_block(dtype):
    """Without a block's output the stream is x, whatever the scales."""
    shape = ops.make_residual_shape(2, 33, 264, dtype, pre_norm=True, residual_scale=0.5, branch_scale=2.0)
    t = make(9, 2, 33, 264, dtype, False, True, "none")
    t["y"] = None
    got = check(shape, "none", t)
    assert got["h"] is t["x"] and got["dy"] is None


@pytest.mark.parametrize("d", [64, 1024, 4096])
def test_in_place(d):
    """Outputs in the place of inputs give what new tensors give."""
    shape = ops.make_residual_shape(2, 301, d, post_norm=True, pre_norm=True, gate="token")
    t = make(11, 2, 301, d, "bf16", True, True, "token")
    ins = {n: t[n] for n in ("x", "y", "w_post", "gate", "w_pre")}
    h, n = ops.residual_norm(shape, **ins)
    grads = ops.residual_norm_backward(shape, **ins, dh=t["dh"], dn=t["dn"])
    x, y = t["x"].clone(), t["y"].clone()
    ops.residual_norm(shape, **{**ins, "x": x, "y": y}, h_out=x, n_out=y)
    assert torch.equal(x, h) and torch.equal(y, n)
    for swap in (False, True):
        dh, dn = t["dh"].clone(), t["dn"].clone()
        got = ops.residual_norm_backward(shape, **ins, dh=dh, dn=dn, dx=dn if swap else dh, dy=dh if swap else dn)
        for a, b in zip(got, grads):
            assert torch.equal(a, b)


def test_reproducible_and_only_what_is_asked():
    """Gradients that are not asked for leave the others as they are."""
    shape = ops.make_residual_shape(3, 500, 256, post_norm=True, pre_norm=True, gate="sequence")
    t = make(12, 3, 500, 256, "bf16", True, True, "sequence")
    ins = {n: t[n] for n in ("x", "y", "w_post", "gate", "w_pre")}
    first = ops.residual_norm_backward(shape, **ins, dh=t["dh"], dn=t["dn"])
    again = ops.residual_norm_backward(shape, **ins, dh=t["dh"], dn=t["dn"])
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    # through the C entry, which takes NULL for each of the sums
    def R(x):
        return ops.Rows(x.data_ptr(), x.stride(0), 0, x.stride(1))

    def G(x):
        return ops.Rows(x.data_ptr(), x.stride(0), 0, 0)
    for keep in range(8):
        out = [torch.zeros_like(a) for a in first]
        scratch = ops.alloc_residual_scratch(shape)
        ptr = [out[2].data_ptr() if keep & 1 else None, G(out[3]) if keep & 2 else None, out[4].data_ptr() if keep & 4 else None]
        ops._call("mosa_residual_norm_backward", t["x"].device, None, shape, R(t["x"]), R(t["y"]), t["w_post"].data_ptr(),
                  G(t["gate"]), t["w_pre"].data_ptr(), R(t["dh"]), R(t["dn"]), R(out[0]), R(out[1]), *ptr,
                  scratch.data_ptr(), scratch.numel())
        for i, a in enumerate(out):
            asked = i < 2 or keep & (1 << (i - 2))
            assert torch.equal(a, first[i] if asked else torch.zeros_like(a)), (keep, i)


def test_rows_keep_to_themselves():
    """A row of NaN or infinities reaches no other row; rows beside the tensors stay as they are."""
    shape = ops.make_residual_shape(2, 40, 136, post_norm=True, pre_norm=True, gate="token")
    t = make(13, 2, 40, 136, "bf16", True, True, "token")
    ins = {n: t[n] for n in ("x", "y", "w_post", "gate", "w_pre")}
    h, n = ops.residual_norm(shape, **ins)
    dx, dy, *_ = ops.residual_norm_backward(shape, **ins, dh=t["dh"], dn=t["dn"])
    t["x"][0, 7, 3], t["y"][1, 11, 5], t["dn"][1, 39, 0] = float("nan"), float("inf"), float("nan")
    store = torch.full((2, 42, 152), 5.0, dtype=torch.bfloat16, device="cuda")
    view = store[:, 1:41, 8:144]
    h2, n2 = ops.residual_norm(shape, **ins, h_out=view)
    dx2, dy2, *_ = ops.residual_norm_backward(shape, **ins, dh=t["dh"], dn=t["dn"])
    hit = torch.zeros(2, 40, dtype=torch.bool, device="cuda")
    hit[0, 7] = hit[1, 11] = hit[1, 39] = True
    for a, b in ((h, h2), (n, n2), (dx, dx2), (dy, dy2)):
        assert torch.equal(a[~hit], b[~hit])
    assert torch.isnan(n2[0, 7]).all() and torch.isnan(dx2[1, 39]).all()
    around = torch.ones_like(store, dtype=torch.bool)
    around[:, 1:41, 8:144] = False
    assert bool((store[around] == 5.0).all())


def test_differences():
    """The gradients are those of the forward: central differences in fp32 along random directions."""
    B, T, d = 2, 5, 24
    shape = ops.make_residual_shape(B, T, d, "f32", post_norm=True, pre_norm=True, gate="sequence", residual_scale=0.8,
                                    branch_scale=1.3, eps=1e-3)
    t = make(14, B, T, d, "f32", True, True, "sequence")
    ins = {n: t[n] for n in ("x", "y", "w_post", "gate", "w_pre")}
    grads = dict(zip(("x", "y", "w_post", "gate", "w_pre"),
                     ops.residual_norm_backward(shape, **ins, dh=t["dh"], dn=t["dn"])))
    g = torch.Generator().manual_seed(15)

    def loss(**change):
        h, n = ops.residual_norm(shape, **{**ins, **change})
        return float((h.double() * t["dh"].double()).sum() + (n.double() * t["dn"].double()).sum())
    for name, v in ins.items():
        step = torch.randn(v.shape, generator=g).cuda()
        eps = 2.0 ** -7
        num = (loss(**{name: v + eps * step}) - loss(**{name: v - eps * step})) / (2 * eps)
        ana = float((grads[name].double() * step.double()).sum())
        size = float((grads[name].double() * step.double()).abs().sum())
        # third differences of functions of size 1: eps^2 times the sum of the magnitudes, a few times
        assert abs(num - ana) < 0.01 * size, (name, num, ana, size)


@pytest.mark.parametrize("d", [64, 1024])
def test_captured(d):
    """A captured step replays to the eager results, beside eager work on the same tensors."""
    shape = ops.make_residual_shape(3, 130, d, post_norm=True, pre_norm=True, gate="sequence")
    t = make(16, 3, 130, d, "bf16", True, True, "sequence")
    ins = {n: t[n] for n in ("x", "y", "w_post", "gate", "w_pre")}
    out = {n: torch.zeros_like(t["x"]) for n in ("h", "n", "dx", "dy")}
    sums = {"dw_post": torch.zeros_like(t["w_post"]), "dgate": torch.zeros_like(t["gate"]), "dw_pre": torch.zeros_like(t["w_pre"])}
    scratch = ops.alloc_residual_scratch(shape)

    def step():
        ops.residual_norm(shape, **ins, h_out=out["h"], n_out=out["n"])
        ops.residual_norm_backward(shape, **ins, dh=t["dh"], dn=t["dn"], dx=out["dx"], dy=out["dy"], **sums, scratch=scratch)
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        t["x"].copy_(t["x"].flip(0))
        t["dn"].mul_(1.5)
        h, n = ops.residual_norm(shape, **ins)
        want = ops.residual_norm_backward(shape, **ins, dh=t["dh"], dn=t["dn"])
        for v in (*out.values(), *sums.values()):
            v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = (out["dx"], out["dy"], sums["dw_post"], sums["dgate"], sums["dw_pre"])
        assert torch.equal(out["h"], h) and torch.equal(out["n"], n)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), k


def test_far_rows():
    """Rows whose offsets pass 32 bits."""
    B, T, d = 2, 4, 64
    shape = ops.make_residual_shape(B, T, d, post_norm=True, pre_norm=True)
    far = torch.zeros((1 << 31) + (1 << 30) + 4096, dtype=torch.bfloat16, device="cuda")
    t = make(17, B, T, d, "bf16", True, True, "none")

    def spread(x):
        v = far.as_strided((B, T, d), ((1 << 31) + 64, (1 << 28) + 128, 1))
        v.copy_(x)
        return v
    ins = {n: t[n] for n in ("x", "y", "w_post", "w_pre")}
    h, n = ops.residual_norm(shape, **ins)
    h2, n2 = ops.residual_norm(shape, **{**ins, "x": spread(t["x"])})
    assert torch.equal(h, h2) and torch.equal(n, n2)
    v = far.as_strided((B, T, d), ((1 << 31) + 64, (1 << 28) + 128, 1))
    ops.residual_norm(shape, **ins, h_out=v)
    assert torch.equal(v, h)
