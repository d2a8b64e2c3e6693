"""Products with a weight matrix, their epilogue and gradients, against 64-bit forms."""
import pytest
import torch

from block_util import linear64, linear_grads64, within
from paper_2505_00315_amd import ops

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def matrix(g, rows, cols, dtype, layout="whole", scale=1.0):
    def normal(*s):
        return (torch.randn(s, generator=g) * scale).to(dtype).cuda()
    if layout == "whole":
        return normal(rows, cols)
    if layout == "part":  # columns of wider rows, NaN around them
        t = torch.full((rows, cols + 24), float("nan"), dtype=dtype, device="cuda")
        t[:, 8:cols + 8] = normal(rows, cols)
        return t[:, 8:cols + 8]
    if layout == "one":  # one row for all
        return normal(cols).expand(rows, cols)
    raise ValueError(layout)


def make(seed, M, K, N, dtype, order, layouts="whole whole whole whole", bias=True, residual=True):
    g, dt = torch.Generator().manual_seed(seed), DT[dtype]
    lx, lw, lr, ld = layouts.split()
    w = (K, N) if order == "in_out" else (N, K)
    t = {"x": matrix(g, M, K, dt, lx), "w": matrix(g, *w, dt, lw, K ** -0.5), "dy": matrix(g, M, N, dt, ld)}
    t["bias"] = (0.5 * torch.randn(N, generator=g)).to(dt).cuda() if bias else None
    t["residual"] = matrix(g, M, N, dt, lr) if residual else None
    return t


def check(M, K, N, dtype, act, order, t):
    shape = ops.make_linear_shape(M, K, N, dtype, act=act, w_order=order)
    z = torch.zeros(M, N, dtype=DT[dtype], device="cuda")
    y = ops.linear(shape, t["x"], t["w"], bias=t["bias"], residual=t["residual"], z=z)
    want = linear64(t["x"], t["w"], act, order, t["bias"], t["residual"])
    for name, got in (("y", y), ("z", z)):
        within(got, *want[name], f"{name} {M} {K} {N} {dtype} {act} {order}")
    keep = z if act != "none" else None
    got = ops.linear_backward(shape, t["x"], t["w"], t["dy"], z=keep, grads="xwb")
    want = linear_grads64(t["x"], t["w"], t["dy"], act, order, keep)
    for name, v in zip(("dx", "dw", "db"), got):
        within(v, *want[name], f"{name} {M} {K} {N} {dtype} {act} {order}")
    return y, z, got


# one row to several tiles, edges on every side of a tile and of a chunk of k
SIZES = [(1, 8, 8), (1, 64, 64), (2, 1024, 72), (3, 40, 72), (16, 128, 264), (17, 136, 200), (33, 2056, 64),
         (63, 72, 8), (64, 64, 64), (65, 72, 136), (100, 4104, 24), (128, 128, 128), (129, 264, 520), (300, 520, 1304),
         (1000, 64, 8), (1025, 24, 1032), (1, 4104, 3232), (20, 520, 3200), (32, 1096, 4104), (31, 8, 3080)]


@pytest.mark.parametrize("order", ["in_out", "out_in"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", SIZES)
def test_sizes(size, dtype, order):
    check(*size, dtype, "gelu", order, make(sum(size), *size, dtype, order))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("bias,residual", [(False, False), (True, False), (False, True)])
def test_epilogues(act, dtype, bias, residual):
    for size in ((5, 72, 136), (150, 200, 264)):
        check(*size, dtype, act, "in_out", make(3, *size, dtype, "in_out", bias=bias, residual=residual))


@pytest.mark.parametrize("order", ["in_out", "out_in"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layouts", ["part part part part", "one whole one one", "part whole whole part"])
def test_strides(layouts, dtype, order):
    """Rows inside wider ones, whose neighbours are NaN, and one row for all."""
    for size in ((7, 72, 88), (140, 136, 328)):
        check(*size, dtype, "silu", order, make(4, *size, dtype, order, layouts))


@pytest.mark.parametrize("size,order", [((4096, 1024, 4096), "in_out"), ((8192, 1024, 1280), "out_in"),
                                        ((2048, 4096, 2112), "in_out"), ((40, 8192, 4096), "in_out"),
                                        ((5000, 2048, 520), "out_in")])
def test_large_tiles(size, order):
    check(*size, "bf16", "silu", order, make(6, *size, "bf16", order))


@pytest.mark.parametrize("size,order", [((2100, 520, 2056), "in_out"), ((4000, 264, 1288), "out_in")])
def test_large_tiles_fp32(size, order):
    check(*size, "f32", "gelu", order, make(7, *size, "f32", order))


@pytest.mark.parametrize("order", ["in_out", "out_in"])
@pytest.mark.parametrize("size,dtype", [((1, 1000, 2056), "bf16"), ((16, 1032, 4104), "bf16"), ((17, 520, 8200), "bf16"),
                                        ((32, 72, 40), "bf16"), ((1, 2104, 8264), "f32"), ((15, 1000, 2056), "f32"),
                                        ((32, 1544, 8200), "f32"), ((18, 40, 104), "f32")])
def test_strips_of_a_few_rows(size, dtype, order):
    """Few rows by strips of columns, forward and (with the sides exchanged) dx: ends inside a strip and a chunk."""
    M, K, N = size if order == "in_out" else (size[0], size[2], size[1])
    check(M, K, N, dtype, "silu", order, make(11, M, K, N, dtype, order))


@pytest.mark.parametrize("M", [1, 3, 9, 70, 400])
def test_rows_keep_to_themselves(M):
    """NaN in one row of x reaches that row of y and dx only; memory around the outputs stays as it is."""
    K, N = 328, 456
    shape = ops.make_linear_shape(M, K, N, act="silu")
    t = make(8, M, K, N, "bf16", "in_out")
    store = torch.full((M + 2, N + 16), 7.0, dtype=torch.bfloat16, device="cuda")
    view = store[1:M + 1, 8:N + 8]
    y = ops.linear(shape, t["x"], t["w"], bias=t["bias"])
    t["x"][M // 2, 5] = float("nan")
    ops.linear(shape, t["x"], t["w"], bias=t["bias"], y=view)
    others = [i for i in range(M) if i != M // 2]
    assert torch.equal(view[others], y[others]) and torch.isnan(view[M // 2]).all()
    around = torch.ones_like(store, dtype=torch.bool)
    around[1:M + 1, 8:N + 8] = False
    assert bool((store[around] == 7.0).all())


@pytest.mark.parametrize("M", [1, 50, 300])
def test_residual_in_place(M):
    shape = ops.make_linear_shape(M, 256, 512)
    t = make(9, M, 256, 512, "bf16", "in_out")
    want = ops.linear(shape, t["x"], t["w"], bias=t["bias"], residual=t["residual"])
    r = t["residual"].clone()
    assert ops.linear(shape, t["x"], t["w"], bias=t["bias"], residual=r, y=r) is r
    assert torch.equal(r, want)


def test_only_what_is_asked():
    shape = ops.make_linear_shape(70, 136, 264, act="gelu")
    t = make(10, 70, 136, 264, "bf16", "in_out")
    z = torch.empty_like(t["dy"])
    ops.linear(shape, t["x"], t["w"], z=z)
    every = ops.linear_backward(shape, t["x"], t["w"], t["dy"], z=z, grads="xwb")
    for grads in ("x", "w", "b", "xw", "wb", ""):
        got = ops.linear_backward(shape, t["x"], t["w"], t["dy"], z=z, grads=grads)
        for letter, a, b in zip("xwb", got, every):
            assert (a is None) if letter not in grads else torch.equal(a, b)


def test_relu_at_and_around_zero():
    """The slope at 0 is 0; a NaN stays one."""
    shape = ops.make_linear_shape(2, 8, 8, "f32", act="relu")
    x, w = torch.zeros(2, 8, device="cuda"), torch.eye(8, device="cuda")
    x[0, :4] = torch.tensor([0.0, -1.0, 2.0, float("nan")], device="cuda")
    z = torch.empty(2, 8, device="cuda")
    # (NaN times the other weights, all 0, is NaN in the whole row)
    y = ops.linear(shape, x, w, z=z)
    assert torch.isnan(y[0]).all() and bool((y[1] == 0).all())
    z = torch.tensor([[0.0, -1.0, 2.0, float("nan"), -0.0, 3.0, -3.0, 1e-30]] * 2, device="cuda")
    _, _, db = ops.linear_backward(shape, x, w, torch.ones(2, 8, device="cuda"), z=z, grads="b")
    want = torch.tensor([0.0, 0.0, 2.0, float("nan"), 0.0, 2.0, 0.0, 2.0], device="cuda")
    assert torch.equal(db.isnan(), want.isnan()) and torch.equal(db.nan_to_num(9.0), want.nan_to_num(9.0))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["gelu", "silu", "relu"])
def test_infinities(act, dtype):
    """An infinite product gives the activation's limit and the slope's; NaN stays."""
    inf, nan = float("inf"), float("nan")
    z = torch.tensor([[inf, -inf, nan, 60.0, -60.0, 3e38, -3e38, 0.0]] * 3, device="cuda").to(DT[dtype])
    shape = ops.make_linear_shape(3, 8, 8, dtype, act=act)
    x, w = torch.zeros(3, 8, dtype=DT[dtype], device="cuda"), torch.zeros(8, 8, dtype=DT[dtype], device="cuda")
    y = ops.linear(shape, x, w, bias=z[0].contiguous())
    big = float(z[0, 5])
    want = torch.tensor([inf, 0.0, nan, 60.0, 0.0, big, 0.0, 0.0], device="cuda")
    assert torch.equal(y[0].isnan(), want.isnan())
    assert float((y[0].float().nan_to_num(0.0, posinf=1.0) - want.nan_to_num(0.0, posinf=1.0)).abs().max()) < 1e-15
    _, _, db = ops.linear_backward(shape, x, w, torch.ones_like(z), z=z, grads="b")
    half = {"gelu": 0.5, "silu": 0.5, "relu": 0.0}[act]
    want = 3 * torch.tensor([1.0, 0.0, nan, 1.0, 0.0, 1.0, 0.0, half], device="cuda")
    assert torch.equal(db.isnan(), want.isnan()) and float((db.float() - want).nan_to_num(0.0).abs().max()) < 1e-6


@pytest.mark.parametrize("size", [(1, 1024, 512), (200, 520, 264), (2048, 512, 1024)])
def test_captured(size):
    M, K, N = size
    shape = ops.make_linear_shape(M, K, N, act="gelu")
    t = make(11, M, K, N, "bf16", "in_out")
    y, z, dx = (torch.zeros(M, n, dtype=torch.bfloat16, device="cuda") for n in (N, N, K))
    dw, db, scratch = torch.zeros_like(t["w"]), torch.zeros_like(t["bias"]), ops.alloc_linear_scratch(shape)

    def step():
        ops.linear(shape, t["x"], t["w"], bias=t["bias"], residual=t["residual"], y=y, z=z, scratch=scratch)
        ops.linear_backward(shape, t["x"], t["w"], t["dy"], z=z, grads="xwb", dx=dx, dw=dw, db=db, scratch=scratch)
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        t["x"].mul_(0.75)
        t["dy"].copy_(t["dy"].flip(0))
        z2 = torch.empty_like(z)
        want = [ops.linear(shape, t["x"], t["w"], bias=t["bias"], residual=t["residual"], z=z2)]
        want += ops.linear_backward(shape, t["x"], t["w"], t["dy"], z=z2, grads="xwb")
        for v in (y, z, dx, dw, db):
            v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((y, dx, dw, db), want):
            assert torch.equal(a, b), k


def test_two_streams():
    """Calls at once on two streams, with scratch of their own, on other streams than the tensors' first one."""
    shape = ops.make_linear_shape(24, 4096, 1024, act="silu")
    t = [make(12 + i, 24, 4096, 1024, "bf16", "in_out") for i in range(2)]
    want = [ops.linear(shape, u["x"], u["w"], bias=u["bias"], residual=u["residual"]) for u in t]
    streams, scratch = [torch.cuda.Stream() for _ in t], [ops.alloc_linear_scratch(shape) for _ in t]
    out = [[torch.zeros_like(want[0]) for _ in range(20)] for _ in t]
    torch.cuda.synchronize()
    for k in range(20):
        for i, u in enumerate(t):
            ops.linear(shape, u["x"], u["w"], bias=u["bias"], residual=u["residual"], y=out[i][k], scratch=scratch[i],
                       stream=streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(o, want[i]) for o in out[i])


def test_far_rows():
    """Rows whose offsets pass 32 bits."""
    M, K, N = 3000, 64, 72
    shape = ops.make_linear_shape(M, K, N, act="silu")
    t = make(14, M, K, N, "bf16", "in_out", bias=False, residual=False)
    want = ops.linear(shape, t["x"], t["w"])
    far = torch.zeros(M * (1 << 20) + 4096, dtype=torch.bfloat16, device="cuda")
    x = far.as_strided((M, K), (1 << 20, 1))
    y = far.as_strided((M, N), (1 << 20, 1), 128)
    x.copy_(t["x"])
    ops.linear(shape, x, t["w"], y=y)
    assert torch.equal(y, want)
    dy = far.as_strided((M, N), (1 << 20, 1), 512)
    dy.copy_(t["dy"])
    z = torch.empty_like(t["dy"])
    ops.linear(shape, t["x"], t["w"], z=z)
    a = ops.linear_backward(shape, t["x"], t["w"], t["dy"], z=z, grads="xwb")
    b = ops.linear_backward(shape, x, t["w"], dy, z=z, grads="xwb")
    assert all(torch.equal(p, q) for p, q in zip(a, b))
