"""Attention with a sliding window and first tokens that stay visible, against the 64-bit form."""
import math

import pytest
import torch

from ops_util import attention64, attention_bounds, mask_of, rand_rows, within
from paper_2505_00315_amd import ops

pytestmark = pytest.mark.gpu

# B, Hq, Hkv, dh, Q, N, window, sinks, layout, (q_lens, kv_lens) or None
CASES = [
    (1, 1, 1, 64, 1, 1, 0, 0, "bhtd", None),
    (2, 4, 2, 64, 1, 300, 0, 0, "bhtd", None),
    (2, 4, 1, 128, 1, 1000, 100, 4, "bthd", None),
    (3, 6, 2, 32, 3, 77, 10, 2, "bthd", ([3, 1, 0], [77, 5, 20])),
    (1, 2, 2, 64, 64, 64, 0, 0, "packed", None),
    (2, 4, 2, 64, 65, 65, 16, 1, "bthd", None),
    (1, 3, 1, 128, 129, 129, 1, 0, "bhtd", None),          # a query sees itself alone
    (1, 2, 1, 128, 200, 200, 64, 4, "bthd", None),
    (2, 2, 1, 64, 257, 257, 100, 70, "bhtd", None),        # more sinks than a tile of keys
    (1, 4, 4, 32, 300, 300, 33, 5, "packed", None),
    (2, 5, 5, 64, 100, 331, 50, 3, "bthd", None),          # later queries of a longer sequence
    (2, 2, 1, 64, 150, 40, 7, 2, "bhtd", None),            # more queries than keys: rows that see nothing
    (4, 3, 1, 64, 190, 190, 31, 4, "bthd", ([190, 0, 1, 77], [190, 0, 1, 77])),
    (3, 4, 2, 128, 90, 160, 40, 4, "bhtd", ([90, 13, 90], [160, 100, 30])),
    (1, 16, 2, 64, 20, 500, 0, 0, "bthd", None),
    (1, 1, 1, 64, 700, 700, 0, 0, "bhtd", None),
    (1, 2, 1, 128, 513, 513, 600, 9, "bhtd", None),        # a window of everything
    (1, 8, 1, 32, 5, 2050, 700, 3, "bthd", None),
    (2, 1, 1, 128, 3, 4100, 0, 0, "bhtd", ([3, 2], [4100, 1])),
    # few key blocks with many rows: their rows in parts
    (2, 8, 2, 64, 500, 700, 0, 0, "bthd", ([500, 77], [700, 300])),
    (1, 12, 2, 128, 400, 400, 0, 3, "bhtd", None),
    (1, 16, 4, 32, 333, 333, 0, 0, "packed", None),
    # more heads to a key head than a tile has rows
    (1, 70, 1, 32, 9, 40, 7, 2, "bthd", None),
    (2, 130, 2, 64, 5, 70, 20, 1, "bhtd", ([5, 2], [70, 40])),
]
IDS = [f"{c[0]}x{c[1]}/{c[2]}x{c[3]}-{c[4]}of{c[5]}-w{c[6]}s{c[7]}" for c in CASES]


def setup(case, dtype, seed):
    B, Hq, Hkv, dh, T, N, window, sinks, layout, lens = case
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator().manual_seed(seed)
    x = {"q": rand_rows(g, B, Hq, T, dh, dt, layout, 1.5), "k": rand_rows(g, B, Hkv, N, dh, dt, layout),
         "v": rand_rows(g, B, Hkv, N, dh, dt, layout), "do": rand_rows(g, B, Hq, T, dh, dt, layout)}
    kw = {}
    if lens:
        kw = {n: torch.tensor(v, dtype=torch.int32).cuda() for n, v in zip(("q_lens", "kv_lens"), lens)}
    shape = ops.make_attn_shape(B, Hq, Hkv, T, N, dh, dtype, window=window, sinks=sinks)
    return shape, x, kw, dt


def reference(case, x, kw, grad=True):
    return attention64(x["q"], x["k"], x["v"], case[6], case[7], kw.get("q_lens"), kw.get("kv_lens"),
                       do=x["do"] if grad else None)


def spoil_padding(x, kw):
    """Rows past the lengths hold NaN and infinities."""
    if not kw:
        return
    for b in range(x["q"].shape[0]):
        for n in ("q", "do"):
            x[n][b, :, int(kw["q_lens"][b]):] = math.nan
        for n in ("k", "v"):
            x[n][b, :, int(kw["kv_lens"][b]):] = math.inf


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_forward_and_backward(case, dtype):
    shape, x, kw, dt = setup(case, dtype, 1)
    ref = reference(case, x, kw)
    spoil_padding(x, kw)
    out, lse = ops.window_attention(shape, x["q"], x["k"], x["v"], **kw)
    dq, dk, dv = ops.window_attention_backward(shape, x["q"], x["k"], x["v"], out, lse, x["do"], **kw)
    count = max(case[5], case[4] * case[1] // case[2])
    bounds = attention_bounds(ref, dt, case[3], count)
    for n, t in (("out", out), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
        within(t, ref[n], bounds[n], f"{n} {case} {dtype}")


# enough blocks of 128 rows and keys for every CU
WIDE = [
    (4, 16, 8, 128, 2077, 2077, 300, 5, "bthd", None),
    (5, 8, 8, 64, 1733, 1733, 200, 4, "bhtd", ([1733, 1, 900, 0, 1600], [1733, 1, 900, 0, 1600])),
    (4, 24, 8, 32, 2049, 2049, 77, 70, "packed", None),
    (8, 8, 8, 128, 1100, 1100, 0, 0, "bthd", None),
    (4, 8, 8, 64, 2050, 2100, 500, 300, "bthd", None),     # sinks that are key blocks' own work
]


@pytest.mark.parametrize("case", WIDE, ids=[f"dh{c[3]}w{c[6]}s{c[7]}" for c in WIDE])
def test_wide_blocks(case):
    shape, x, kw, dt = setup(case, "bf16", 11)
    ref = reference(case, x, kw)
    spoil_padding(x, kw)
    out, lse = ops.window_attention(shape, x["q"], x["k"], x["v"], **kw)
    dq, dk, dv = ops.window_attention_backward(shape, x["q"], x["k"], x["v"], out, lse, x["do"], **kw)
    bounds = attention_bounds(ref, dt, case[3], max(case[5], case[4] * case[1] // case[2]))
    for n, t in (("out", out), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
        within(t, ref[n], bounds[n], f"{n} {case}")


@pytest.mark.parametrize("dh", [64, 128])
def test_unseen_keys_stay_out_of_wide_blocks(dh):
    case = (4, 8, 8, dh, 2100, 2100, 300, 4, "bthd", None)
    shape, x, _, _ = setup(case, "bf16", 12)
    see = mask_of(2100, 2100, 2100, 2100, 300, 4).cuda()
    clean = ops.window_attention(shape, x["q"], x["k"], x["v"])
    cg = ops.window_attention_backward(shape, x["q"], x["k"], x["v"], *clean, x["do"])
    for j in (1000, 2):
        k, v = x["k"].clone(), x["v"].clone()
        k[1, 3, j, 1], v[1, 3, j] = math.nan, math.inf
        got = ops.window_attention(shape, x["q"], k, v)
        grads = ops.window_attention_backward(shape, x["q"], k, v, *got, x["do"])
        hit = torch.zeros(4, 8, 2100, dtype=torch.bool, device="cuda")
        hit[1, 3] = see[:, j]
        assert bool(torch.isnan(got[0][hit].float()).all())
        torch.testing.assert_close(got[0][~hit].float(), clean[0][~hit].float(), rtol=2 ** -7, atol=2 ** -7)
        torch.testing.assert_close(grads[0][~hit].float(), cg[0][~hit].float(), rtol=2 ** -7, atol=2 ** -5)
        apart = torch.ones(4, 8, 2100, dtype=torch.bool, device="cuda")
        apart[1, 3] = ~(see & see[:, j:j + 1]).any(0)
        for t, c in zip(grads[1:], cg[1:]):
            torch.testing.assert_close(t[apart].float(), c[apart].float(), rtol=2 ** -7, atol=2 ** -3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("Q,N,window,sinks", [(150, 150, 20, 3), (1, 150, 20, 3), (70, 300, 0, 0)])
def test_unseen_keys_stay_out(dh, dtype, Q, N, window, sinks):
    """A key row of NaN and infinities reaches the queries that see it, and no other's output or gradient."""
    case = (1, 2, 1, dh, Q, N, window, sinks, "bhtd", None)
    shape, x, kw, _ = setup(case, dtype, 2)
    see = mask_of(Q, N, Q, N, window, sinks).cuda()
    clean = ops.window_attention(shape, x["q"], x["k"], x["v"])
    cg = ops.window_attention_backward(shape, x["q"], x["k"], x["v"], *clean, x["do"])
    for j in (N // 3, N - 1, N - 2 - window, 0):
        if not 0 <= j < N:
            continue
        k, v = x["k"].clone(), x["v"].clone()
        k[0, 0, j, 1], v[0, 0, j] = math.nan, math.inf
        got = ops.window_attention(shape, x["q"], k, v)
        free = ~see[:, j]
        # weights of the rows that do not see j are summed in another order at most
        same = free.clone()
        tol = 2 ** -7 if dtype == "bf16" else 2 ** -16
        assert bool(torch.isfinite(got[0][:, :, same].float()).all())
        torch.testing.assert_close(got[0][:, :, same].float(), clean[0][:, :, same].float(), rtol=tol, atol=tol)
        assert bool(torch.isnan(got[0][:, :, ~free].float()).all())
        # gradients: queries that do not see j, and keys that none of j's queries sees
        dq, dk, dv = ops.window_attention_backward(shape, x["q"], k, v, *got, x["do"])
        assert bool(torch.isfinite(dq[:, :, free].float()).all())
        torch.testing.assert_close(dq[:, :, free].float(), cg[0][:, :, free].float(), rtol=tol, atol=4 * tol)
        apart = ~(see & ~free[:, None]).any(0)
        apart[j] = False
        for t, c in ((dk, cg[1]), (dv, cg[2])):
            assert bool(torch.isfinite(t[:, :, apart].float()).all())
            torch.testing.assert_close(t[:, :, apart].float(), c[:, :, apart].float(), rtol=tol, atol=16 * tol)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_bad_query_stays_alone(dtype):
    case = (1, 2, 1, 64, 200, 200, 30, 2, "bhtd", None)
    shape, x, kw, _ = setup(case, dtype, 3)
    see = mask_of(200, 200, 200, 200, 30, 2).cuda()
    clean = ops.window_attention(shape, x["q"], x["k"], x["v"])
    cg = ops.window_attention_backward(shape, x["q"], x["k"], x["v"], *clean, x["do"])
    q, do = x["q"].clone(), x["do"].clone()
    q[0, 1, 77, 5], do[0, 1, 78, 6] = math.nan, math.inf
    out, lse = ops.window_attention(shape, q, x["k"], x["v"])
    hit = torch.zeros(1, 2, 200, dtype=torch.bool, device="cuda")
    hit[0, 1, 77] = True
    torch.testing.assert_close(out[~hit].float(), clean[0][~hit].float(), rtol=2 ** -7, atol=2 ** -7)
    assert bool(torch.isnan(out[hit].float()).all())
    dq, dk, dv = ops.window_attention_backward(shape, q, x["k"], x["v"], out, lse, do)
    hit[0, 1, 78] = True
    torch.testing.assert_close(dq[~hit].float(), cg[0][~hit].float(), rtol=2 ** -7, atol=2 ** -6)
    apart = ~(see[77] | see[78])
    for t, c in ((dk, cg[1]), (dv, cg[2])):
        torch.testing.assert_close(t[:, :, apart].float(), c[:, :, apart].float(), rtol=2 ** -7, atol=2 ** -4)
        assert not bool(torch.isfinite(t[:, :, 78].float()).all())  # dk: inf - inf; dv: p inf


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_scores(dtype):
    """Scores of magnitude 200 and more: one key takes a row, and nothing overflows."""
    case = (1, 2, 2, 64, 130, 130, 0, 0, "bhtd", None)
    shape, x, kw, dt = setup(case, dtype, 4)
    x["q"] *= 20
    ref = reference(case, x, kw, grad=False)
    out, lse = ops.window_attention(shape, x["q"], x["k"], x["v"])
    bounds = attention_bounds(ref, dt, 64, 130)
    within(out, ref["out"], bounds["out"], "out")
    within(lse, ref["lse"], bounds["lse"], "lse")


def test_broadcast_inputs_and_given_outputs():
    shape = ops.make_attn_shape(3, 4, 2, 40, 40, 64, window=9, sinks=1)
    g = torch.Generator().manual_seed(5)
    q = rand_rows(g, 3, 4, 40, 64, torch.bfloat16)
    k = rand_rows(g, 1, 2, 40, 64, torch.bfloat16).expand(3, 2, 40, 64)
    v = rand_rows(g, 1, 1, 40, 64, torch.bfloat16).expand(3, 2, 40, 64)
    do = rand_rows(g, 1, 1, 1, 64, torch.bfloat16).expand(3, 4, 40, 64)
    a = ops.window_attention(shape, q, k, v)
    b = ops.window_attention(shape, q, k.contiguous(), v.contiguous())
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    ga = ops.window_attention_backward(shape, q, k, v, *a, do)
    gb = ops.window_attention_backward(shape, q, k.contiguous(), v.contiguous(), *b, do.contiguous())
    for s, t in zip(ga, gb):
        assert torch.equal(s, t)
    # outputs inside a larger tensor: the rest of it stays as it was
    wide = torch.full((3, 40, 10, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    ops.window_attention(shape, q, k, v, out=wide[:, :, 2:6].transpose(1, 2))
    assert torch.equal(wide[:, :, 2:6].transpose(1, 2), a[0])
    assert bool((wide[:, :, :2] == 3).all()) and bool((wide[:, :, 6:] == 3).all())


def test_lengths_are_taken_into_the_tensors():
    case = (3, 2, 1, 64, 70, 70, 20, 2, "bhtd", None)
    shape, x, _, _ = setup(case, "bf16", 6)
    over = {n: torch.tensor([500, -3, 70], dtype=torch.int32).cuda() for n in ("q_lens", "kv_lens")}
    fair = {n: torch.tensor([70, 0, 70], dtype=torch.int32).cuda() for n in ("q_lens", "kv_lens")}
    a = ops.window_attention(shape, x["q"], x["k"], x["v"], **over)
    b = ops.window_attention(shape, x["q"], x["k"], x["v"], **fair)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert not bool(a[0][1].any()) and bool((a[1][1] == -math.inf).all())


@pytest.mark.parametrize("case", [CASES[7], CASES[2], CASES[17]], ids=["rows", "step", "few"])
def test_same_bits_again_and_beside(case):
    shape, x, kw, _ = setup(case, "bf16", 7)

    def both(stream=None):
        o = ops.window_attention(shape, x["q"], x["k"], x["v"], stream=stream)
        return (*o, *ops.window_attention_backward(shape, x["q"], x["k"], x["v"], *o, x["do"], stream=stream))
    first = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = both(side)
    again = both()
    torch.cuda.synchronize()
    for a, b, c in zip(first, other, again):
        assert torch.equal(a, b) and torch.equal(a, c)


@pytest.mark.parametrize("case", [CASES[7], CASES[2], CASES[13]], ids=["rows", "step", "ragged"])
def test_captured_and_replayed(case):
    shape, x, kw, _ = setup(case, "bf16", 8)
    scratch = ops.alloc_attn_scratch(shape)
    out, lse = ops.window_attention(shape, x["q"], x["k"], x["v"], scratch=scratch, **kw)
    g = ops.window_attention_backward(shape, x["q"], x["k"], x["v"], out, lse, x["do"], scratch=scratch, **kw)

    def step():
        ops.window_attention(shape, x["q"], x["k"], x["v"], out=out, lse=lse, scratch=scratch, **kw)
        ops.window_attention_backward(shape, x["q"], x["k"], x["v"], out, lse, x["do"], dq=g[0], dk=g[1], dv=g[2],
                                      scratch=scratch, **kw)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    res = (out, lse, *g)
    for seed in range(3):
        _, y, _, _ = setup(case, "bf16", 30 + seed)
        for n in x:
            x[n].copy_(y[n])
        for t in res:
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in res]
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, res):
            assert torch.equal(a, b)


def test_backward_is_the_slope():
    """Differences of the 64-bit form along random directions against the kernel's gradients (fp32)."""
    case = (1, 4, 2, 32, 40, 60, 13, 3, "bhtd", None)
    shape, x, kw, _ = setup(case, "f32", 9)
    o = ops.window_attention(shape, x["q"], x["k"], x["v"])
    grads = ops.window_attention_backward(shape, x["q"], x["k"], x["v"], *o, x["do"])
    g = torch.Generator().manual_seed(10)
    for n, grad in zip(("q", "k", "v"), grads):
        d = torch.randn(x[n].shape, generator=g, dtype=torch.float64).cuda()
        f = []
        for h in (1e-4, -1e-4):
            y = {m: x[m].double() for m in ("q", "k", "v")}
            y[n] = y[n] + h * d
            f.append(float((_plain(y["q"], y["k"], y["v"], 13, 3) * x["do"].double()).sum()))
        size = float((grad.double().abs() * d.abs()).sum())
        # fp32 sums of up to 60 products and 32 columns, and the difference's third-order term
        assert abs((f[0] - f[1]) / 2e-4 - float((grad.double() * d).sum())) <= 1e-4 * size


def _plain(q, k, v, window, sinks):
    G = q.shape[1] // k.shape[1]
    k, v = k.repeat_interleave(G, 1), v.repeat_interleave(G, 1)
    see = mask_of(q.shape[2], k.shape[2], q.shape[2], k.shape[2], window, sinks, q.device)
    s = (q @ k.transpose(-1, -2).contiguous()) / math.sqrt(q.shape[-1])
    return torch.softmax(s.masked_fill(~see, -math.inf), -1) @ v


# few key blocks whose windows span many rows: parts of them, beside chunks of the sinks' far rows or without
PARTS = [
    (2, 8, 2, 64, 500, 700, 200, 5, "bthd", ([500, 77], [700, 300])),
    (1, 12, 2, 128, 400, 400, 190, 70, "bhtd", None),
    (1, 16, 2, 32, 333, 420, 120, 0, "packed", None),
    (2, 24, 2, 64, 350, 350, 90, 300, "bhtd", ([350, 10], [350, 200])),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", PARTS, ids=[f"dh{c[3]}w{c[6]}s{c[7]}" for c in PARTS])
def test_parts_of_windows(case, dtype):
    shape, x, kw, dt = setup(case, dtype, 44)
    ref = reference(case, x, kw)
    spoil_padding(x, kw)
    out, lse = ops.window_attention(shape, x["q"], x["k"], x["v"], **kw)
    dq, dk, dv = ops.window_attention_backward(shape, x["q"], x["k"], x["v"], out, lse, x["do"], **kw)
    bounds = attention_bounds(ref, dt, case[3], max(case[5], case[4] * case[1] // case[2]))
    for n, t in (("out", out), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
        within(t, ref[n], bounds[n], f"{n} {case}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_sinks_than_go_by_chunks(dtype):
    case = (2, 4, 2, 64, 420, 420, 40, 300, "bthd", ([420, 350], [420, 350]))
    shape, x, kw, dt = setup(case, dtype, 40)
    ref = reference(case, x, kw)
    spoil_padding(x, kw)
    out, lse = ops.window_attention(shape, x["q"], x["k"], x["v"], **kw)
    dq, dk, dv = ops.window_attention_backward(shape, x["q"], x["k"], x["v"], out, lse, x["do"], **kw)
    bounds = attention_bounds(ref, dt, case[3], max(case[5], case[4] * case[1] // case[2]))
    for n, t in (("out", out), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
        within(t, ref[n], bounds[n], f"{n} {case}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_far_apart(dtype):
    """Strides that pass 32 bits within a tile, of rows, heads and sequences."""
    B, Hq, Hkv, dh, T = 2, 4, 2, 32, 70
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    shape = ops.make_attn_shape(B, Hq, Hkv, T, T, dh, dtype, window=30, sinks=3)
    g = torch.Generator().manual_seed(41)
    near = [rand_rows(g, B, H, T, dh, dt) for H in (Hq, Hkv, Hkv, Hq)]
    want = ops.window_attention(shape, *near[:3])
    wantg = ops.window_attention_backward(shape, *near[:3], *want, near[3])
    row, head = 1 << 25, 1 << 28
    room = torch.zeros(T * row, dtype=dt, device="cuda")  # holds B Hq heads as well
    for by_rows in (True, False):
        def place(i, H):  # the i-th tensor
            if by_rows:  # rows apart, the heads beside each other
                return torch.as_strided(room, (B, H, T, dh), (H * dh, dh, row, 1), i * B * Hq * dh)
            return torch.as_strided(room, (B, H, T, dh), (H * head, head, dh, 1), i * T * dh)
        heads = (Hq, Hkv, Hkv, Hq, Hq, Hq, Hkv, Hkv)
        q, k, v, do, out, dq, dk, dv = (place(i, H) for i, H in enumerate(heads))
        for t, x in zip((q, k, v, do), near):
            t.copy_(x)
        _, lse = ops.window_attention(shape, q, k, v, out=out)
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
        grads = ops.window_attention_backward(shape, q, k, v, out, lse, do, dq=dq, dk=dk, dv=dv)
        for a, b in zip(grads, wantg):
            assert torch.equal(a, b)


def test_two_graphs_with_one_scratch():
    """Replayed in turn, on one stream."""
    case = (1, 8, 2, 64, 1, 2000, 0, 0, "bthd", None)
    shape, x, _, _ = setup(case, "bf16", 42)
    _, y, _, _ = setup(case, "bf16", 43)
    scratch = ops.alloc_attn_scratch(shape)
    outs, graphs = [], []
    for z in (x, y):
        outs.append(ops.window_attention(shape, z["q"], z["k"], z["v"], scratch=scratch))
    want = [o[0].clone() for o in outs]
    assert not torch.equal(*want)
    torch.cuda.synchronize()
    for z, o in zip((x, y), outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            ops.window_attention(shape, z["q"], z["k"], z["v"], out=o[0], lse=o[1], scratch=scratch)
    for _ in range(3):
        for o in outs:
            o[0].fill_(5)
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0][0], want[0]) and torch.equal(outs[1][0], want[1])
