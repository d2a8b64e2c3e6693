"""Keys, values and queries that hold infinities or NaN: they reach what sees them, nothing else, and in about the
time of any other call, also where a row's keys or a key's rows are worked on in parts."""
import math

import pytest
import torch

from ops_util import HALF, U32, cache64, mask_of, rand_rows
from paper_2505_00315_amd import ops

pytestmark = pytest.mark.gpu

# B, Hq, Hkv, dh, Q, N, window, sinks
CASES = [
    (1, 2, 1, 64, 1, 3000, 0, 0),       # one token, its keys in parts
    (2, 4, 2, 128, 5, 2500, 700, 3),    # a few tokens, their keys in parts
    (1, 4, 2, 64, 300, 300, 40, 70),
    (2, 8, 2, 64, 250, 350, 100, 5),    # few key blocks: their rows in parts
    (1, 12, 2, 128, 200, 200, 0, 0),    # the same without a window
    (1, 6, 2, 32, 150, 260, 60, 2),     # a group that does not divide a tile
    (1, 70, 1, 32, 9, 40, 7, 2),        # more heads to a key head than a tile has rows
]
IDS = [f"{c[0]}x{c[1]}/{c[2]}x{c[3]}-{c[4]}of{c[5]}-w{c[6]}s{c[7]}" for c in CASES]
WIDE = (5, 16, 8, 64, 1700, 1700, 200, 4)  # enough blocks of 128 rows and of 128 keys for every CU


def setup(case, dtype, seed):
    B, Hq, Hkv, dh, Q, N, window, sinks = case
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator().manual_seed(seed)
    x = {n: rand_rows(g, B, H, T, dh, dt, "bthd") for n, H, T in (("q", Hq, Q), ("k", Hkv, N), ("v", Hkv, N), ("do", Hq, Q))}
    x["q"] = torch.where(x["q"] == 0, 1.0, x["q"])  # (0 times infinity would be another case)
    return ops.make_attn_shape(B, Hq, Hkv, Q, N, dh, dtype, window=window, sinks=sinks), x, dt


def sums(see, w, y):
    """sum over the pairs that see names of w [i, j] y [j, :], in 64 bits; other pairs take no part, whatever y holds."""
    out = [torch.where(see[i:i + 64, :, None], w[i:i + 64, :, None] * y, 0.0).sum(1) for i in range(0, see.shape[0], 64)]
    return torch.cat(out)


def formula(x, b, h, G, see):
    """One query head by the definition.  A row whose scores are all minus infinity counts as one that sees nothing."""
    Q, K, V = x["q"][b, h].double(), x["k"][b, h // G].double(), x["v"][b, h // G].double()
    scale = 1 / math.sqrt(Q.shape[1])
    S = torch.where(see, Q @ K.T * scale, -math.inf)
    top = S.amax(1, keepdim=True)
    E = torch.where(see, torch.exp(S - torch.where(top == -math.inf, 0.0, top)), 0.0)
    total = E.sum(1, keepdim=True)
    P = E / torch.where(total == 0, 1.0, total)
    O = sums(see, P, V)
    return {"out": O, "lse": (top + torch.log(total)).squeeze(1), "mag": sums(see, P, V.abs()), "P": P}


def gradients(x, b, hk, G, see, dt):
    """Gradients of a key head and of its query heads, and the terms of their bounds, as in attention64; a pair that see
    does not name takes no part."""
    K, V = x["k"][b, hk].double(), x["v"][b, hk].double()
    scale, half, back = 1 / math.sqrt(K.shape[1]), HALF[dt], see.T.contiguous()
    res = {n: 0.0 for n in ("dk", "dk_mag", "dk_d", "dv", "dv_mag")}
    for h in range(hk * G, (hk + 1) * G):
        f = formula(x, b, h, G, see)
        P, O, Q, D = f["P"], f["out"], x["q"][b, h].double(), x["do"][b, h].double()
        dS = torch.where(see, P * (D @ V.T - (D * O).sum(1, keepdim=True)), 0.0)
        eD = half * (D.abs() * (f["mag"] + O.abs())).sum(1, keepdim=True)
        mag = torch.where(see, P * (D.abs() @ V.abs().T + (D * O).abs().sum(1, keepdim=True)), 0.0)
        off = torch.where(see, P * eD + half * dS.abs(), 0.0)
        for n, w, y in (("", dS, K), ("_mag", mag, K.abs()), ("_d", off, K.abs())):
            res["dq" + n, h] = sums(see, w, y) * scale
        for n, w, y in (("", dS, Q), ("_mag", mag, Q.abs()), ("_d", off, Q.abs())):
            res["dk" + n] = res["dk" + n] + sums(back, w.T, y) * scale
        for n, w, y in (("", P, D), ("_mag", P, D.abs())):
            res["dv" + n] = res["dv" + n] + sums(back, w.T, y)
    return res


def agree(got, ref, bound, what):
    """Not finite in the same places, and within the bound elsewhere."""
    g, r = got.double(), ref
    assert torch.equal(torch.isfinite(g), torch.isfinite(r)), (what, int((torch.isfinite(g) != torch.isfinite(r)).sum()))
    err = torch.where(torch.isfinite(r), (g - r).abs(), 0.0)
    bad = ~(err <= bound) & torch.isfinite(r)
    assert not bool(bad.any()), (what, float(err.max()))


def rounding(dh, n):
    return U32 * ((dh + 4) * 16 + n + dh + 16)


def bound(ref, dt, dh, n):
    """As in attention_bounds: weights rounded to the storage type (bf16), the result once, and fp32 sums; scores of
    standard normal rows are below 16 in magnitude here."""
    e = rounding(dh, n)
    return HALF[dt] * (ref["out"].abs() + (ref["mag"] if dt == torch.bfloat16 else 0)) + e * ref["mag"]


def spoil_values(v, b, h, N, first, row):
    """An infinity of either sign, NaN, and both infinities in one column, at keys spread from ``first`` on; a row of NaN."""
    at = [first + (N - first) * i // 6 for i in range(6)]
    v[b, h, at[0], 1], v[b, h, at[1], 2], v[b, h, at[2], 3] = math.inf, -math.inf, math.nan
    v[b, h, at[3], 4], v[b, h, at[4], 4] = math.inf, -math.inf
    if row:
        v[b, h, at[5]] = math.nan


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", [*CASES, WIDE], ids=[*IDS, "wide"])
def test_values_reach_the_rows_that_see_them(case, dtype):
    B, Hq, Hkv, dh, Q, N, window, sinks = case
    shape, x, dt = setup(case, dtype, 1)
    G, b, hk = Hq // Hkv, B - 1, Hkv - 1
    clean = ops.window_attention(shape, x["q"], x["k"], x["v"])
    see = mask_of(Q, N, Q, N, window, sinks, "cuda")
    for first, row in ((0, True), (N // 2, True), (0, False), (N // 2, False)):
        y = {**x, "v": x["v"].clone()}
        spoil_values(y["v"], b, hk, N, first, row)
        out, lse = ops.window_attention(shape, y["q"], y["k"], y["v"])
        # m ln 2 + log l, in the second walk with another m, up to 24 away in log2 units.  Either has 6 roundings of
        # terms of at most |lse| + 24, and those of the exponentials' arguments, half a step of numbers below 64
        assert bool(((lse - clean[1]).abs() <= 2 * U32 * (6 * (clean[1].abs() + 24) + 64 * math.log(2))).all())
        for h in range(hk * G, (hk + 1) * G):
            ref = formula(y, b, h, G, see)
            agree(out[b, h], ref["out"], bound(ref, dt, dh, N), (case, h))
            for s in (math.inf, -math.inf):
                assert torch.equal(out[b, h].double() == s, ref["out"] == s)
        rest = torch.ones(B, Hq, dtype=torch.bool, device="cuda")
        rest[b, hk * G:(hk + 1) * G] = False
        assert torch.equal(out[rest], clean[0][rest])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_keys_and_queries_reach_the_rows_that_see_them(case, dtype):
    """NaN in a key; an infinity in one, which takes the weight of rows that it is against; NaN in a query."""
    B, Hq, Hkv, dh, Q, N, window, sinks = case
    shape, x, dt = setup(case, dtype, 2)
    G, b, hk = Hq // Hkv, B - 1, Hkv - 1
    see = mask_of(Q, N, Q, N, window, sinks, "cuda")
    for j, what in ((N - 1 - N // 5, math.nan), (N // 3, math.inf), (N - 1, -math.inf), (0, math.inf)):
        y = {**x, "k": x["k"].clone(), "q": x["q"].clone()}
        y["k"][b, hk, j, 5] = what
        y["q"][b, hk * G, Q // 2, 6] = math.nan
        out, lse = ops.window_attention(shape, y["q"], y["k"], y["v"])
        for h in range(hk * G, (hk + 1) * G):
            ref = formula(y, b, h, G, see)
            agree(out[b, h], ref["out"], bound(ref, dt, dh, N), (case, h, j))
            assert torch.equal(torch.isnan(lse[b, h]), torch.isnan(ref["lse"]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_sums_of_the_largest_values_are_finite(case, dtype):
    """Values of up to 3e38: weights that reach 2^8 within the walk would take their sums past the type's range."""
    B, Hq, Hkv, dh, Q, N, window, sinks = case
    shape, x, dt = setup(case, dtype, 6)
    x["v"] = (x["v"].sign() * 3e38 * torch.linspace(0.1, 1.0, dh, device="cuda")).to(dt)
    out, _ = ops.window_attention(shape, x["q"], x["k"], x["v"])
    see = mask_of(Q, N, Q, N, window, sinks, "cuda")
    for h in range(Hq):
        ref = formula(x, 0, h, Hq // Hkv, see)
        agree(out[0, h], ref["out"], bound(ref, dt, dh, N), (case, h))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=IDS)
@pytest.mark.parametrize("size", [1e4, 1e6, 1e15])
def test_the_largest_score_takes_the_row(case, dtype, size):
    """Scores of 1e9 to 1e31, whose products with the scale are rounded by far more than an exponential may be off: a row
    is the value of its largest score (the next is further away than the roundings of a score, 2^-17 of its size)."""
    B, Hq, Hkv, dh, Q, N, window, sinks = case
    shape, x, dt = setup(case, dtype, 11)
    q, k = (x["q"].float() * size).to(dt), (x["k"].float() * size).to(dt)
    out, lse = ops.window_attention(shape, q, k, x["v"])
    see = mask_of(Q, N, Q, N, window, sinks, "cuda")
    for h in range(Hq):
        s = (q[0, h].double() @ k[0, h // (Hq // Hkv)].double().T / math.sqrt(dh)).masked_fill(~see, -math.inf)
        top = s.topk(min(2, N), 1)
        clear = see.any(1) & ((top.values[:, 0] - top.values[:, -1]) > 2.0 ** -17 * top.values[:, 0].abs())
        assert int(clear.sum()) >= int(see.any(1).sum()) * 0.9
        r = x["v"][0, h // (Hq // Hkv)].double()[top.indices[:, 0]]
        assert bool(((out[0, h].double() - r).abs() <= 2 * HALF[dt] * r.abs())[clear].all())
        assert bool(((lse[0, h].double() - top.values[:, 0]).abs() <= 2.0 ** -17 * top.values[:, 0].abs())[clear].all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_past_the_lengths_are_zero_whatever_the_others_hold(dtype):
    case = (2, 4, 2, 64, 200, 200, 30, 3)
    shape, x, _ = setup(case, dtype, 3)
    lens = torch.tensor([200, 77], dtype=torch.int32, device="cuda")
    x["v"][:, :, 5::9] = math.inf
    x["v"][1, :, 77:] = math.nan
    out, lse = ops.window_attention(shape, x["q"], x["k"], x["v"], q_lens=lens, kv_lens=lens)
    assert not bool(out[1, :, 77:].any()) and bool((lse[1, :, 77:] == -math.inf).all())


def check_gradients(case, y, got, dt, b, hk):
    B, Hq, Hkv, dh, Q, N, window, sinks = case
    G, e = Hq // Hkv, rounding(dh, max(N, Q * Hq // Hkv))
    ref = gradients(y, b, hk, G, mask_of(Q, N, Q, N, window, sinks, "cuda"), dt)
    for n, t in (("dk", got[1]), ("dv", got[2])):
        off = ref["dk_d"] if n == "dk" else HALF[dt] * ref["dv_mag"] * (dt == torch.bfloat16)
        agree(t[b, hk], ref[n], HALF[dt] * ref[n].abs() + off + 3 * e * ref[n + "_mag"], (n, case))
    for h in range(hk * G, (hk + 1) * G):
        r = ref["dq", h]
        agree(got[0][b, h], r, HALF[dt] * r.abs() + ref["dq_d", h] + 3 * e * ref["dq_mag", h], ("dq", h, case))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", [*CASES, WIDE], ids=[*IDS, "wide"])
@pytest.mark.parametrize("what", ["v", "k", "k_inf", "q", "do", "do_inf"])
def test_gradients_of_what_pairs_with_them(case, dtype, what):
    """A value that is not finite reaches the gradients of its row, of what pairs with that, and of no others."""
    B, Hq, Hkv, dh, Q, N, window, sinks = case
    shape, x, dt = setup(case, dtype, 5)
    G, b, hk = Hq // Hkv, B - 1, Hkv - 1
    clean = ops.window_attention(shape, x["q"], x["k"], x["v"])
    cg = ops.window_attention_backward(shape, x["q"], x["k"], x["v"], *clean, x["do"])
    name = what.split("_")[0]
    value = math.inf if what.endswith("inf") else math.nan
    T = N if name in ("k", "v") else Q
    for j in sorted({0, T // 3, T - 1}):
        y = {**x, name: x[name].clone()}
        y[name][b, hk if name in ("k", "v") else hk * G, j, 5] = value
        if name == "v":
            y[name][b, hk, j, 6] = -math.inf
        out, lse = ops.window_attention(shape, y["q"], y["k"], y["v"])
        got = ops.window_attention_backward(shape, y["q"], y["k"], y["v"], out, lse, y["do"])
        check_gradients(case, y, got, dt, b, hk)
        for t, c, H, n in ((got[0], cg[0], Hq, G), (got[1], cg[1], Hkv, 1), (got[2], cg[2], Hkv, 1)):
            rest = torch.ones(B, H, dtype=torch.bool, device="cuda")
            rest[b, hk * n:(hk + 1) * n] = False
            assert torch.equal(t[rest], c[rest])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sinks", [(30, 3), (0, 0), (20, 70)])
def test_gradients_past_the_lengths_are_zero_whatever_the_others_hold(dtype, window, sinks):
    case = (2, 8, 2, 64, 200, 200, window, sinks)
    shape, x, _ = setup(case, dtype, 3)
    lens = torch.tensor([200, 77], dtype=torch.int32, device="cuda")
    for n in ("q", "k", "v", "do"):
        y = {**x, n: x[n].clone()}
        y[n][:, :, 5::9] = math.inf
        y[n][1, :, 77:] = math.nan
        out, lse = ops.window_attention(shape, y["q"], y["k"], y["v"], q_lens=lens, kv_lens=lens)
        for t in ops.window_attention_backward(shape, y["q"], y["k"], y["v"], out, lse, y["do"], q_lens=lens, kv_lens=lens):
            assert not bool(t[1, :, 77:].any())


def best_time(f, n=9):
    f()
    torch.cuda.synchronize()
    times = []
    for _ in range(n):
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        f()
        b.record()
        b.synchronize()
        times.append(a.elapsed_time(b))
    return min(times)


# calls of some tenths of a millisecond
TIMED = [(1, 16, 4, 128, 4096, 4096, 0, 0), (2, 8, 8, 64, 8192, 8192, 1000, 4), (16, 32, 8, 128, 1, 16384, 0, 0)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", TIMED, ids=[f"{c[3]}x{c[4]}of{c[5]}w{c[6]}" for c in TIMED])
def test_a_diverged_call_takes_no_longer_than_a_few_others(case, dtype):
    """All of a tensor NaN, or one early value that every later row sees: two walks, in the second of which the tiles that
    are seen in part (2 or 3 of a row block's) are visited twice; nothing is done key by key."""
    shape, x, _ = setup(case, dtype, 4)
    scratch = ops.alloc_attn_scratch(shape)
    out, lse = ops.window_attention(shape, x["q"], x["k"], x["v"], scratch=scratch)

    def call(y):
        return lambda: ops.window_attention(shape, y["q"], y["k"], y["v"], out=out, lse=lse, scratch=scratch)
    base = best_time(call(x))
    for names in (("q", "k", "v"), ("v",), ("k",)):
        y = {**x, **{n: torch.full_like(x[n], math.nan) for n in names}}
        assert best_time(call(y)) <= 4 * base, names
        assert bool(torch.isnan(out).all())
    y = {**x, "v": x["v"].clone()}
    y["v"][:, :, 0, 3] = math.inf
    assert best_time(call(y)) <= 4 * base


TIMED_BACK = [(1, 16, 4, 128, 4096, 4096, 0, 0), (2, 8, 8, 64, 8192, 8192, 1000, 4), (1, 24, 8, 64, 4096, 4096, 0, 0)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", TIMED_BACK, ids=[f"{c[3]}x{c[4]}of{c[5]}w{c[6]}g{c[1] // c[2]}" for c in TIMED_BACK])
def test_a_diverged_backward_takes_no_longer_than_a_few_others(case, dtype):
    """Two walks, and in the second two barriers and two visits more of tiles that pair in part (all of them where a
    group does not divide a tile)."""
    shape, x, _ = setup(case, dtype, 7)
    scratch = ops.alloc_attn_scratch(shape)
    d = [torch.empty_like(x[n]) for n in ("q", "k", "v")]

    def call(y):
        out, lse = ops.window_attention(shape, y["q"], y["k"], y["v"], scratch=scratch)
        return lambda: ops.window_attention_backward(shape, y["q"], y["k"], y["v"], out, lse, y["do"], dq=d[0], dk=d[1],
                                                     dv=d[2], scratch=scratch)
    base = best_time(call(x))
    for names in (("q", "k", "v", "do"), ("do",), ("v",)):
        y = {**x, **{n: torch.full_like(x[n], math.nan) for n in names}}
        assert best_time(call(y)) <= 6 * base, names
        assert bool(torch.isnan(d[0]).all()) and bool(torch.isnan(d[1]).all())
    for n in ("v", "k", "do", "q"):
        y = {**x, n: x[n].clone()}
        y[n][:, :, -1 if n in ("do", "q") else 0, 3] = math.inf
        assert best_time(call(y)) <= 6 * base, n


# ---------------------------------------------------------------------------
# attention over the 4-bit cache
# ---------------------------------------------------------------------------
# B, Hq, Hkv, dh, Q, N, page, window, sinks
CACHED = [
    (1, 4, 2, 64, 1, 2500, 16, 0, 0),      # one token, its positions in parts
    (2, 8, 2, 128, 5, 2300, 64, 0, 0),     # 20 rows to a key head
    (1, 12, 1, 32, 3, 2100, 48, 0, 0),     # 36
    (1, 8, 1, 32, 1, 2100, 16, 1500, 4),
    (1, 6, 2, 64, 17, 300, 16, 40, 3),
    (2, 4, 4, 128, 40, 200, 16, 24, 70),
]
CIDS = [f"{c[0]}x{c[1]}/{c[2]}x{c[3]}-{c[4]}of{c[5]}-w{c[7]}s{c[8]}" for c in CACHED]


def cached(case, dtype, seed):
    """Shapes, a cache of random rows with pages in any order, what it holds, and the call."""
    B, Hq, Hkv, dh, Q, N, ps, window, sinks = case
    shape, x, dt = setup((B, Hq, Hkv, dh, Q, N, window, sinks), dtype, seed)
    per = -(-N // ps)
    cs = ops.make_cache_shape(B, Hkv, dh, B * per, ps, per, dtype)
    g = torch.Generator().manual_seed(seed)
    table = torch.randperm(B * per, generator=g).view(B, per).to(torch.int32).cuda()
    cache = ops.alloc_cache4(cs)
    lens = torch.full((B,), N, dtype=torch.int32, device="cuda")

    def call(k, v, q=x["q"]):
        cache.fill_(0xff)  # what was there before means nothing
        ops.cache4_append(cs, cache, table, None, k, v)
        lse = torch.empty(B, Hq, Q, dtype=torch.float32, device="cuda")
        return ops.cache4_attention(shape, cs, q, cache, table, lens, lse=lse), lse
    return x, dt, call, (shape, cs, cache, table, lens)


def check_cached(case, y, out, lse, dt, b):
    B, Hq, Hkv, dh, Q, N, ps, window, sinks = case
    see = mask_of(Q, N, Q, N, window, sinks, "cuda")
    (kh, ks), (vh, vs) = cache64(y["k"]), cache64(y["v"])
    held = {"q": y["q"], "k": kh, "v": vh}
    # a score adds up q times m and s code apart
    smag = float((y["q"].double().abs().amax((0, 1, 2)) * ks.nan_to_num(0).amax((0, 1, 2))).sum()) / math.sqrt(dh)
    e = U32 * ((dh + 4) * smag + N + dh + 16)
    for h in range(Hq):
        ref = formula(held, b, h, Hq // Hkv, see)
        mag = sums(see, ref["P"], vs[b, h // (Hq // Hkv)])
        off = HALF[dt] * (ref["out"].abs() + (mag if dt == torch.bfloat16 else 0)) + e * mag
        agree(out[b, h], ref["out"], off, (case, h))
        some = torch.isfinite(ref["lse"])
        assert torch.equal(torch.isnan(lse[b, h]), torch.isnan(ref["lse"]))
        assert bool(((lse[b, h].double() - ref["lse"]).abs() <= e * (1 + ref["lse"].abs()))[some].all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CACHED, ids=CIDS)
def test_cached_rows_reach_the_queries_that_see_them(case, dtype):
    """A group of values that is not finite stands for NaN throughout, in K for every column of the rows that see it."""
    B, Hq, Hkv, dh, Q, N = case[:6]
    x, dt, call, _ = cached(case, dtype, 8)
    for at in ((0, N // 3), (N // 2, N - 1), (N - 2,)):
        y = {**x, "k": x["k"].clone(), "v": x["v"].clone()}
        for n, j in enumerate(at):
            y["v"][:, :, j, (7 + 40 * n) % dh] = math.inf if n else math.nan
        out, lse = call(y["k"], y["v"])
        check_cached(case, y, out, lse, dt, B - 1)
        y["k"][B - 1, 0, at[-1], 3] = math.nan
        out, lse = call(y["k"], y["v"])
        check_cached(case, y, out, lse, dt, B - 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CACHED, ids=CIDS)
def test_cached_rows_of_the_largest_values(case, dtype):
    """Values of up to 3e38, whose scales meet the weights before the codes do; and keys whose scores are about 1e37, of
    which the largest takes the row (its distance to the next is far above a rounding, 1e30)."""
    B, Hq, Hkv, dh, Q, N, ps, window, sinks = case
    x, dt, call, _ = cached(case, dtype, 9)
    v = (x["v"][..., :1].sign() * 3e38 * torch.linspace(0.1, 1.0, dh, device="cuda")).to(dt)
    out, lse = call(x["k"], v)
    check_cached(case, {**x, "v": v}, out, lse, dt, B - 1)
    k = (x["k"].float() * 5e36).to(dt)
    out, lse = call(k, x["v"])
    see = mask_of(Q, N, Q, N, window, sinks, "cuda")
    kh, (vh, vs) = cache64(k)[0], cache64(x["v"])
    G = Hq // Hkv
    for h in range(Hq):
        s = (x["q"][B - 1, h].double() @ kh[B - 1, h // G].T).masked_fill(~see, -math.inf)
        best = s.argmax(1)
        r = vh[B - 1, h // G][best]
        assert bool(((out[B - 1, h].double() - r).abs() <= 2 * HALF[dt] * (r.abs() + vs[B - 1, h // G][best])).all())


TIMED_CACHE = [(4, 32, 8, 128, 1, 16000, 64, 0, 0), (2, 16, 4, 64, 64, 8000, 64, 0, 0), (4, 12, 4, 32, 8, 8000, 16, 4000, 4)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", TIMED_CACHE, ids=[f"{c[3]}x{c[4]}of{c[5]}w{c[7]}" for c in TIMED_CACHE])
def test_a_diverged_cache_takes_no_longer(case, dtype):
    """One walk, whatever the cache holds."""
    x, _, call, (shape, cs, cache, table, lens) = cached(case, dtype, 10)
    scratch, out = ops.alloc_attn_scratch(shape), torch.empty_like(x["q"])

    def attend():
        ops.cache4_attention(shape, cs, x["q"], cache, table, lens, out=out, scratch=scratch)
    call(x["k"], x["v"])
    base = best_time(attend)
    for names in (("v",), ("k", "v")):
        y = {**x, **{n: torch.full_like(x[n], math.nan) for n in names}}
        call(y["k"], y["v"])
        assert best_time(attend) <= 2 * base, names
        assert bool(torch.isnan(out).all())


def test_second_walks_beside_other_calls_and_in_graphs():
    """Calls that walk twice on one stream, ordinary ones on another, and both captured: the bits of a call alone."""
    case = (2, 8, 2, 64, 400, 400, 90, 5)
    shape, x, _ = setup(case, "bf16", 12)
    y = {**x, "v": x["v"].clone(), "do": x["do"].clone()}
    spoil_values(y["v"], 1, 1, 400, 10, False)
    y["do"][0, 3, 50, 7] = math.inf

    def call(z, stream=None):
        o = ops.window_attention(shape, z["q"], z["k"], z["v"], stream=stream)
        return (*o, *ops.window_attention_backward(shape, z["q"], z["k"], z["v"], *o, z["do"], stream=stream))

    def same(a, b):
        return all(torch.equal(s.nan_to_num(7.0, 8.0, 9.0), t.nan_to_num(7.0, 8.0, 9.0)) for s, t in zip(a, b))
    want = [call(x), call(y)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        got = [[], []]
        for _ in range(4):
            for i, z in enumerate((x, y)):
                got[i].append(call(z, streams[i]))
        torch.cuda.synchronize()
        for i in range(2):
            assert all(same(g, want[i]) for g in got[i])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = [call(x), call(y)]
    for _ in range(3):
        for t in (*held[0], *held[1]):
            t.fill_(5)
        graph.replay()
        torch.cuda.synchronize()
        assert same(held[0], want[0]) and same(held[1], want[1])
        assert same(call(y), want[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Q,lens", [(1, (50, 1, 100)), (6, (50, 6, 100)), (40, (50, 41, 100))])
@pytest.mark.parametrize("bits", [0x7e, 0x7f, 0xff, 0x80])
def test_what_the_cache_never_held_may_be_any_bits(dtype, Q, lens, bits):
    """Positions past the lengths that were never written: numbers near the type's end, NaN, and a page that no table names."""
    B, Hq, Hkv, dh, N, ps = 3, 4, 2, 64, 112, 16
    shape, x, dt = setup((B, Hq, Hkv, dh, Q, N, 20, 2), dtype, 13)
    per = N // ps
    cs = ops.make_cache_shape(B, Hkv, dh, B * per + 1, ps, per, dtype)
    table = (1 + torch.arange(B * per, dtype=torch.int32, device="cuda")).view(B, per)
    kl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    table[0, 2] = -1
    got = []
    for fill in (0, bits):
        cache = ops.alloc_cache4(cs)
        cache.fill_(fill)
        ops.cache4_append(cs, cache, table, None, x["k"], x["v"], lens=kl)
        lse = torch.empty(B, Hq, Q, dtype=torch.float32, device="cuda")
        got.append((ops.cache4_attention(shape, cs, x["q"], cache, table, kl, q_lens=kl.clamp(max=Q), lse=lse), lse))
    assert bool(torch.isfinite(got[0][0].float()).all())
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
