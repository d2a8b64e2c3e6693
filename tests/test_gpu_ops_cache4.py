"""The 4-bit cache: rows written and read back, and attention over it, against the 64-bit form."""
import math

import pytest
import torch

from ops_util import attention64, attention_bounds, cache64, mask_of, rand_rows, within
from paper_2505_00315_amd import ops

pytestmark = pytest.mark.gpu


def make(B, Hkv, dh, N, ps, dtype, seed, spare=3, extra_pages=0):
    per = -(-N // ps) + extra_pages
    cs = ops.make_cache_shape(B, Hkv, dh, B * per + spare, ps, per, dtype)
    g = torch.Generator().manual_seed(seed)
    table = torch.randperm(B * per + spare, generator=g)[: B * per].view(B, per).to(torch.int32).cuda()
    cache = ops.alloc_cache4(cs)
    cache.fill_(0xff)  # what was there before means nothing: scales and minima of NaN
    return cs, cache, table, g


def dt_of(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("ps", [16, 48, 64])
def test_rows_come_back_as_the_values_held(dh, dtype, ps):
    B, H, N = 2, 3, 150
    cs, cache, table, g = make(B, H, dh, N, ps, dtype, 1)
    k, v = (rand_rows(g, B, H, N, dh, dt_of(dtype), "bthd", 3.0) for _ in range(2))
    ops.cache4_append(cs, cache, table, None, k, v)
    for got, x in zip(ops.cache4_read(cs, cache, table, None, rows=N), (k, v)):
        assert torch.equal(got, cache64(x)[0].float().to(got.dtype))  # m + s code is rounded once, from fp32


@pytest.mark.parametrize("dh", [32, 64, 128])
def test_values_at_borders_and_extremes(dh):
    """Midpoints between codes, one value throughout, signed zeros, tiny and huge spreads, values that are not finite."""
    H, N = 1, 12
    cs, cache, table, g = make(1, H, dh, N, 16, "f32", 2)
    x = torch.zeros(1, H, N, dh)
    x[0, 0, 0] = torch.arange(dh) % 31 * 0.5                 # s = 1: codes and midpoints
    x[0, 0, 1] = 0.75 * (torch.arange(dh) % 31)              # s = 1.5
    x[0, 0, 2] = 2.5
    x[0, 0, 3] = torch.where(torch.arange(dh) % 2 == 0, 0.0, -0.0)
    x[0, 0, 4] = torch.arange(dh) % 32 * 1e-40               # spread below the least scale
    x[0, 0, 5] = torch.randn(dh, generator=g) * 1e37
    x[0, 0, 6, 3] = math.nan
    x[0, 0, 7, dh - 1] = math.inf
    x[0, 0, 8, 0] = -math.inf
    x[0, 0, 9] = torch.where(torch.arange(dh) % 2 == 0, 3e38, -3e38)  # the spread overflows
    x[0, 0, 10] = 1 + torch.arange(dh) * 2.0 ** -20          # m rounds, all below or above it
    x[0, 0, 11] = torch.randn(dh, generator=g) * 1e-30 + (torch.arange(dh) % 32 == 5) * 1.0
    x = x.cuda()
    ops.cache4_append(cs, cache, table, None, x, -x)
    for got, y in zip(ops.cache4_read(cs, cache, table, None, rows=N), (x, -x)):
        want = cache64(y)[0].float()
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        assert torch.equal(got.nan_to_num(7.0), want.nan_to_num(7.0))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [32, 64, 128])
def test_appended_in_pieces(dh, dtype):
    """Token by token, and runs that start and end inside groups of 4 and pages: the bits of one long append."""
    B, H, N, ps = 2, 2, 100, 16
    cs, cache, table, g = make(B, H, dh, N, ps, dtype, 3)
    k, v = (rand_rows(g, B, H, N, dh, dt_of(dtype)) for _ in range(2))
    ops.cache4_append(cs, cache, table, None, k, v)
    other = torch.full_like(cache, 0xff)
    at = 0
    for n in (1, 1, 1, 1, 1, 2, 3, 6, 13, 1, 40, 30):
        start = torch.full((B,), at, dtype=torch.int32, device="cuda")
        ops.cache4_append(cs, other, table, start, k[:, :, at:at + n], v[:, :, at:at + n])
        at += n
    assert at == N and torch.equal(cache, other)


def test_other_rows_stay_as_they_were():
    """Different starts and lengths per sequence; positions and pages that do not exist are dropped."""
    B, H, dh, ps = 5, 2, 64, 16
    cs, cache, table, g = make(B, H, dh, 48, ps, "bf16", 4)
    base, _ = (rand_rows(g, B, H, 48, dh, torch.bfloat16) for _ in range(2))
    ops.cache4_append(cs, cache, table, None, base, base)
    held = ops.cache4_read(cs, cache, table, None, rows=48)[0]
    table = table.clone()
    table[2, 1], table[3, 0], table[3, 1] = -1, cs.pages, 2 ** 31 - 1
    x = rand_rows(g, B, H, 21, dh, torch.bfloat16)
    start = torch.tensor([5, 40, 10, 0, -7], dtype=torch.int32).cuda()
    lens = torch.tensor([9, 21, 21, 99, 21], dtype=torch.int32).cuda()
    before = cache.clone()
    ops.cache4_append(cs, cache, table, start, x, x, lens=lens)
    want = held.clone()
    val = cache64(x)[0].to(torch.bfloat16)
    for b in range(B):
        for t in range(min(int(lens[b]), 21)):
            p = int(start[b]) + t
            if 0 <= p < 48 and 0 <= int(table[b, p // ps]) < cs.pages:
                want[b, :, p] = val[b, :, t]
    full = torch.where((table >= 0) & (table < cs.pages), table, 0)
    got = ops.cache4_read(cs, cache, table, None, rows=48)[0]
    for b in range(B):
        for p in range(48):
            if 0 <= int(table[b, p // ps]) < cs.pages:
                assert torch.equal(got[b, :, p], want[b, :, p]), (b, p)
            else:
                assert not bool(got[b, :, p].any())
    # pages that no table names keep their bytes
    page = cache.view(cs.pages, -1)
    spare = [i for i in range(cs.pages) if i not in set(full.flatten().tolist())]
    assert torch.equal(page[spare], before.view(cs.pages, -1)[spare])
    # rows read past lens, and from positions before the first, are zero
    part = ops.cache4_read(cs, cache, table, start, rows=21, lens=lens)[1]
    assert not bool(part[0, :, 9:].any()) and not bool(part[4, :, :7].any()) and not bool(part[1, :, 8:].any())
    assert torch.equal(part[0, :, :9], val[0, :, :9])


# B, Hq, Hkv, dh, Q, N, page, window, sinks, q_lens, kv_lens
ATTEND = [
    (1, 1, 1, 64, 1, 1, 16, 0, 0, None, [1]),
    (1, 8, 2, 64, 1, 1000, 16, 512, 4, None, [1000]),
    (3, 4, 1, 128, 1, 333, 32, 0, 0, None, [333, 1, 0]),
    (2, 8, 8, 32, 1, 700, 48, 100, 3, None, [700, 650]),
    (2, 6, 2, 64, 5, 260, 16, 40, 2, [5, 3], [260, 17]),
    (2, 4, 2, 128, 17, 150, 64, 0, 0, [17, 17], [150, 10]),     # queries before the first key see nothing
    (1, 16, 1, 128, 3, 500, 16, 64, 70, None, [471]),
    (1, 4, 4, 32, 64, 300, 16, 33, 5, None, [300]),
    (1, 5, 1, 64, 40, 90, 16, 0, 0, [31], [90]),
    (2, 32, 8, 128, 1, 5000, 64, 0, 0, None, [5000, 4099]),
    (1, 2, 2, 64, 1, 4500, 1024, 3000, 4, None, [4500]),
    (1, 24, 1, 32, 2, 2000, 16, 0, 0, None, [1999]),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", ATTEND, ids=[f"{c[0]}x{c[1]}/{c[2]}x{c[3]}-{c[4]}of{c[5]}-w{c[7]}s{c[8]}" for c in ATTEND])
def test_attention(case, dtype):
    B, Hq, Hkv, dh, Q, N, ps, window, sinks, ql, kl = case
    cs, cache, table, g = make(B, Hkv, dh, N, ps, dtype, 5)
    dt = dt_of(dtype)
    k, v = (rand_rows(g, B, Hkv, N, dh, dt, "bhtd", 1.0) for _ in range(2))
    k += 2.0 * torch.randn(1, Hkv, 1, dh, generator=g).cuda().to(dt)  # minima away from zero
    q = rand_rows(g, B, Hq, Q, dh, dt, "bthd", 0.7)
    kv_lens = torch.tensor(kl, dtype=torch.int32).cuda()
    q_lens = None if ql is None else torch.tensor(ql, dtype=torch.int32).cuda()
    ops.cache4_append(cs, cache, table, None, k, v, lens=kv_lens)
    shape = ops.make_attn_shape(B, Hq, Hkv, Q, N, dh, dtype, window=window, sinks=sinks)
    lse = torch.empty(B, Hq, Q, dtype=torch.float32, device="cuda")
    out = ops.cache4_attention(shape, cs, q, cache, table, kv_lens, q_lens=q_lens, lse=lse)
    (kh, ks), (vh, vs) = cache64(k), cache64(v)
    ref = attention64(q, kh, vh, window, sinks, q_lens, kv_lens, spread=vs)
    # a score adds up q times m and s code apart: |q| (|m| + |k|)
    ref["smag"] = max(ref["smag"], float((q.double().abs().amax((0, 1, 2)) * ks.amax((0, 1, 2))).sum()) / math.sqrt(dh))
    bounds = attention_bounds(ref, dt, dh, N)
    within(out, ref["out"], bounds["out"], f"out {case}")
    within(lse, ref["lse"], bounds["lse"], f"lse {case}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Q", [1, 6, 40])
def test_unseen_positions_stay_out(dtype, Q):
    """Keys that hold NaN reach the queries that see them and no others; bad pages are keys that nobody sees."""
    B, Hq, Hkv, dh, N, ps, window, sinks = 1, 4, 2, 64, 200, 16, 24, 3
    cs, cache, table, g = make(B, Hkv, dh, N, ps, dtype, 6)
    dt = dt_of(dtype)
    k, v = (rand_rows(g, B, Hkv, N, dh, dt) for _ in range(2))
    q = rand_rows(g, B, Hq, Q, dh, dt)
    kl = torch.tensor([N - 5], dtype=torch.int32).cuda()
    shape = ops.make_attn_shape(B, Hq, Hkv, Q, N, dh, dtype, window=window, sinks=sinks)
    see = mask_of(Q, N, Q, N - 5, window, sinks).cuda()
    ops.cache4_append(cs, cache, table, None, k, v)
    clean = ops.cache4_attention(shape, cs, q, cache, table, kl)
    tol = 2 ** -7 if dtype == "bf16" else 2 ** -16
    for j in (N - 6, N - 5, N - 6 - window, N - 5 - window, 3, 0, 100):
        k2, v2 = k.clone(), v.clone()
        k2[:, :, j, 7], v2[:, :, j, 9] = math.nan, math.inf
        ops.cache4_append(cs, cache, table, None, k2, v2)
        got = ops.cache4_attention(shape, cs, q, cache, table, kl)
        free = ~see[:, j]
        assert bool(torch.isfinite(got[:, :, free].float()).all()), j
        torch.testing.assert_close(got[:, :, free].float(), clean[:, :, free].float(), rtol=tol, atol=tol)
        assert bool(torch.isnan(got[:, :, ~free].float()).any(-1).all()), j
    ops.cache4_append(cs, cache, table, None, k, v)
    bad = table.clone()
    hole = [0, 8, 11]  # pages of sinks, of nothing that the last query sees, of its window
    for i, e in enumerate((-1, cs.pages, -2 ** 31)):
        bad[0, hole[i]] = e
    got = ops.cache4_attention(shape, cs, q, cache, bad, kl)
    lost = see.clone()
    for e in hole:
        lost[:, e * ps:(e + 1) * ps] = False
    kh, vh = cache64(k)[0], cache64(v)[0]
    for h in range(Hq):
        s = (q[0, h].double() @ kh[0, h // 2].T / 8).masked_fill(~lost, -math.inf)
        some = lost.any(1)
        want = torch.where(some[:, None], torch.softmax(s.masked_fill(~some[:, None], 0.0), 1) @ vh[0, h // 2], 0.0)
        torch.testing.assert_close(got[0, h].double(), want, rtol=2 * tol, atol=2 * tol)


def test_table_and_cache_beyond_four_gigabytes():
    """A page far into a cache of more than 2^32 bytes."""
    Hkv, dh, ps = 8, 128, 64
    page = Hkv * ps * (dh + dh // 4)
    pages = (1 << 32) // page + 40
    cs = ops.make_cache_shape(1, Hkv, dh, pages, ps, 2)
    cache = torch.empty(ops.cache4_size(cs), dtype=torch.uint8, device="cuda")
    table = torch.tensor([[pages - 1, 1]], dtype=torch.int32, device="cuda")
    g = torch.Generator().manual_seed(7)
    k, v = (rand_rows(g, 1, Hkv, 100, dh, torch.bfloat16) for _ in range(2))
    ops.cache4_append(cs, cache, table, None, k, v)
    got = ops.cache4_read(cs, cache, table, None, rows=100)
    assert torch.equal(got[0], cache64(k)[0].to(torch.bfloat16))
    q = rand_rows(g, 1, Hkv, 1, dh, torch.bfloat16)
    shape = ops.make_attn_shape(1, Hkv, Hkv, 1, 128, dh)
    out = ops.cache4_attention(shape, cs, q, cache, table, torch.tensor([100], dtype=torch.int32, device="cuda"))
    ref = attention64(q, cache64(k)[0], cache64(v)[0], 0, 0, spread=cache64(v)[1])
    within(out, ref["out"], attention_bounds(ref, torch.bfloat16, dh, 100)["out"], "out")


@pytest.mark.parametrize("Q,N,window", [(1, 3000, 0), (1, 200, 50), (30, 700, 100)])
def test_same_bits_again_beside_and_captured(Q, N, window):
    B, Hq, Hkv, dh, ps = 2, 8, 2, 64, 32
    cs, cache, table, g = make(B, Hkv, dh, N, ps, "bf16", 8)
    shape = ops.make_attn_shape(B, Hq, Hkv, Q, N, dh, window=window, sinks=4)
    q = rand_rows(g, B, Hq, Q, dh, torch.bfloat16)
    k, v = (rand_rows(g, B, Hkv, N, dh, torch.bfloat16) for _ in range(2))
    kl = torch.tensor([N, N - 7], dtype=torch.int32).cuda()
    scratch, out = ops.alloc_attn_scratch(shape), torch.empty_like(q)
    ops.cache4_append(cs, cache, table, None, k, v)
    first = ops.cache4_attention(shape, cs, q, cache, table, kl)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = ops.cache4_attention(shape, cs, q, cache, table, kl, stream=side)
    again = ops.cache4_attention(shape, cs, q, cache, table, kl)
    torch.cuda.synchronize()
    assert torch.equal(first, other) and torch.equal(first, again)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ops.cache4_append(cs, cache, table, None, k, v)
        ops.cache4_attention(shape, cs, q, cache, table, kl, out=out, scratch=scratch)
    for seed in range(3):
        h = torch.Generator().manual_seed(40 + seed)
        for t in (q, k, v):
            t.copy_(rand_rows(h, *t.shape, torch.bfloat16))
        out.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        ops.cache4_append(cs, cache, table, None, k, v)
        want = ops.cache4_attention(shape, cs, q, cache, table, kl)
        torch.cuda.synchronize()
        assert torch.equal(got, want)
