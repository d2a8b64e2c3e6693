"""The dense heads' operators as a program runs them: norm and rotation, attention over a prompt, the cache, single
tokens; and beside the layer whose local heads they continue."""
import math

import pytest
import torch

import workloads as wl
from gpu_util import run_forward
from ops_util import attention64, attention_bounds, cache64, rand_rows, within
from paper_2505_00315_amd import mosa, ops

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_then_tokens(dtype):
    """A prompt through attention, its keys into the cache, then tokens one by one: every token's output is that of
    attention over what the cache holds, and close to attention over the rows themselves."""
    B, Hq, Hkv, dh, T, new, window, sinks, ps = 2, 6, 2, 64, 90, 8, 40, 3, 16
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    N = T + new
    g = torch.Generator().manual_seed(1)
    packed = torch.randn(B, N, Hq + 2 * Hkv, dh, generator=g).to(dt).cuda()  # projections of every token
    wq, wk = ((1 + 0.1 * torch.randn(dh, generator=g)).to(dt).cuda() for _ in range(2))
    q, k, v = (t.transpose(1, 2) for t in packed.split([Hq, Hkv, Hkv], 2))
    whole = ops.make_norm_shape(B, N, Hq, Hkv, dh, dtype)
    qn, kn = ops.qk_norm_rope(whole, q, k, wq, wk)
    full = ops.make_attn_shape(B, Hq, Hkv, N, N, dh, dtype, window=window, sinks=sinks)
    want, _ = ops.window_attention(full, qn, kn, v)

    per = -(-N // ps)
    cs = ops.make_cache_shape(B, Hkv, dh, B * per, ps, per, dtype)
    cache = ops.alloc_cache4(cs)
    table = torch.randperm(B * per, generator=g).view(B, per).to(torch.int32).cuda()
    prompt = ops.make_norm_shape(B, T, Hq, Hkv, dh, dtype)
    qp, kp = ops.qk_norm_rope(prompt, q[:, :, :T], k[:, :, :T], wq, wk)
    assert torch.equal(qp, qn[:, :, :T]) and torch.equal(kp, kn[:, :, :T])
    out, _ = ops.window_attention(ops.make_attn_shape(B, Hq, Hkv, T, T, dh, dtype, window=window, sinks=sinks), qp, kp,
                                  v[:, :, :T])
    torch.testing.assert_close(out.float(), want[:, :, :T].float(), rtol=2 ** -7, atol=2 ** -7)
    ops.cache4_append(cs, cache, table, None, kp, v[:, :, :T])
    step, one = ops.make_norm_shape(B, 1, Hq, Hkv, dh, dtype), ops.make_attn_shape(B, Hq, Hkv, 1, N, dh, dtype,
                                                                                  window=window, sinks=sinks)
    kh, vh = cache64(kn), cache64(v)
    for t in range(T, N):
        pos = torch.full((B, 1), t, dtype=torch.int32, device="cuda")
        q1, k1 = ops.qk_norm_rope(step, q[:, :, t:t + 1], k[:, :, t:t + 1], wq, wk, positions=pos)
        assert torch.equal(q1, qn[:, :, t:t + 1]) and torch.equal(k1, kn[:, :, t:t + 1])
        ops.cache4_append(cs, cache, table, pos.view(B), k1, v[:, :, t:t + 1])
        o = ops.cache4_attention(one, cs, q1, cache, table, (pos + 1).view(B))
        ref = attention64(q1, kh[0][:, :, :t + 1], vh[0][:, :, :t + 1], window, sinks, spread=vh[1][:, :, :t + 1])
        ref["smag"] = max(ref["smag"], float((q1.double().abs().amax((0, 1, 2)) * kh[1].amax((0, 1, 2))).sum()) / 8)
        within(o, ref["out"], attention_bounds(ref, dt, dh, N)["out"], f"token {t}")
        wide, _ = ops.window_attention(ops.make_attn_shape(B, Hq, Hkv, 1, t + 1, dh, dtype, window=window, sinks=sinks),
                                       q1, kn[:, :, :t + 1], v[:, :, :t + 1])
        torch.testing.assert_close(wide.float(), want[:, :, t:t + 1].float(), rtol=2 ** -7, atol=2 ** -7)
        # 16 steps over a group's spread: half a step of about 4.5 / 15 on values of spread 1, averaged over the keys
        assert float((o.float() - wide.float()).abs().max()) < 0.5


def test_training_step():
    """Forward and backward through norm, rotation and attention against differentiation in 64 bits (fp32 storage)."""
    B, Hq, Hkv, dh, T, window, sinks = 2, 4, 2, 32, 70, 16, 2
    g = torch.Generator().manual_seed(2)
    x = {n: rand_rows(g, B, h, T, dh, torch.float32, "bthd") for n, h in (("q", Hq), ("k", Hkv), ("v", Hkv))}
    w = {n: (1 + 0.1 * torch.randn(dh, generator=g)).cuda() for n in ("wq", "wk")}
    do = rand_rows(g, B, Hq, T, dh, torch.float32)
    ns = ops.make_norm_shape(B, T, Hq, Hkv, dh, "f32")
    sh = ops.make_attn_shape(B, Hq, Hkv, T, T, dh, "f32", window=window, sinks=sinks)
    qn, kn = ops.qk_norm_rope(ns, x["q"], x["k"], w["wq"], w["wk"])
    out, lse = ops.window_attention(sh, qn, kn, x["v"])
    dqn, dkn, dv = ops.window_attention_backward(sh, qn, kn, x["v"], out, lse, do)
    dq, dk, dwq, dwk = ops.qk_norm_rope_backward(ns, x["q"], x["k"], w["wq"], w["wk"], dqn, dkn)

    leaf = {n: t.double().requires_grad_() for n, t in {**x, **w}.items()}
    theta = 10000.0 ** (-2.0 * torch.arange(dh // 4, dtype=torch.float64, device="cuda") / (dh // 2))
    a = torch.arange(T, device="cuda").double()[:, None] * theta

    def turned(t, wt):
        n = t / torch.sqrt((t * t).mean(-1, keepdim=True) + 1e-6) * wt
        u, v = n[..., 0:dh // 2:2], n[..., 1:dh // 2:2]
        y = torch.stack([u * a.cos() - v * a.sin(), u * a.sin() + v * a.cos()], -1).flatten(-2)
        return torch.cat([y, n[..., dh // 2:]], -1)
    Q, K = turned(leaf["q"], leaf["wq"]), turned(leaf["k"], leaf["wk"])
    i, j = torch.arange(T, device="cuda")[:, None], torch.arange(T, device="cuda")[None]
    hide = (j > i) | ((i - j >= window) & (j >= sinks))
    G = Hq // Hkv
    s = (Q @ K.repeat_interleave(G, 1).transpose(-1, -2).contiguous() / math.sqrt(dh)).masked_fill(hide, -math.inf)
    o = torch.softmax(s, -1) @ leaf["v"].repeat_interleave(G, 1)
    o.backward(do.double())
    # a chain of fp32 sums of at most T G + dh terms: a few hundred u of the tensor's largest value
    for n, got, ref in [("out", out, o.detach()), ("dv", dv, leaf["v"].grad), ("dq", dq, leaf["q"].grad),
                        ("dk", dk, leaf["k"].grad), ("dwq", dwq, leaf["wq"].grad), ("dwk", dwk, leaf["wk"].grad)]:
        err = float((got.double() - ref).abs().max() / ref.abs().max())
        assert err < 400 * 2.0 ** -24, (n, err)


@pytest.mark.parametrize("dh,rope", [(64, True), (32, False)])
def test_beside_the_layer(dh, rope):
    """The layer's local heads and the operators agree: attention over the layer's saved rows gives its head outputs,
    its keys go into the cache as they lie, and norm without weights turns rows as the layer does."""
    T, window = 200, 48
    w = wl.small("beside", batch=2, seq_len=T, d_model=128, heads=2, d_head=dh, k=16, dense_heads=3, rope=rope,
                 window=window)
    inp = wl.make_inputs(w)
    res = run_forward(w, inp)
    shape, saved = res["shape"], res["saved"]
    q, k, v = (mosa.saved_view(shape, saved, n) for n in ("Qd", "Kd", "Vd"))
    sh = ops.make_attn_shape(2, 3, 3, T, T, dh, window=window)
    out, lse = ops.window_attention(sh, q, k, v)
    ref = attention64(q, k, v, window, 0)
    bounds = attention_bounds(ref, torch.bfloat16, dh, window)
    for n, a, b in (("out", out, mosa.saved_view(shape, saved, "Ad")), ("lse", lse, mosa.saved_view(shape, saved, "lsed"))):
        within(a, ref[n], bounds[n], n)
        within(b, ref[n], bounds[n], "the layer's " + n)
    per = -(-T // 32)
    cs = ops.make_cache_shape(2, 3, dh, 2 * per, 32, per)
    cache, table = ops.alloc_cache4(cs), torch.arange(2 * per, dtype=torch.int32, device="cuda").view(2, per)
    ops.cache4_append(cs, cache, table, None, k, v)
    one = ops.make_attn_shape(2, 3, 3, 1, T, dh, window=window)
    last = ops.cache4_attention(one, cs, q[:, :, -1:], cache, table, torch.full((2,), T, dtype=torch.int32, device="cuda"))
    (kh, _), (vh, vs) = cache64(k), cache64(v)
    held = attention64(q[:, :, -1:], kh, vh, window, 0, spread=vs)
    held["smag"] = 4 * held["smag"]
    within(last, held["out"], attention_bounds(held, torch.bfloat16, dh, T)["out"], "last token")
    if rope:
        # unit rows keep their size under the norm up to sqrt(dh): the turned columns are the layer's rotation
        x = torch.zeros(1, 1, T, dh, dtype=torch.float32, device="cuda")
        x[..., 0] = 1.0
        y, _ = ops.qk_norm_rope(ops.make_norm_shape(1, T, 1, 1, dh, "f32", eps=0.0), x, x)
        t = torch.arange(T, device="cuda").double()
        want = torch.stack([t.cos(), t.sin()], 1) * math.sqrt(dh)
        torch.testing.assert_close(y[0, 0, :, :2].double(), want, rtol=1e-6, atol=1e-5)
