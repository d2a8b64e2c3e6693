"""Plain 64-bit forms of the dense heads' operators, and how far a kernel of a
storage type may be from them.

A rounding to a type moves a value by at most half a step, eps / 2 of it.  The
bounds below add up the roundings that the operators make:

* bf16 attention rounds the weights p (or p times a scale) and the weighted
  differences ds to bf16 where they enter a matrix product, and every result
  once; all sums are fp32.
* fp32: a sum of n products is off by at most n u times the sum of the
  magnitudes, u = 2^-24; an exponential by the error of its argument, itself a
  sum over d_head products, and a few u.
"""
import math

import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
U32 = 2.0 ** -24


def rand_rows(g, B, H, T, dh, dtype, layout="bhtd", scale=1.0):
    """Random rows [B, H, T, dh] in one of the memory orders that callers use."""
    def normal(*s):
        return (torch.randn(s, generator=g, dtype=torch.float32) * scale).to(dtype).cuda()
    if layout == "bhtd":
        return normal(B, H, T, dh)
    if layout == "bthd":
        return normal(B, T, H, dh).transpose(1, 2)
    if layout == "packed":  # one of three parts of packed rows, as the layer keeps them
        return normal(B, H, T, 3, dh)[:, :, :, 1]
    raise ValueError(layout)


def mask_of(T, N, qn, kn, window, sinks, device="cpu"):
    """[T, N] truth values: query i of a sequence with qn queries and kn keys sees key j."""
    i = torch.arange(T, device=device)[:, None]
    j = torch.arange(N, device=device)[None]
    p = kn - qn + i
    m = (j <= p) & (j < kn) & (i < qn)
    if window:
        m &= (p - j < window) | (j < sinks)
    return m


def attention64(q, k, v, window, sinks, q_lens=None, kv_lens=None, scale=None, do=None, spread=None):
    """Attention in 64 bits.  Returns a dict of out and lse, dq, dk, dv where do
    is given, and for each of them the bound's terms ("<name>_mag": the sum of
    the magnitudes of its products, "ds..." ).  ``spread`` [B, Hkv, N, dh]: what
    stands for |v| where the kernel's products are larger than v (a cache that
    holds v as m + s code)."""
    B, Hq, T, dh = q.shape
    Hkv, N = k.shape[1], k.shape[2]
    G = Hq // Hkv
    scale = 1 / math.sqrt(dh) if scale is None else scale
    dev = q.device
    res = {n: torch.zeros(B, Hq, T, dh, dtype=torch.float64, device=dev) for n in ("out", "out_mag")}
    res["lse"] = torch.full((B, Hq, T), -math.inf, dtype=torch.float64, device=dev)
    res["smag"] = 0.0
    if do is not None:
        for n in ("dq", "dq_mag", "dq_d"):
            res[n] = torch.zeros(B, Hq, T, dh, dtype=torch.float64, device=dev)
        for n in ("dk", "dv", "dk_mag", "dv_mag", "dk_d"):
            res[n] = torch.zeros(B, Hkv, N, dh, dtype=torch.float64, device=dev)
    half = HALF[q.dtype]
    for b in range(B):
        qn = T if q_lens is None else min(max(int(q_lens[b]), 0), T)
        kn = N if kv_lens is None else min(max(int(kv_lens[b]), 0), N)
        if qn == 0:
            continue
        see = mask_of(T, N, qn, kn, window, sinks, dev)[:qn, :kn]
        for h in range(Hq):
            Q, K, V = q[b, h, :qn].double(), k[b, h // G, :kn].double(), v[b, h // G, :kn].double()
            S = (Q @ K.T * scale).masked_fill(~see, -math.inf)
            some = see.any(1)
            lse = torch.where(some, torch.logsumexp(S.masked_fill(~some[:, None], 0.0), 1) if kn else S.sum(1), -math.inf)
            P = torch.where(see, torch.exp(S - torch.where(some, lse, 0.0)[:, None]), 0.0)
            O = P @ V
            W = V.abs() if spread is None else spread[b, h // G, :kn].double()
            res["out"][b, h, :qn], res["out_mag"][b, h, :qn], res["lse"][b, h, :qn] = O, P @ W, lse
            if kn:
                res["smag"] = max(res["smag"], float((Q.abs() @ K.abs().T).max()) * scale)
            if do is None:
                continue
            D = do[b, h, :qn].double()
            dP = D @ V.T
            dS = P * (dP - (D * O).sum(1, keepdim=True))
            # the forward's out, rounded, stands for O in the backward
            eD = half * (D.abs() * (P @ V.abs() + O.abs())).sum(1, keepdim=True)
            mag = P * (D.abs() @ V.abs().T + (D.abs() * O.abs()).sum(1, keepdim=True))
            res["dq"][b, h, :qn] = dS @ K * scale
            res["dq_mag"][b, h, :qn] = mag @ K.abs() * scale
            res["dq_d"][b, h, :qn] = ((P * eD) + half * dS.abs()) @ K.abs() * scale
            res["dk"][b, h // G, :kn] += dS.T @ Q * scale
            res["dk_mag"][b, h // G, :kn] += mag.T @ Q.abs() * scale
            res["dk_d"][b, h // G, :kn] += ((P * eD) + half * dS.abs()).T @ Q.abs() * scale
            res["dv"][b, h // G, :kn] += P.T @ D
            res["dv_mag"][b, h // G, :kn] += P.T @ D.abs()
    return res


def attention_bounds(ref, dtype, dh, count):
    """Bounds of every result; ``count``: most products of a sum (keys, or
    queries times heads of a group)."""
    half = HALF[dtype]
    # relative error of a weight: its argument (dh products of magnitude smag,
    # scaled to log2 units), the exponential and the division
    e = U32 * (dh * ref["smag"] + 4 * ref["smag"] + count + dh + 16)
    out = {"out": half * (ref["out"].abs() + (ref["out_mag"] if dtype == torch.bfloat16 else 0)) + e * ref["out_mag"],
           "lse": e * (1 + ref["lse"].abs())}
    if "dq" in ref:
        w = 1 if dtype == torch.bfloat16 else 0
        out["dv"] = half * (ref["dv"].abs() + w * ref["dv_mag"]) + e * ref["dv_mag"]
        for n in ("dq", "dk"):
            out[n] = half * ref[n].abs() + ref[n + "_d"] + 3 * e * ref[n + "_mag"]
    return out


def within(got, ref, bound, what):
    """got is within the bound of ref everywhere, and infinite where ref is."""
    g, r = got.double(), ref
    same = torch.isinf(r) & (g == r)
    err = torch.where(same, 0.0, (g - r).abs())
    tiny = 1e-37
    bad = ~(err <= bound + tiny) & ~same
    if bool(bad.any()):
        at = tuple(int(x) for x in bad.nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} outside the bound, first at {at}: "
                             f"{float(g[at])} against {float(r[at])}, bound {float(bound[at])}")


# ---------------------------------------------------------------------------
def norm64(x, w, pos, rope, pairs, base, eps, dy=None):
    """Norm and rotation of rows x [B, H, T, dh] in 64 bits; gradients (dx, dw)
    where dy is given, dw with the sum of its products' magnitudes."""
    x = x.double().requires_grad_(dy is not None)
    wt = torch.ones(x.shape[-1], dtype=torch.float64, device=x.device) if w is None else w.double()
    wt = wt.detach().requires_grad_(dy is not None)
    z = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    n = z * wt
    if rope:
        theta = base ** (-2.0 * torch.arange(rope // 2, dtype=torch.float64, device=x.device) / rope)
        a = pos.double()[:, None, :, None] * theta
        c, s = a.cos(), a.sin()
        if pairs == "adjacent":
            u, v = n[..., 0:rope:2], n[..., 1:rope:2]
            y = torch.stack([u * c - v * s, u * s + v * c], -1).flatten(-2)
        else:
            u, v = n[..., : rope // 2], n[..., rope // 2: rope]
            y = torch.cat([u * c - v * s, u * s + v * c], -1)
        y = torch.cat([y, n[..., rope:]], -1)
    else:
        y = n
    if dy is None:
        return y
    y.backward(dy.double())
    return y.detach(), x.grad, wt.grad


def cache64(x):
    """Values that a 4-bit cache holds for rows x (fp32 steps of the format, borders decided in 64 bits), and |m| + |value|."""
    y = x.float().unflatten(-1, (-1, 32))
    lo, hi = y.amin(-1, keepdim=True), y.amax(-1, keepdim=True)
    m = lo.bfloat16().float()
    s = ((hi - m) * torch.tensor(1 / 15, dtype=torch.float32, device=x.device)).bfloat16().float()
    s = torch.where(s >= 2.0 ** -126, s, 0.0)
    bad = ~(torch.isfinite(y).all(-1, keepdim=True) & torch.isfinite(s) & torch.isfinite(m))
    code = ((y - m).double() / torch.where(s > 0, s, 1.0).double()).round().clamp(0, 15)
    val = m.double() + s.double() * torch.where(s > 0, code, 0.0)
    val = torch.where(bad, math.nan, val).flatten(-2)
    return val, val.abs() + m.double().abs().expand_as(y).flatten(-2)
