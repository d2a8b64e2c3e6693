"""Plain 64-bit forms of the operators around a block, and how far a kernel of a
storage type may be from them.

A rounding to a type moves a value by at most half a step, HALF of it; an fp32
operation by U32.  The bounds add up the roundings that the operators make:

* a sum of n terms, lane by lane and then over lanes, is off by at most its depth (the
  longest chain of additions) times U32 times the sum of the magnitudes;
* a norm's factor 1 / sqrt(mean + eps) by half the mean's error and a few U32;
* bf16 storage rounds each result once, and dy act'(z) where it enters the products.
"""
import math

import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
U32 = 2.0 ** -24
# A row's sum: at most 8 terms (two units of 4) per lane, 6 steps over a wave, 16 waves; its factor, 2 operations and
# a square root each.  Products of up to 4 factors around it.
ROW = 48 * U32


def within(got, ref, bound, what):
    """got is within the bound of ref everywhere, infinite where ref is, and NaN where ref is."""
    g, r = got.double(), ref.double()
    same = (torch.isinf(r) & (g == r)) | (torch.isnan(r) & torch.isnan(g))
    bad = ~((g - r).abs() <= bound + 1e-37) & ~same
    if bool(bad.any()):
        at = tuple(int(x) for x in bad.nonzero()[0])
        b = bound[at] if torch.is_tensor(bound) and bound.shape == r.shape else bound
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} outside the bound, first at {at}: "
                             f"{float(g[at])} against {float(r[at])}, bound {float(b)}")


# ---------------------------------------------------------------------------
# residual stream
# ---------------------------------------------------------------------------
def _wide(gate, x, kind):
    if gate is None:
        return torch.ones_like(x)
    g = gate.double()
    return g[:, None].expand_as(x) if kind == "sequence" else g.expand_as(x)


def residual64(shape, kind, x, y, w_post=None, gate=None, w_pre=None, dh=None, dn=None, grads=False):
    """Results in 64 bits and their bounds: {name: (value, bound)}."""
    dt, d = x.dtype, x.shape[-1]
    half, out = HALF[dt], {}
    X = x.double()
    one = torch.ones(d, dtype=torch.float64, device=x.device)
    wp, wn = (one if w is None else w.double() for w in (w_post, w_pre))
    ra, rb, eps = shape.residual_scale, shape.branch_scale, shape.eps
    if y is None:
        h = hm = X
        hm = X.abs()
    else:
        Y, g = y.double(), _wide(gate, X, kind)
        sy = 1 / torch.sqrt((Y * Y).mean(-1, keepdim=True) + eps) if shape.post_norm else torch.ones_like(X[..., :1])
        zy = Y * sy
        u = zy * wp
        h = ra * X + rb * g * u
        hm = (ra * X).abs() + (rb * g * u).abs()  # what h's roundings are relative to
        out["h"] = (h, half * h.abs() + ROW * hm)
    if shape.pre_norm:
        sh = 1 / torch.sqrt((h * h).mean(-1, keepdim=True) + eps)
        zh, zm = h * sh, hm * sh
        # h's errors in the mean of squares: relative to mean(h hm)
        grow = 1 + (zh.abs() * zm).mean(-1, keepdim=True)
        out["n"] = (zh * wn, half * (zh * wn).abs() + 2 * ROW * grow * zm * wn.abs())
    if not grads:
        return out
    D = torch.zeros_like(X) if dh is None else dh.double()
    Dm = D.abs()
    rows = X.shape[0] * X.shape[1]
    if shape.pre_norm:
        N = dn.double()
        e = N * wn
        c, cm = (e * zh).mean(-1, keepdim=True), (e.abs() * zm).mean(-1, keepdim=True)
        D = D + sh * (e - zh * c)
        Dm = Dm + sh * (e.abs() + zm * cm) * grow
        s, sm = (N * zh).sum((0, 1)), (N.abs() * zm * grow).sum((0, 1))
        out["dw_pre"] = (s, half * s.abs() + (rows * U32 + 3 * ROW) * sm)
    scale = ra if y is not None else 1.0
    out["dx"] = (scale * D, half * (scale * D).abs() + 4 * ROW * abs(scale) * Dm)
    if y is None:
        return out
    dg, dgm = rb * D * u, abs(rb) * Dm * u.abs()
    if gate is not None:
        axes = {"vector": (0, 1), "sequence": (1,), "token": ()}[kind]
        s, sm = (dg.sum(axes), dgm.sum(axes)) if axes else (dg, dgm)
        out["dgate"] = (s, half * s.abs() + (rows * U32 + 6 * ROW) * sm)
    k, km = rb * D * g, abs(rb) * Dm * g.abs()
    if shape.post_norm:
        s, sm = (k * zy).sum((0, 1)), (km * zy.abs()).sum((0, 1))
        out["dw_post"] = (s, half * s.abs() + (rows * U32 + 6 * ROW) * sm)
        e, em = k * wp, km * wp.abs()
        c, cm = (e * zy).mean(-1, keepdim=True), (em * zy.abs()).mean(-1, keepdim=True)
        v, vm = sy * (e - zy * c), sy * (em + zy.abs() * cm)
    else:
        v, vm = k, km
    out["dy"] = (v, half * v.abs() + 8 * ROW * vm)
    return out


# ---------------------------------------------------------------------------
# products
# ---------------------------------------------------------------------------
def act64(z, act):
    if act == "relu":
        return z.clamp_min(0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z / math.sqrt(2)))
    return z * torch.sigmoid(z) if act == "silu" else z


def slope64(z, act):
    if act == "relu":
        return (z > 0).double()
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z / math.sqrt(2))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    s = torch.sigmoid(z)
    return s * (1 + z * (1 - s)) if act == "silu" else torch.ones_like(z)


def linear64(x, w, act, order, bias=None, residual=None):
    """{name: (value, bound)} of y and z.  The slopes of the activations are at most 1.13."""
    half, K = HALF[x.dtype], x.shape[1]
    X, W = x.double(), w.double() if order == "in_out" else w.double().t()
    z, mag = X @ W, X.abs() @ W.abs()
    if bias is not None:
        z, mag = z + bias.double(), mag + bias.double().abs()
    ez = (K + 2) * U32 * mag
    y = act64(z, act)
    if residual is not None:
        y = y + residual.double()
    # (the error function and the exponential: a few units of their result, times z)
    return {"z": (z, half * z.abs() + ez), "y": (y, half * y.abs() + 1.13 * ez + 8 * U32 * z.abs() + U32 * y.abs())}


def linear_grads64(x, w, dy, act, order, z=None):
    half, (M, K), N = HALF[x.dtype], x.shape, dy.shape[1]
    X, W, D = x.double(), w.double() if order == "in_out" else w.double().t(), dy.double()
    ez = torch.zeros_like(D)
    if act != "none":
        Z = z.double()
        ez = D.abs() * 16 * U32 * (1 + Z.abs())  # the slope's terms: up to 1 + |z| in size
        D = D * slope64(Z, act)
    ed = ez + (half * D.abs() if act != "none" and x.dtype == torch.bfloat16 else 0)
    Da = D.abs()
    dx, dw, db = D @ W.t(), X.t() @ D, D.sum(0)
    bx = half * dx.abs() + ed @ W.abs().t() + (N + 2) * U32 * (Da @ W.abs().t())
    bw = half * dw.abs() + X.abs().t() @ ed + (M + 2) * U32 * (X.abs().t() @ Da)
    bb = half * db.abs() + ez.sum(0) + M * U32 * Da.sum(0)
    if order == "out_in":
        dw, bw = dw.t(), bw.t()
    return {"dx": (dx, bx), "dw": (dw, bw), "db": (db, bb)}


# ---------------------------------------------------------------------------
# log probabilities
# ---------------------------------------------------------------------------
def order64(x):
    """Indices of every row's values, largest first, equal ones by index, NaN as -inf."""
    v = torch.where(torch.isnan(x.double()), -math.inf, x.double())
    return torch.sort(v + 0.0, dim=1, descending=True, stable=True).indices  # (-0 as 0)


def logprobs64(x, targets, scale, top=0, d_logp=None, d_lse=None, d_entropy=None):
    """{name: (value, bound)}; rows of -inf alone: log p and lse -inf, entropy and gradients 0; rows with +inf or NaN:
    NaN."""
    half, (R, V) = HALF[x.dtype], x.shape
    x64 = x.double()
    odd = (torch.isnan(x64) | (x64 == math.inf)).any(1)
    none = (x64 == -math.inf).all(1)
    plain = ~(odd | none)
    z = torch.where(plain[:, None], x64, 0.0) * scale
    m = z.amax(1, keepdim=True)
    L = torch.log(torch.exp(z - m).sum(1, keepdim=True))
    logq = z - m - L
    p = torch.exp(logq)
    # an exponential's argument is off by 3 roundings of it (weights below e^-104 are 0); a sum of V terms of one
    # sign by at most the additions of a lane and those over lanes and parts
    far = (m - z).clamp(max=104)
    ew = U32 * (4 * far + 8)
    el = (p * ew).sum(1, keepdim=True) + U32 * (V / 256 + 64)
    eq = U32 * (3 * (m - z).clamp(max=1e30) + 4 * L.abs()) + el

    def rows(v, odd_value, none_value):
        v = torch.where(none.view(-1, *[1] * (v.dim() - 1)), none_value, v)
        return torch.where(odd.view(-1, *[1] * (v.dim() - 1)), odd_value, v)
    out = {"lse": (rows((m + L)[:, 0], math.nan, -math.inf), (el + U32 * (2 * m.abs() + 4 * L.abs()))[:, 0])}
    H = -torch.where(p > 0, p * logq, 0.0).sum(1, keepdim=True)
    eH = (torch.where(p > 0, p * (ew + U32 * (V / 256 + 64)) * (far + 1), 0.0)).sum(1, keepdim=True) + el * (1 + L.abs() + H)
    out["entropy"] = (rows(H[:, 0], math.nan, 0.0), eH[:, 0])
    if targets is not None:
        t = targets.long()
        here = (t >= 0) & (t < V)
        at = t.clamp(0, V - 1)[:, None]
        # (a masked target: -inf - m)
        v = torch.where(here, rows(logq.gather(1, at)[:, 0], math.nan, -math.inf), 0.0)
        out["logp"] = (v, eq.gather(1, at)[:, 0].nan_to_num(posinf=0.0))
    if top:
        order = order64(x)[:, :top]
        out["top_index"] = order
        out["top_logp"] = (rows(logq.gather(1, order), math.nan, -math.inf), eq.gather(1, order))
    if d_logp is None and d_lse is None and d_entropy is None:
        return out

    def grad(t):
        return torch.zeros(R, 1, dtype=torch.float64, device=x.device) if t is None else t.double()[:, None]
    g = torch.where(here[:, None], grad(d_logp), 0.0) if d_logp is not None else grad(None)
    gl, ge = grad(d_lse), grad(d_entropy)
    lq = torch.where(p > 0, logq, 0.0)
    dz = p * (gl - g - ge * (lq + H))
    mag = p * (gl.abs() + g.abs() + ge.abs() * (lq.abs() + H + eH / U32))
    hit = torch.zeros_like(p)
    if d_logp is not None:
        hit.scatter_(1, at, g)
    dz = dz + hit
    e = ew + el + U32 * (4 * L.abs() + 16)
    # the exponential gives 0 for weights below 2^-126, the least normal number: an error of at most 2^-126 times what
    # the weight is multiplied with
    tiny = 2.0 ** -126 * (gl.abs() + g.abs() + ge.abs() * (lq.abs() + H))
    out["dx"] = (rows(scale * dz, math.nan, 0.0),
                 half * (scale * dz).abs() + scale * (e * mag + 4 * U32 * hit.abs() + tiny))
    return out
