"""Calls of the operators around a block: what is timed, and what it is compared with.

What a model runs between its attention layers and behind the last of them:

  resnorm  the residual stream: a block's output normed, gated, scaled and added
           to the stream, and the stream normed for the next block, in one pass;
           forward, forward and backward
  linear   a product with a weight matrix with bias, activation and residual
           in its epilogue; forward, forward and backward, single tokens
  logprob  log probabilities of given tokens out of rows of logits, with the
           rows' entropy and their most probable tokens; forward, forward and
           backward

A case is a dict of plain values.  With ``own`` false, ``run`` computes the
operators from elementary torch operations in 32 bits; with ``own`` true it
makes the calls of ``paper_2505_00315_amd.ops``.  ``exact`` gives the results
in 64 bits.
"""
import math

import torch

own = False

DEVICE = "cuda"
EPS = 1e-6


def _resnorm(name, pas, B, T, d, post, pre, gate, dtype="bf16", scales=(1.0, 1.0)):
    c = {"op": "resnorm", "pass": pas, "B": B, "T": T, "d": d, "post": post, "pre": pre, "gate": gate, "dtype": dtype,
         "residual_scale": scales[0], "branch_scale": scales[1]}
    if name:
        c["name"] = name
    return c


def _linear(name, pas, rows, d_in, d_out, act, order, bias, residual, dtype="bf16"):
    c = {"op": "linear", "pass": pas, "rows": rows, "d_in": d_in, "d_out": d_out, "act": act, "order": order,
         "bias": bias, "residual": residual, "dtype": dtype}
    if name:
        c["name"] = name
    return c


def _logprob(name, pas, rows, vocab, top, entropy, masked=False, scale=1.0, dtype="bf16"):
    c = {"op": "logprob", "pass": pas, "rows": rows, "vocab": vocab, "top": top, "entropy": entropy, "masked": masked,
         "scale": scale, "dtype": dtype}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one new token between two blocks: launches and host time are all there is
        _resnorm("norm_step", "fwd", 1, 1, 1024, True, True, "vector"),
        # the stream of a wide model in training, norms on both sides of the block
        _resnorm("norm_train", "train", 4, 4096, 4096, True, True, "vector", scales=(1.0, 0.5)),
        # a small fp32 study of odd sizes, a gate that every token computes, no norm behind the block
        _resnorm("norm_f32", "train", 3, 333, 200, False, True, "token", dtype="f32"),
        # one token through the first product of a feed-forward block
        _linear("lin_step", "fwd", 1, 1024, 4096, "silu", "in_out", True, False),
        # one token each of 32 conversations through the second one, added to the stream
        _linear("lin_batch", "fwd", 32, 16384, 4096, "none", "in_out", False, True),
        # the first product of the feed-forward block beside the layer of 8 x 1024 tokens of 1024
        _linear("lin_block", "train", 8192, 1024, 4096, "gelu", "in_out", True, False),
        # a wide model's second product in training, added to the stream
        _linear("lin_wide", "train", 16384, 8192, 4096, "none", "in_out", True, True),
        # an fp32 study of odd sizes, its weight shared with an embedding of tokens (rows of the outputs)
        _linear("lin_f32", "train", 777, 520, 1304, "silu", "out_in", True, True, dtype="f32"),
        # the next token of one conversation: its alternatives among those that a grammar allows
        _logprob("lp_step", "fwd", 1, 32000, 20, True, masked=True, scale=1.25),
        # prompts scored with their alternatives, fp32 logits of an odd vocabulary
        _logprob("lp_score_f32", "fwd", 300, 50001, 5, False, dtype="f32"),
        # a loss with an entropy term over a large vocabulary
        _logprob("lp_train", "train", 4096, 131072, 0, True),
        # a loss over the rows of a short batch
        _logprob("lp_small", "train", 515, 8000, 0, False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _wide(rng, lo, hi):
    """A width: a multiple of 8, often one of 64."""
    unit = rng.choice([8, 64, 64])
    return max(1, _log(rng, lo, hi) // unit) * unit


def _draw(rng):
    kind = rng.choice(["resnorm", "linear", "linear", "logprob"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if kind == "resnorm":
        pre = rng.random() < 0.8
        return _resnorm(None, rng.choice(["fwd", "train"]), _log(rng, 1, 16), _log(rng, 1, 4096), _wide(rng, 64, 8192),
                        rng.random() < 0.6 or not pre, pre, rng.choice(["none", "vector", "sequence", "token"]), dtype,
                        rng.choice([(1.0, 1.0), (1.0, 0.25), (0.8, 1.5)]))
    if kind == "linear":
        rows = rng.choice([_log(rng, 1, 64), _log(rng, 1, 16384), _log(rng, 64, 16384)])
        return _linear(None, rng.choice(["fwd", "train"]), rows, _wide(rng, 64, 16384), _wide(rng, 64, 16384),
                       rng.choice(["none", "gelu", "silu"]), rng.choice(["in_out", "out_in"]),
                       rng.random() < 0.6, rng.random() < 0.4, dtype)
    if rng.random() < 0.5:
        return _logprob(None, "train", _log(rng, 1, 8192), _log(rng, 8, 200000), 0, rng.random() < 0.5,
                        rng.random() < 0.3, rng.choice([1.0, 1.0, 0.7]), dtype)
    vocab = _log(rng, 8, 200000)
    return _logprob(None, "fwd", _log(rng, 1, 2048), vocab, min(vocab, rng.choice([0, 1, 5, 20, 32])),
                    rng.random() < 0.5, rng.random() < 0.3, rng.choice([1.0, 1.0, 1.4]), dtype)


def draw(rng):
    """A drawn case, none of its costs above the largest listed one's (fp32 products count 8 times)."""
    top = {"bytes": 0, "flops": 0}
    for c in listed():
        w = work(c)
        top = {n: max(top[n], w[n]) for n in top}
    while True:
        c = _draw(rng)
        w = work(c)
        flops = w["flops"] * (8 if c["dtype"] == "f32" and c["op"] == "linear" else 1)
        if w["bytes"] <= top["bytes"] and flops <= top["flops"]:
            return c


def work(c):
    es = 2 if c["dtype"] == "bf16" else 4
    train = c["pass"] == "train"
    if c["op"] == "resnorm":
        rows, d = c["B"] * c["T"], c["d"]
        token = c["gate"] == "token"
        # forward: x, y (and the token's gate) read, h (and n) written; backward: x, y, the gate and the outputs'
        # gradients read, dx, dy (and the gate's gradient) written
        moved = 2 + token + 1 + c["pre"]
        if train:
            moved += 2 + token + 1 + c["pre"] + 2 + token
        return {"bytes": rows * d * moved * es, "flops": rows * d * (40 if train else 12)}
    if c["op"] == "linear":
        M, K, N = c["rows"], c["d_in"], c["d_out"]
        z = train and c["act"] != "none"
        size = M * K + K * N + M * N * (1 + c["residual"] + z)
        if train:
            size += (M * K + K * N + M * N * (1 + z)) + (M * K + K * N)
        return {"bytes": size * es, "flops": 2 * M * K * N * (3 if train else 1)}
    size = c["rows"] * c["vocab"]
    return {"bytes": size * es * (3 if train else 1), "flops": size * (20 if train else 8)}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _dt(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _inputs(c, seed):
    """The call's data, from the seed alone."""
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    dt = _dt(c)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEVICE, dtype=torch.float32)

    if c["op"] == "resnorm":
        B, T, d = c["B"], c["T"], c["d"]
        # a stream that grows over the blocks, tokens and channels of different sizes
        size, chan = torch.exp(0.5 * normal(B, T, 1)), torch.exp(0.3 * normal(d))
        x = {"x": (3 * normal(B, T, d) * size * chan).to(dt), "y": (normal(B, T, d) * chan).to(dt)}
        if c["post"]:
            x["w_post"] = (1 + 0.2 * normal(d)).to(dt)
        if c["pre"]:
            x["w_pre"] = (1 + 0.2 * normal(d)).to(dt)
        if c["gate"] != "none":
            shape = {"vector": (d,), "sequence": (B, d), "token": (B, T, d)}[c["gate"]]
            x["gate"] = torch.sigmoid(normal(*shape)).to(dt)
        if c["pass"] == "train":
            x["dh"] = normal(B, T, d).to(dt)
            if c["pre"]:
                x["dn"] = normal(B, T, d).to(dt)
        return x
    if c["op"] == "linear":
        M, K, N = c["rows"], c["d_in"], c["d_out"]
        w = (K, N) if c["order"] == "in_out" else (N, K)
        x = {"x": normal(M, K).to(dt), "w": (normal(*w) / math.sqrt(K)).to(dt)}
        if c["bias"]:
            x["b"] = (0.3 * normal(N)).to(dt)
        if c["residual"]:
            x["r"] = normal(M, N).to(dt)
        if c["pass"] == "train":
            x["dy"] = normal(M, N).to(dt)
        return x
    R, V = c["rows"], c["vocab"]
    # some tokens are likely everywhere; rows differ in how sure they are
    logits = (normal(R, V) * torch.exp(0.3 * normal(R, 1)) + normal(V)) * 2
    x = {"targets": torch.randint(0, V, (R,), generator=g, device=DEVICE, dtype=torch.int32)}
    if c["masked"]:  # about a third of the tokens cannot come next
        closed = torch.rand(R, V, generator=g, device=DEVICE) < 0.3
        closed.scatter_(1, x["targets"].long()[:, None], False)
        logits.masked_fill_(closed, -math.inf)
    x["logits"] = logits.to(dt)
    if c["pass"] == "train":
        # a twentieth of the rows has no target (padding, prompts)
        x["targets"] = torch.where(torch.rand(R, generator=g, device=DEVICE) < 0.05, -1, x["targets"])
        x["d_logp"] = normal(R)
        if c["entropy"]:
            x["d_entropy"] = 0.1 * normal(R)
    return x


def prepare(c, seed):
    st = {"case": c, **_inputs(c, seed)}
    if not own:
        return st
    from paper_2505_00315_amd import ops

    train = c["pass"] == "train"
    if c["op"] == "resnorm":
        st["shape"] = sh = ops.make_residual_shape(c["B"], c["T"], c["d"], c["dtype"], post_norm=c["post"],
                                                   pre_norm=c["pre"], gate=c["gate"],
                                                   residual_scale=c["residual_scale"],
                                                   branch_scale=c["branch_scale"], eps=EPS)
        st["h"] = torch.empty_like(st["x"])
        st["n"] = torch.empty_like(st["x"]) if c["pre"] else None
        if train:
            st["scratch"] = ops.alloc_residual_scratch(sh)
            for n in ("x", "y", "w_post", "gate", "w_pre"):
                if n in st:
                    st["d_" + n] = torch.empty_like(st[n])
        return st
    if c["op"] == "linear":
        st["shape"] = sh = ops.make_linear_shape(c["rows"], c["d_in"], c["d_out"], c["dtype"], act=c["act"],
                                                 w_order=c["order"])
        st["scratch"] = ops.alloc_linear_scratch(sh)
        st["out"] = torch.empty(c["rows"], c["d_out"], dtype=_dt(c), device=DEVICE)
        if train:
            st["z"] = torch.empty_like(st["out"]) if c["act"] != "none" else None
            for n in ("x", "w", "b"):
                if n in st:
                    st["d_" + n] = torch.empty_like(st[n])
        return st
    st["shape"] = sh = ops.make_logprob_shape(c["rows"], c["vocab"], c["dtype"], top=c["top"], scale=c["scale"])
    st["scratch"] = ops.alloc_logprob_scratch(sh)

    def new(*shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device=DEVICE)

    st["logp"], st["lse"], st["stats"] = new(c["rows"]), new(c["rows"]), new(c["rows"], 2)
    st["entropy"] = new(c["rows"]) if c["entropy"] else None
    if c["top"]:
        st["top_logp"], st["top_index"] = new(c["rows"], c["top"]), new(c["rows"], c["top"], dtype=torch.int32)
    if train:
        st["d_logits"] = torch.empty_like(st["logits"])
    return st


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(st):
    c = st["case"]
    if own:
        return _run_own(st, c)
    return {"resnorm": _plain_resnorm, "linear": _plain_linear, "logprob": _plain_logprob}[c["op"]](st, c)


def _run_own(st, c):
    from paper_2505_00315_amd import ops

    train, sh, get = c["pass"] == "train", st["shape"], st.get
    if c["op"] == "resnorm":
        ops.residual_norm(sh, st["x"], st["y"], w_post=get("w_post"), gate=get("gate"), w_pre=get("w_pre"),
                          h_out=st["h"], n_out=st["n"])
        out = {"h": st["h"], **({"n": st["n"]} if c["pre"] else {})}
        if train:
            ops.residual_norm_backward(sh, st["x"], st["y"], w_post=get("w_post"), gate=get("gate"), w_pre=get("w_pre"),
                                       dh=st["dh"], dn=get("dn"), dx=st["d_x"], dy=st["d_y"], dw_post=get("d_w_post"),
                                       dgate=get("d_gate"), dw_pre=get("d_w_pre"), scratch=st["scratch"])
            out.update({n: st[n] for n in ("d_x", "d_y", "d_w_post", "d_gate", "d_w_pre") if n in st})
        return out
    if c["op"] == "linear":
        ops.linear(sh, st["x"], st["w"], bias=get("b"), residual=get("r"), y=st["out"], z=get("z"),
                   scratch=st["scratch"])
        out = {"y": st["out"]}
        if train:
            ops.linear_backward(sh, st["x"], st["w"], st["dy"], z=st["z"], grads="xwb" if c["bias"] else "xw",
                                dx=st["d_x"], dw=st["d_w"], db=get("d_b"), scratch=st["scratch"])
            out.update({n: st[n] for n in ("d_x", "d_w", "d_b") if n in st})
        return out
    ops.token_logprobs(sh, st["logits"], st["targets"], logp=st["logp"], lse=st["lse"], stats=st["stats"],
                       entropy=st["entropy"], top_logp=get("top_logp"), top_index=get("top_index"),
                       scratch=st["scratch"])
    out = {n: st[n] for n in ("logp", "lse", "entropy", "top_logp", "top_index") if get(n) is not None}
    if train:
        ops.token_logprobs_backward(sh, st["logits"], st["targets"], st["stats"], entropy=st["entropy"],
                                    d_logp=st["d_logp"], d_entropy=get("d_entropy"), d_logits=st["d_logits"])
        out["d_logits"] = st["d_logits"]
    return out


# ---------------------------------------------------------------------------
# plain forms (32 bits)
# ---------------------------------------------------------------------------
def _rows_of(gate, c):
    """The gate as it goes with rows [B, T, d]."""
    return gate.float()[:, None] if c["gate"] == "sequence" else gate.float()


def _plain_resnorm(st, c):
    dt, a, b = _dt(c), c["residual_scale"], c["branch_scale"]
    x, y = st["x"].float(), st["y"].float()
    if c["post"]:
        sy = torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS)
        zy, wp = y * sy, st["w_post"].float()
        u = zy * wp
    else:
        u = y
    g = _rows_of(st["gate"], c) if "gate" in st else None
    h = a * x + b * (u if g is None else g * u)
    out = {"h": h.to(dt)}
    if c["pre"]:
        sh = torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS)
        zh, wn = h * sh, st["w_pre"].float()
        out["n"] = (zh * wn).to(dt)
    if c["pass"] == "fwd":
        return out
    dh = st["dh"].float()
    if c["pre"]:
        dn = st["dn"].float()
        out["d_w_pre"] = (dn * zh).double().sum((0, 1)).to(dt)
        e = dn * wn
        dh = dh + sh * (e - zh * (e * zh).mean(-1, keepdim=True))
    out["d_x"] = (a * dh).to(dt)
    du = b * dh
    if g is not None:
        dg = du * u
        out["d_gate"] = {"vector": lambda: dg.double().sum((0, 1)), "sequence": lambda: dg.double().sum(1),
                         "token": lambda: dg}[c["gate"]]().to(dt)
        du = du * g
    if c["post"]:
        out["d_w_post"] = (du * zy).double().sum((0, 1)).to(dt)
        e = du * wp
        du = sy * (e - zy * (e * zy).mean(-1, keepdim=True))
    out["d_y"] = du.to(dt)
    return out


def _act(z, act):
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _act_slope(z, act):
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    s = 1 / (1 + torch.exp(-z))
    return s * (1 + z * (1 - s))


def _plain_linear(st, c):
    dt = _dt(c)
    x, w = st["x"].float(), st["w"].float()
    wt = w if c["order"] == "in_out" else w.t()
    z = x @ wt
    if c["bias"]:
        z += st["b"].float()
    y = _act(z, c["act"])
    if c["residual"]:
        y = y + st["r"].float()
    out = {"y": y.to(dt)}
    if c["pass"] == "fwd":
        return out
    dz = st["dy"].float()
    if c["act"] != "none":
        dz = dz * _act_slope(z, c["act"])
    out["d_x"] = (dz @ wt.t()).to(dt)
    out["d_w"] = (x.t() @ dz if c["order"] == "in_out" else dz.t() @ x).to(dt)
    if c["bias"]:
        out["d_b"] = dz.double().sum(0).to(dt)
    return out


def _plain_logprob(st, c):
    R, V, scale = c["rows"], c["vocab"], c["scale"]
    x = st["logits"]
    z = x.float() * scale
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    lse = top + torch.log(total)
    t = st["targets"].long()[:, None]
    here = t >= 0
    out = {"lse": lse[:, 0], "logp": torch.where(here, z.gather(1, t.clamp_min(0)) - lse, 0.0)[:, 0]}
    if c["entropy"]:
        p = e / total
        logq = torch.where(p > 0, z - lse, 0.0)
        H = -(p * logq).sum(1, keepdim=True)
        out["entropy"] = H[:, 0]
    if c["top"]:
        # whole numbers in the order of the logits, equal ones with the lower index first
        u = (x.float() + 0.0).view(torch.int32).long()
        key = torch.where(u >= 0, u, -(u + 2 ** 31)) * 2 ** 20 + (2 ** 20 - 1 - torch.arange(V, device=DEVICE))
        index = torch.topk(key, c["top"], 1).indices
        out["top_logp"], out["top_index"] = z.gather(1, index) - lse, index.to(torch.int32)
    if c["pass"] == "fwd":
        return out
    if not c["entropy"]:
        p = e / total
    d = st["d_logp"][:, None].where(here, 0.0)
    dz = -d * p
    if c["entropy"]:
        dz -= st["d_entropy"][:, None] * p * (logq + H)
    dz.scatter_add_(1, t.clamp_min(0), d)
    out["d_logits"] = (dz * scale).to(_dt(c))
    return out


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def exact(c, seed):
    x = _inputs(c, seed)
    return {"resnorm": _exact_resnorm, "linear": _exact_linear, "logprob": _exact_logprob}[c["op"]](c, x)


def _exact_resnorm(c, x):
    """Sequence by sequence; gradients by differentiation, the shared ones adding up in their leaves."""
    train = c["pass"] == "train"
    out = {n: torch.empty(x["x"].shape, dtype=torch.float64, device=DEVICE)
           for n in ["h"] + ["n"] * c["pre"] + (["d_x", "d_y"] if train else [])}
    leaf = {n: x[n].double().requires_grad_(train) for n in ("w_post", "w_pre", "gate") if n in x}

    def normed(v, w):
        v = v / math.sqrt(c["d"])
        size = torch.linalg.vector_norm(torch.cat([v, torch.full_like(v[:, :1], math.sqrt(EPS))], 1), dim=1)
        return v * (math.sqrt(c["d"]) / size)[:, None] * w

    for s in range(c["B"]):
        X, Y = (x[n][s].double().requires_grad_(train) for n in ("x", "y"))
        u = normed(Y, leaf["w_post"]) if c["post"] else Y
        if "gate" in leaf:
            u = u * (leaf["gate"] if c["gate"] == "vector" else leaf["gate"][s])
        h = c["residual_scale"] * X + c["branch_scale"] * u
        out["h"][s] = h.detach()
        loss = (h * x["dh"][s].double()).sum() if train else None
        if c["pre"]:
            n = normed(h, leaf["w_pre"])
            out["n"][s] = n.detach()
            if train:
                loss = loss + (n * x["dn"][s].double()).sum()
        if train:
            loss.backward()
            out["d_x"][s], out["d_y"][s] = X.grad, Y.grad
    if train:
        out.update({"d_" + n: t.grad for n, t in leaf.items()})
    return out


def _exact_linear(c, x):
    """A block of rows at a time; gradients by differentiation."""
    train, M = c["pass"] == "train", c["rows"]
    W = x["w"].double().requires_grad_(train)
    b = x["b"].double().requires_grad_(train) if c["bias"] else None
    y = torch.empty(M, c["d_out"], dtype=torch.float64, device=DEVICE)
    dx = torch.empty(M, c["d_in"], dtype=torch.float64, device=DEVICE) if train else None
    for a in range(0, M, 4096):
        X = x["x"][a:a + 4096].double().requires_grad_(train)
        z = torch.nn.functional.linear(X, W.t() if c["order"] == "in_out" else W, b)
        o = {"none": lambda v: v, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}[c["act"]](z)
        y[a:a + 4096] = (o + x["r"][a:a + 4096].double() if c["residual"] else o).detach()
        if train:
            o.backward(x["dy"][a:a + 4096].double())
            dx[a:a + 4096] = X.grad
    out = {"y": y}
    if train:
        out.update(d_x=dx, d_w=W.grad, **({"d_b": b.grad} if c["bias"] else {}))
    return out


def _exact_logprob(c, x):
    """Rows in blocks, from log_softmax."""
    R, V, train = c["rows"], c["vocab"], c["pass"] == "train"
    out = {n: torch.zeros(R, dtype=torch.float64, device=DEVICE) for n in ["logp", "lse"] + ["entropy"] * c["entropy"]}
    if train:
        out["d_logits"] = torch.empty(R, V, dtype=torch.float64, device=DEVICE)
    if c["top"]:
        out["top_logp"], out["top_index"] = torch.empty(R, c["top"], dtype=torch.float64, device=DEVICE), None
    step = max(1, 2 ** 26 // V)
    for a in range(0, R, step):
        z = x["logits"][a:a + step].double() * c["scale"]
        logq = torch.log_softmax(z, 1)
        t = x["targets"][a:a + step].long()
        at = torch.nonzero(t >= 0)[:, 0]
        out["lse"][a:a + step] = torch.logsumexp(z, 1)
        out["logp"][a + at] = logq[at, t[at]]
        p = torch.exp(logq)
        if c["entropy"]:
            H = torch.special.entr(p).sum(1)
            out["entropy"][a:a + step] = H
        if c["top"]:
            out["top_logp"][a:a + step] = torch.sort(logq, 1, descending=True).values[:, :c["top"]]
        if train:
            g = torch.zeros_like(p)
            g[at, t[at]] = 1.0
            w = torch.zeros(t.numel(), 1, dtype=torch.float64, device=DEVICE)
            w[at] = x["d_logp"][a:a + step].double()[at, None]
            dz = w * (g - p)
            if c["entropy"]:
                dz += x["d_entropy"][a:a + step].double()[:, None] * (torch.special.entr(p) - p * H[:, None])
            out["d_logits"][a:a + step] = c["scale"] * dz
    return out
