"""Operators of the dense heads: norm and rotation of query and key rows,
attention with a sliding window and first tokens that stay visible, and a paged
cache that holds keys and values in 4 bits.  Operators around a block: the residual
stream with its norms and gate, products with weight matrices, log probabilities
of tokens.

Python binding of the functions that ``include/mosa.h`` declares for them:
argument marshalling and checks only, every step runs in the HIP kernels.

Rows are tensors of shape [batch, heads, length, d_head] in any memory order
whose last axis is contiguous and whose other strides are multiples of 16
bytes: ``x.transpose(1, 2)`` of a [batch, length, heads, d_head] tensor, a slice
of packed rows, ``mosa.saved_view(shape, saved, "Kd")``.  The stream is [batch,
seq_len, d_model] likewise, and a matrix has two axes.  Work goes to the
current stream of the tensors' device (or ``stream``), whichever device is
current.
"""
import ctypes
import functools
import math

import torch

from . import mosa

PAIRS = {"adjacent": 0, "halves": 1}  # MOSA_PAIRS_*
GATES = {"none": 0, "vector": 1, "sequence": 2, "token": 3}  # MOSA_GATE_*
ACTS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}  # MOSA_ACT_*
W_ORDERS = {"in_out": 0, "out_in": 1}  # MOSA_W_*


class Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("batch_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
                ("row_stride", ctypes.c_int64)]


class NormShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("batch", "seq_len", "q_heads", "kv_heads", "d_head", "dtype", "rope_dim",
                                              "rope_pairs")] + [("rope_base", ctypes.c_float), ("eps", ctypes.c_float)]


class AttnShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("batch", "q_heads", "kv_heads", "q_len", "kv_len", "d_head", "dtype",
                                              "window", "sinks")] + [("scale", ctypes.c_float)]


class CacheShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("batch", "kv_heads", "d_head", "dtype", "pages", "page_size",
                                              "max_pages")]


class Matrix(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("row_stride", ctypes.c_int64)]


class ResidualShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("batch", "seq_len", "d_model", "dtype", "post_norm", "pre_norm", "gate")] + [
        (n, ctypes.c_float) for n in ("residual_scale", "branch_scale", "eps")]


class LinearShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("rows", "d_in", "d_out", "dtype", "act", "w_order")]


class LogprobShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("rows", "vocab", "dtype", "top")] + [("scale", ctypes.c_float)]


_fn = None


def _lib():
    """The library with the prototypes of these functions (set once)."""
    global _fn
    if _fn is None:
        L = mosa.lib()
        P, V, Z = ctypes.POINTER, ctypes.c_void_p, ctypes.c_size_t
        norm, attn, cache, rows = P(NormShape), P(AttnShape), P(CacheShape), P(Rows)
        res, lin, lp, mat = P(ResidualShape), P(LinearShape), P(LogprobShape), P(Matrix)
        table = {
            "mosa_norm_scratch_size": [norm, P(Z)],
            "mosa_qk_norm_rope": [norm, rows, rows, V, V, V, rows, rows, V],
            "mosa_qk_norm_rope_backward": [norm, rows, rows, V, V, V, rows, rows, rows, rows, V, V, V, Z, V],
            "mosa_attn_scratch_size": [attn, P(Z), P(Z)],
            "mosa_window_attention": [attn, rows, rows, rows, V, V, rows, V, V, Z, V],
            "mosa_window_attention_backward": [attn, rows, rows, rows, rows, V, rows, V, V, rows, rows, rows, V, Z, V],
            "mosa_cache4_size": [cache, P(Z)],
            "mosa_cache4_append": [cache, V, V, V, V, ctypes.c_int, rows, rows, V],
            "mosa_cache4_read": [cache, V, V, V, V, ctypes.c_int, rows, rows, V],
            "mosa_cache4_attention": [attn, cache, rows, V, V, V, V, rows, V, V, Z, V],
            "mosa_residual_scratch_size": [res, P(Z)],
            "mosa_residual_norm": [res, rows, rows, V, rows, V, rows, rows, V],
            "mosa_residual_norm_backward": [res, rows, rows, V, rows, V, rows, rows, rows, rows, V, rows, V, V, Z, V],
            "mosa_linear_scratch_size": [lin, P(Z), P(Z)],
            "mosa_linear": [lin, mat, mat, V, mat, mat, mat, V, Z, V],
            "mosa_linear_backward": [lin, mat, mat, mat, mat, mat, mat, V, V, Z, V],
            "mosa_logprob_scratch_size": [lp, P(Z)],
            "mosa_token_logprobs": [lp, mat, V, V, V, V, V, V, V, V, Z, V],
            "mosa_token_logprobs_backward": [lp, mat, V, V, V, V, V, V, mat, V],
        }
        for name, args in table.items():
            f = getattr(L, name)
            f.argtypes, f.restype = args, ctypes.c_int
        _fn = L
    return _fn


@functools.lru_cache(maxsize=None)
def _function(name):
    return getattr(_lib(), name)


_DTYPE = {"bf16": mosa.MOSA_BF16, "f32": mosa.MOSA_F32, torch.bfloat16: mosa.MOSA_BF16, torch.float32: mosa.MOSA_F32}
_TORCH = {mosa.MOSA_BF16: torch.bfloat16, mosa.MOSA_F32: torch.float32}


def make_norm_shape(batch, seq_len, q_heads, kv_heads, d_head, dtype="bf16", rope_dim=None, rope_pairs="adjacent",
                    rope_base=10000.0, eps=1e-6):
    """``rope_dim``: columns that are turned, by default half of them as in the layer."""
    return NormShape(batch, seq_len, q_heads, kv_heads, d_head, _DTYPE[dtype],
                     d_head // 2 if rope_dim is None else rope_dim, PAIRS[rope_pairs], rope_base, eps)


def make_attn_shape(batch, q_heads, kv_heads, q_len, kv_len, d_head, dtype="bf16", window=0, sinks=0, scale=None):
    """``scale``: of the scores, by default 1 / sqrt(d_head)."""
    return AttnShape(batch, q_heads, kv_heads, q_len, kv_len, d_head, _DTYPE[dtype], window, sinks,
                     1.0 / math.sqrt(d_head) if scale is None else scale)


def make_cache_shape(batch, kv_heads, d_head, pages, page_size, max_pages, dtype="bf16"):
    return CacheShape(batch, kv_heads, d_head, _DTYPE[dtype], pages, page_size, max_pages)


def make_residual_shape(batch, seq_len, d_model, dtype="bf16", post_norm=False, pre_norm=True, gate="none",
                        residual_scale=1.0, branch_scale=1.0, eps=1e-6):
    """``gate``: "none", or how it is shared: "vector" [d_model], "sequence" [batch, d_model], "token" [batch, seq_len,
    d_model]."""
    return ResidualShape(batch, seq_len, d_model, _DTYPE[dtype], int(bool(post_norm)), int(bool(pre_norm)), GATES[gate],
                         residual_scale, branch_scale, eps)


def make_linear_shape(rows, d_in, d_out, dtype="bf16", act="none", w_order="in_out"):
    """``w_order``: w is [d_in, d_out] ("in_out", as the layer's weights) or [d_out, d_in] ("out_in")."""
    return LinearShape(rows, d_in, d_out, _DTYPE[dtype], ACTS[act], W_ORDERS[w_order])


def make_logprob_shape(rows, vocab, dtype="bf16", top=0, scale=1.0):
    """``top``: alternatives that token_logprobs lists; ``scale``: of the logits (1 / temperature)."""
    return LogprobShape(rows, vocab, _DTYPE[dtype], top, scale)


# ---------------------------------------------------------------------------
# checks
# ---------------------------------------------------------------------------
def _rows(t, what, shape, dtype, device):
    """The Rows of a tensor that has to be [B, H, T, dh] of this type on this device."""
    if t.dtype != dtype:
        raise TypeError(f"{what}: dtype {t.dtype}, expected {dtype}")
    if t.shape != shape:
        raise ValueError(f"{what}: shape {tuple(t.shape)}, expected {shape}")
    if t.device != device:
        raise ValueError(f"{what}: on {t.device}, expected {device}")
    b, h, r, c = t.stride()
    if c != 1:
        raise ValueError(f"{what}: the last axis is not contiguous")
    return Rows(t.data_ptr(), b, h, r)


def _matrix(t, what, shape, dtype, device):
    """The Matrix of a tensor that has to be [rows, columns] of this type on this device (None: NULL)."""
    if t is None:
        return None
    if t.dtype != dtype:
        raise TypeError(f"{what}: dtype {t.dtype}, expected {dtype}")
    if t.shape != shape:
        raise ValueError(f"{what}: shape {tuple(t.shape)}, expected {shape}")
    if t.device != device:
        raise ValueError(f"{what}: on {t.device}, expected {device}")
    r, c = t.stride()
    if c != 1 and shape[1] != 1:
        raise ValueError(f"{what}: the last axis is not contiguous")
    return Matrix(t.data_ptr(), r)


def _device(t, what):
    if not t.is_cuda:
        raise ValueError(f"{what}: the operators run on the GPU only")
    return t.device


def _array(t, what, dtype, numel, device, required=False):
    """Address of a contiguous device array (None: NULL)."""
    if t is None and not required:
        return None
    mosa._check_tensor(t, what, dtype, numel, device)
    return t.data_ptr()


def _new(make, stream, *args, **kw):
    """A tensor made for a call on ``stream`` comes from that stream's memory."""
    if stream is None:
        return make(*args, **kw)
    with torch.cuda.stream(stream):
        return make(*args, **kw)


def _like(t, given, stream):
    return _new(torch.empty_like, stream, t) if given is None else given


def _scratch(t, size, device, stream):
    """(tensor, address, bytes) of a call's scratch: the given buffer, whose size the library checks, or a new one of
    size() bytes."""
    if t is None:
        need = size()
        if need == 0:
            return None, None, 0
        t = _new(torch.empty, stream, need, dtype=torch.uint8, device=device)
    elif t.dtype != torch.uint8 or not t.is_contiguous() or t.device != device:
        raise ValueError(f"scratch: a contiguous uint8 tensor on {device} is required")
    return t, t.data_ptr(), t.numel()


def _call(name, device, stream, *args):
    """Call a library function on ``device``, whichever is current; the stream is its last argument."""
    f, index = _function(name), device.index
    if stream is None:  # (torch.cuda.current_stream makes an object first: 1.9 us of a 10 us call)
        handle = torch._C._cuda_getCurrentRawStream(index)
    elif stream.device != device:
        raise ValueError(f"stream: on {stream.device}, expected {device}")
    else:
        handle = stream.cuda_stream
    if torch.cuda.current_device() == index:
        status = f(*args, handle)
    else:
        with torch.cuda.device(device):
            status = f(*args, handle)
    if status:
        mosa._check(status, name)


# ---------------------------------------------------------------------------
# norm and rotation
# ---------------------------------------------------------------------------
def norm_scratch_size(shape):
    n = ctypes.c_size_t()
    mosa._check(_lib().mosa_norm_scratch_size(shape, n), "mosa_norm_scratch_size")
    return n.value


def alloc_norm_scratch(shape, device="cuda"):
    return torch.empty(max(norm_scratch_size(shape), 256), dtype=torch.uint8, device=device)


def _norm_io(shape):
    B, T, dh = shape.batch, shape.seq_len, shape.d_head
    return _TORCH[shape.dtype], (B, shape.q_heads, T, dh), (B, shape.kv_heads, T, dh)


def qk_norm_rope(shape, q, k, wq=None, wk=None, positions=None, q_out=None, k_out=None, stream=None):
    """Norm every query and key row and turn it by its token's position.
    q [B, Hq, T, dh], k [B, Hkv, T, dh]; wq, wk [dh] (None: ones); positions
    int32 [B, T] (None: 0 .. T - 1).  q_out, k_out may be q and k.
    Returns (q_out, k_out)."""
    st, qs, ks = _norm_io(shape)
    dev = _device(q, "q")
    q_out = _like(q, q_out, stream)
    k_out = _like(k, k_out, stream)
    _call("mosa_qk_norm_rope", dev, stream, shape, _rows(q, "q", qs, st, dev), _rows(k, "k", ks, st, dev),
          _array(wq, "wq", st, shape.d_head, dev), _array(wk, "wk", st, shape.d_head, dev),
          _array(positions, "positions", torch.int32, shape.batch * shape.seq_len, dev),
          _rows(q_out, "q_out", qs, st, dev), _rows(k_out, "k_out", ks, st, dev))
    return q_out, k_out


def qk_norm_rope_backward(shape, q, k, wq, wk, dq_out, dk_out, positions=None, dq=None, dk=None, dwq=None, dwk=None,
                          scratch=None, stream=None):
    """Gradients of qk_norm_rope: q, k as they went in, dq_out and dk_out the
    outputs' gradients (dq and dk may be the same tensors).  dwq, dwk: written
    where given, or made where the weight is.  Returns (dq, dk, dwq, dwk)."""
    st, qs, ks = _norm_io(shape)
    dev = _device(q, "q")
    dq = _like(q, dq, stream)
    dk = _like(k, dk, stream)
    dwq = dwq if wq is None else _like(wq, dwq, stream)
    dwk = dwk if wk is None else _like(wk, dwk, stream)
    grads = dwq is not None or dwk is not None
    buf, at, size = _scratch(scratch, lambda: norm_scratch_size(shape) if grads else 0, dev, stream)
    _call("mosa_qk_norm_rope_backward", dev, stream, shape, _rows(q, "q", qs, st, dev), _rows(k, "k", ks, st, dev),
          _array(wq, "wq", st, shape.d_head, dev), _array(wk, "wk", st, shape.d_head, dev),
          _array(positions, "positions", torch.int32, shape.batch * shape.seq_len, dev),
          _rows(dq_out, "dq_out", qs, st, dev), _rows(dk_out, "dk_out", ks, st, dev), _rows(dq, "dq", qs, st, dev),
          _rows(dk, "dk", ks, st, dev), _array(dwq, "dwq", st, shape.d_head, dev),
          _array(dwk, "dwk", st, shape.d_head, dev), at, size)
    return dq, dk, dwq, dwk


# ---------------------------------------------------------------------------
# windowed attention
# ---------------------------------------------------------------------------
def attn_scratch_size(shape):
    """(forward, backward) bytes; the forward's serve cache4_attention too."""
    f, b = ctypes.c_size_t(), ctypes.c_size_t()
    mosa._check(_lib().mosa_attn_scratch_size(shape, f, b), "mosa_attn_scratch_size")
    return f.value, b.value


def alloc_attn_scratch(shape, device="cuda"):
    """One buffer for the forward and the backward of a shape."""
    return torch.empty(max(*attn_scratch_size(shape), 256), dtype=torch.uint8, device=device)


def _attn_io(shape):
    B, dh = shape.batch, shape.d_head
    return _TORCH[shape.dtype], (B, shape.q_heads, shape.q_len, dh), (B, shape.kv_heads, shape.kv_len, dh)


def window_attention(shape, q, k, v, q_lens=None, kv_lens=None, out=None, lse=None, scratch=None, stream=None):
    """Causal attention of q [B, Hq, Q, dh] over k, v [B, Hkv, N, dh], the last
    query at the last key's position: a query at p sees the keys j <= p with
    p - j < window (window 0: all of them) or j < sinks.  q_lens, kv_lens: int32
    [B], the lengths of the sequences of a padded batch.  Returns (out, lse)."""
    st, qs, ks = _attn_io(shape)
    dev = _device(q, "q")
    out = _like(q, out, stream)
    if lse is None:
        lse = _new(torch.empty, stream, qs[:3], dtype=torch.float32, device=dev)
    buf, at, size = _scratch(scratch, lambda: attn_scratch_size(shape)[0], dev, stream)
    _call("mosa_window_attention", dev, stream, shape, _rows(q, "q", qs, st, dev), _rows(k, "k", ks, st, dev),
          _rows(v, "v", ks, st, dev), _array(q_lens, "q_lens", torch.int32, shape.batch, dev),
          _array(kv_lens, "kv_lens", torch.int32, shape.batch, dev), _rows(out, "out", qs, st, dev),
          _array(lse, "lse", torch.float32, qs[0] * qs[1] * qs[2], dev), at, size)
    return out, lse


def window_attention_backward(shape, q, k, v, out, lse, d_out, q_lens=None, kv_lens=None, dq=None, dk=None, dv=None,
                              scratch=None, stream=None):
    """Gradients of window_attention from its out and lse and the gradient of
    out.  Returns (dq, dk, dv), zero past the lengths."""
    st, qs, ks = _attn_io(shape)
    dev = _device(q, "q")
    dq = _like(q, dq, stream)
    dk = _like(k, dk, stream)
    dv = _like(v, dv, stream)
    buf, at, size = _scratch(scratch, lambda: attn_scratch_size(shape)[1], dev, stream)
    _call("mosa_window_attention_backward", dev, stream, shape, _rows(q, "q", qs, st, dev),
          _rows(k, "k", ks, st, dev), _rows(v, "v", ks, st, dev), _rows(out, "out", qs, st, dev),
          _array(lse, "lse", torch.float32, qs[0] * qs[1] * qs[2], dev, required=True),
          _rows(d_out, "d_out", qs, st, dev), _array(q_lens, "q_lens", torch.int32, shape.batch, dev),
          _array(kv_lens, "kv_lens", torch.int32, shape.batch, dev), _rows(dq, "dq", qs, st, dev),
          _rows(dk, "dk", ks, st, dev), _rows(dv, "dv", ks, st, dev), at, size)
    return dq, dk, dv


# ---------------------------------------------------------------------------
# the 4-bit cache
# ---------------------------------------------------------------------------
def cache4_size(shape):
    n = ctypes.c_size_t()
    mosa._check(_lib().mosa_cache4_size(shape, n), "mosa_cache4_size")
    return n.value


@functools.lru_cache(maxsize=64)
def _cache_bytes(fields):
    return cache4_size(CacheShape.from_buffer_copy(fields))


def alloc_cache4(shape, device="cuda"):
    """The cache's memory (uint8).  Positions that were never written hold zeros."""
    return torch.zeros(cache4_size(shape), dtype=torch.uint8, device=device)


def _cache(shape, cache, table, device):
    need = _cache_bytes(bytes(shape))
    if cache.dtype != torch.uint8 or not cache.is_contiguous() or cache.device != device or cache.numel() < need:
        raise ValueError(f"cache: a contiguous uint8 tensor on {device} of at least {need} bytes is required")
    return cache.data_ptr(), _array(table, "page_table", torch.int32, shape.batch * shape.max_pages, device, True)


def _cache_rows(name, shape, cache, table, start, lens, k, v, stream):
    st, dev = _TORCH[shape.dtype], _device(cache, "cache")
    if k.dim() != 4:
        raise ValueError(f"k: shape {tuple(k.shape)}, expected [batch, kv_heads, rows, d_head]")
    want = (shape.batch, shape.kv_heads, k.shape[2], shape.d_head)
    where, pages = _cache(shape, cache, table, dev)
    _call(name, dev, stream, shape, where, pages, _array(start, "start", torch.int32, shape.batch, dev),
          _array(lens, "lens", torch.int32, shape.batch, dev), k.shape[2], _rows(k, "k", want, st, dev),
          _rows(v, "v", want, st, dev))


def cache4_append(shape, cache, page_table, start, k, v, lens=None, stream=None):
    """Hold rows t < lens[b] (None: all) of k and v [B, Hkv, rows, dh] as
    positions start[b] + t (start None: from 0).  page_table: int32 [B,
    max_pages]; a position on no page is dropped."""
    _cache_rows("mosa_cache4_append", shape, cache, page_table, start, lens, k, v, stream)


def cache4_read(shape, cache, page_table, start, rows=None, lens=None, k=None, v=None, stream=None):
    """The values held at positions start[b] + t, t < lens[b] (None: rows), as
    rows [B, Hkv, rows, dh], 0 elsewhere.  Returns (k, v)."""
    if k is None:
        if rows is None:
            raise ValueError("rows: required where k is not given")
        k = _new(torch.empty, stream, (shape.batch, shape.kv_heads, rows, shape.d_head), dtype=_TORCH[shape.dtype],
                 device=cache.device)
    v = _like(k, v, stream)
    _cache_rows("mosa_cache4_read", shape, cache, page_table, start, lens, k, v, stream)
    return k, v


def cache4_attention(shape, cache_shape, q, cache, page_table, kv_lens, q_lens=None, out=None, lse=None, scratch=None,
                     stream=None):
    """window_attention over the positions 0 .. kv_lens[b] - 1 of the cache, for
    a few queries at once (from some dozens on, cache4_read and
    window_attention over its rows take less time).
    ``shape``: an attention shape whose kv_len bounds kv_lens.  lse is written
    where it is given.  Returns out."""
    st, qs, _ = _attn_io(shape)
    dev = _device(q, "q")
    out = _like(q, out, stream)
    where, pages = _cache(cache_shape, cache, page_table, dev)
    buf, at, size = _scratch(scratch, lambda: attn_scratch_size(shape)[0], dev, stream)
    _call("mosa_cache4_attention", dev, stream, shape, cache_shape, _rows(q, "q", qs, st, dev), where, pages,
          _array(q_lens, "q_lens", torch.int32, shape.batch, dev),
          _array(kv_lens, "kv_lens", torch.int32, shape.batch, dev, True), _rows(out, "out", qs, st, dev),
          _array(lse, "lse", torch.float32, qs[0] * qs[1] * qs[2], dev), at, size)
    return out


# ---------------------------------------------------------------------------
# the residual stream
# ---------------------------------------------------------------------------
def residual_scratch_size(shape):
    n = ctypes.c_size_t()
    mosa._check(_lib().mosa_residual_scratch_size(shape, n), "mosa_residual_scratch_size")
    return n.value


def alloc_residual_scratch(shape, device="cuda"):
    return torch.empty(max(residual_scratch_size(shape), 256), dtype=torch.uint8, device=device)


def _stream_rows(t, what, sizes, dtype, device):
    """The Rows of a tensor of these sizes, [batch, seq_len, d_model] or a gate's (None: NULL)."""
    if t is None:
        return None
    if t.dtype != dtype:
        raise TypeError(f"{what}: dtype {t.dtype}, expected {dtype}")
    if t.shape != sizes:
        raise ValueError(f"{what}: shape {tuple(t.shape)}, expected {sizes}")
    if t.device != device:
        raise ValueError(f"{what}: on {t.device}, expected {device}")
    st = t.stride()
    if st[-1] != 1:
        raise ValueError(f"{what}: the last axis is not contiguous")
    return Rows(t.data_ptr(), st[0] if len(st) > 1 else 0, 0, st[1] if len(st) > 2 else 0)


def _residual_io(shape):
    """(storage type, sizes of the stream, sizes of the gate)"""
    B, T, d = sizes = shape.batch, shape.seq_len, shape.d_model
    return _TORCH[shape.dtype], sizes, (None, (d,), (B, d), sizes)[shape.gate]


def _gate_rows(t, what, sizes, dtype, device):
    if t is not None and sizes is None:
        raise ValueError(f"{what}: the shape has no gate")
    return _stream_rows(t, what, sizes, dtype, device)


def residual_norm(shape, x, y, w_post=None, gate=None, w_pre=None, h_out=None, n_out=None, stream=None):
    """The stream behind a block and what the next block reads, from the stream x
    and the block's output y (both [B, T, d]):
        h = residual_scale x + branch_scale gate u,  u = w_post y / rms(y) (post_norm) or y
        n = w_pre h / rms(h)  (pre_norm)
    w_post, w_pre [d] (None: ones).  y None: h is x, and only n is computed.
    h_out may be x or y, and n_out y.  Returns (h, n), n None without pre_norm."""
    dev = _device(x, "x")
    st, sizes, gs = _residual_io(shape)
    d = sizes[2]
    h_out = _like(x, h_out, stream) if y is not None else h_out
    n_out = _like(x, n_out, stream) if shape.pre_norm else n_out
    _call("mosa_residual_norm", dev, stream, shape, _stream_rows(x, "x", sizes, st, dev),
          _stream_rows(y, "y", sizes, st, dev), _array(w_post, "w_post", st, d, dev),
          _gate_rows(gate, "gate", gs, st, dev), _array(w_pre, "w_pre", st, d, dev),
          _stream_rows(h_out, "h_out", sizes, st, dev), _stream_rows(n_out, "n_out", sizes, st, dev))
    return (x if y is None else h_out), n_out


def residual_norm_backward(shape, x, y, w_post=None, gate=None, w_pre=None, dh=None, dn=None, dx=None, dy=None,
                           dw_post=None, dgate=None, dw_pre=None, scratch=None, stream=None):
    """Gradients of residual_norm: x, y as they went in, dh and dn the outputs'
    gradients (dh None: 0).  dw_post, dgate and dw_pre are written where given, or
    made where the weight or the gate is.  dx may be dh or dn, and dy the other of
    them.  Returns (dx, dy, dw_post, dgate, dw_pre)."""
    dev = _device(x, "x")
    st, sizes, gs = _residual_io(shape)
    d = sizes[2]
    dx = _like(x, dx, stream)
    dy = dy if y is None else _like(y, dy, stream)
    dw_post = dw_post if w_post is None else _like(w_post, dw_post, stream)
    dw_pre = dw_pre if w_pre is None else _like(w_pre, dw_pre, stream)
    if gate is not None and dgate is None:  # (a broadcast gate's gradient is one of its whole shape)
        dgate = _new(torch.empty, stream, tuple(gate.shape), dtype=gate.dtype, device=gate.device)
    sums = dw_post is not None or dw_pre is not None or (dgate is not None and shape.gate != GATES["token"])
    buf, at, size = _scratch(scratch, lambda: residual_scratch_size(shape) if sums else 0, dev, stream)
    _call("mosa_residual_norm_backward", dev, stream, shape, _stream_rows(x, "x", sizes, st, dev),
          _stream_rows(y, "y", sizes, st, dev), _array(w_post, "w_post", st, d, dev),
          _gate_rows(gate, "gate", gs, st, dev), _array(w_pre, "w_pre", st, d, dev),
          _stream_rows(dh, "dh", sizes, st, dev), _stream_rows(dn, "dn", sizes, st, dev),
          _stream_rows(dx, "dx", sizes, st, dev), _stream_rows(dy, "dy", sizes, st, dev),
          _array(dw_post, "dw_post", st, d, dev), _gate_rows(dgate, "dgate", gs, st, dev),
          _array(dw_pre, "dw_pre", st, d, dev), at, size)
    return dx, dy, dw_post, dgate, dw_pre


# ---------------------------------------------------------------------------
# products
# ---------------------------------------------------------------------------
def linear_scratch_size(shape):
    """(forward, backward) bytes."""
    f, b = ctypes.c_size_t(), ctypes.c_size_t()
    mosa._check(_lib().mosa_linear_scratch_size(shape, f, b), "mosa_linear_scratch_size")
    return f.value, b.value


def alloc_linear_scratch(shape, device="cuda"):
    """One buffer for the forward and the backward of a shape."""
    return torch.empty(max(*linear_scratch_size(shape), 256), dtype=torch.uint8, device=device)


def _linear_io(shape):
    w = (shape.d_in, shape.d_out) if shape.w_order == 0 else (shape.d_out, shape.d_in)
    return _TORCH[shape.dtype], (shape.rows, shape.d_in), w, (shape.rows, shape.d_out)


def linear(shape, x, w, bias=None, residual=None, y=None, z=None, scratch=None, stream=None):
    """act(x w + bias) + residual of x [rows, d_in], w [d_in, d_out] or [d_out,
    d_in] (w_order), bias [d_out], residual [rows, d_out].  z: x w + bias is written
    too where it is given (linear_backward reads it).  y may be residual.
    Returns y."""
    st, xs, ws, ys = _linear_io(shape)
    dev = _device(x, "x")
    if y is None:
        y = _new(torch.empty, stream, ys, dtype=st, device=dev)
    buf, at, size = _scratch(scratch, lambda: linear_scratch_size(shape)[0], dev, stream)
    _call("mosa_linear", dev, stream, shape, _matrix(x, "x", xs, st, dev), _matrix(w, "w", ws, st, dev),
          _array(bias, "bias", st, shape.d_out, dev), _matrix(residual, "residual", ys, st, dev),
          _matrix(y, "y", ys, st, dev), _matrix(z, "z", ys, st, dev), at, size)
    return y


def linear_backward(shape, x, w, dy, z=None, grads="xw", dx=None, dw=None, db=None, scratch=None, stream=None):
    """Gradients of linear from dy, that of y, and z of the forward (None without
    an activation).  grads: those that are wanted, of "x", "w" and "b"; tensors are
    made for them where none is given.  x may be None where "w" is not wanted, w where
    "x" is not.  The residual's gradient is dy.  Returns (dx, dw, db), None in the place
    of those not wanted."""
    st, xs, ws, ys = _linear_io(shape)
    dev = _device(dy, "dy")
    if not set(grads) <= set("xwb"):
        raise ValueError(f"grads: {grads!r}, expected letters of 'xwb'")

    def wanted(letter, given, sizes):
        if letter not in grads:
            return None
        return _new(torch.empty, stream, sizes, dtype=st, device=dev) if given is None else given
    dx, dw, db = wanted("x", dx, xs), wanted("w", dw, ws), wanted("b", db, (shape.d_out,))
    buf, at, size = _scratch(scratch, lambda: linear_scratch_size(shape)[1], dev, stream)
    _call("mosa_linear_backward", dev, stream, shape, _matrix(x, "x", xs, st, dev), _matrix(w, "w", ws, st, dev),
          _matrix(z, "z", ys, st, dev), _matrix(dy, "dy", ys, st, dev), _matrix(dx, "dx", xs, st, dev),
          _matrix(dw, "dw", ws, st, dev), _array(db, "db", st, shape.d_out, dev), at, size)
    return dx, dw, db


# ---------------------------------------------------------------------------
# log probabilities
# ---------------------------------------------------------------------------
def logprob_scratch_size(shape):
    n = ctypes.c_size_t()
    mosa._check(_lib().mosa_logprob_scratch_size(shape, n), "mosa_logprob_scratch_size")
    return n.value


def alloc_logprob_scratch(shape, device="cuda"):
    return torch.empty(max(logprob_scratch_size(shape), 256), dtype=torch.uint8, device=device)


def token_logprobs(shape, logits, targets=None, logp=None, lse=None, stats=None, entropy=None, top_logp=None,
                   top_index=None, scratch=None, stream=None):
    """Log probabilities of the targets (int32 [rows]; a value outside 0 .. vocab -
    1 is no target: 0) among the rows of logits [rows, vocab], the logits times
    scale.  Returns (logp, lse, top_logp, top_index): logp None without targets, the
    alternatives [rows, top], most probable first, None where the shape has none.
    entropy [rows] and stats [rows, 2] (token_logprobs_backward reads them) are
    written where they are given."""
    dev = _device(logits, "logits")
    R, top = shape.rows, shape.top

    def made(t, sizes, dtype=torch.float32):
        return _new(torch.empty, stream, sizes, dtype=dtype, device=dev) if t is None else t
    logp = made(logp, (R,)) if targets is not None else logp
    lse = made(lse, (R,))
    if top:
        top_logp, top_index = made(top_logp, (R, top)), made(top_index, (R, top), torch.int32)
    buf, at, size = _scratch(scratch, lambda: logprob_scratch_size(shape), dev, stream)
    f32, i32 = torch.float32, torch.int32
    _call("mosa_token_logprobs", dev, stream, shape,
          _matrix(logits, "logits", (R, shape.vocab), _TORCH[shape.dtype], dev), _array(targets, "targets", i32, R, dev),
          _array(logp, "logp", f32, R, dev), _array(lse, "lse", f32, R, dev), _array(stats, "stats", f32, 2 * R, dev),
          _array(entropy, "entropy", f32, R, dev), _array(top_logp, "top_logp", f32, R * top, dev),
          _array(top_index, "top_index", i32, R * top, dev), at, size)
    return logp, lse, top_logp, top_index


def token_logprobs_backward(shape, logits, targets, stats, entropy=None, d_logp=None, d_lse=None, d_entropy=None,
                            d_logits=None, stream=None):
    """Gradient of the logits from those of logp, lse and entropy (fp32 [rows],
    None: 0); stats and entropy are the forward's.  d_logits may be logits.
    Returns d_logits."""
    dev = _device(logits, "logits")
    R, sizes, st, f32 = shape.rows, (shape.rows, shape.vocab), _TORCH[shape.dtype], torch.float32
    if d_logits is None:
        d_logits = _new(torch.empty, stream, sizes, dtype=st, device=dev)
    _call("mosa_token_logprobs_backward", dev, stream, shape, _matrix(logits, "logits", sizes, st, dev),
          _array(targets, "targets", torch.int32, R, dev), _array(stats, "stats", f32, 2 * R, dev, required=True),
          _array(entropy, "entropy", f32, R, dev), _array(d_logp, "d_logp", f32, R, dev),
          _array(d_lse, "d_lse", f32, R, dev), _array(d_entropy, "d_entropy", f32, R, dev),
          _matrix(d_logits, "d_logits", sizes, st, dev))
    return d_logits
