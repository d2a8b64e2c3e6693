"""Operators of the dense heads: norm and rotation of query and key rows,
attention with a sliding window and first tokens that stay visible, and a paged
cache that holds keys and values in 4 bits.

Python binding of the functions that ``include/mosa.h`` declares for them:
argument marshalling and checks only, every step runs in the HIP kernels.

Rows are tensors of shape [batch, heads, length, d_head] in any memory order
whose last axis is contiguous and whose other strides are multiples of 16
bytes: ``x.transpose(1, 2)`` of a [batch, length, heads, d_head] tensor, a slice
of packed rows, ``mosa.saved_view(shape, saved, "Kd")``.  Work goes to the
current stream of the tensors' device (or ``stream``), whichever device is
current.
"""
import ctypes
import functools
import math

import torch

from . import mosa

PAIRS = {"adjacent": 0, "halves": 1}  # MOSA_PAIRS_*


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


_fn = None


def _lib():
    """The library with the prototypes of these functions (set once)."""
    global _fn
    if _fn is None:
        L = mosa.lib()
        P, V, Z = ctypes.POINTER, ctypes.c_void_p, ctypes.c_size_t
        norm, attn, cache, rows = P(NormShape), P(AttnShape), P(CacheShape), P(Rows)
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
