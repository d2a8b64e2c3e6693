"""Operators of the dense heads: bad arguments are refused before any device work (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2505_00315_amd import mosa, ops

INV, UNS, WS = mosa.MOSA_ERR_INVALID_ARG, mosa.MOSA_ERR_UNSUPPORTED, mosa.MOSA_ERR_WORKSPACE
A = 0x100000  # an aligned address that is never read


def rows(B, H, T, dh, **kw):
    r = ops.Rows(A, H * T * dh, T * dh, dh)
    for n, v in kw.items():
        setattr(r, n, v)
    return r


def status(f, *args):
    with pytest.raises(mosa.MosaError) as e:
        mosa._check(getattr(ops._lib(), f)(*args), f)
    return e.value.status


@pytest.mark.parametrize("kw,want", [
    (dict(batch=0), INV), (dict(seq_len=0), INV), (dict(q_heads=0), INV), (dict(kv_heads=0), INV),
    (dict(d_head=48), UNS), (dict(d_head=256), UNS), (dict(rope_dim=-2), INV), (dict(rope_dim=66), INV),
    (dict(rope_dim=7), INV), (dict(rope_dim=24, rope_pairs="halves"), INV), (dict(rope_base=1.0), INV),
    (dict(rope_base=float("inf")), INV), (dict(eps=-1e-6), INV), (dict(eps=float("nan")), INV),
    (dict(batch=1 << 16, seq_len=1 << 14), UNS), (dict(q_heads=70000, seq_len=1), UNS),
])
def test_norm_shapes(kw, want):
    base = dict(batch=2, seq_len=8, q_heads=4, kv_heads=2, d_head=64)
    with pytest.raises(mosa.MosaError) as e:
        ops.norm_scratch_size(ops.make_norm_shape(**{**base, **kw}))
    assert e.value.status == want


@pytest.mark.parametrize("kw,want", [
    (dict(batch=0), INV), (dict(q_len=0), INV), (dict(kv_len=0), INV), (dict(q_heads=3), INV), (dict(window=-1), INV),
    (dict(sinks=-1), INV), (dict(scale=0.0), INV), (dict(scale=float("inf")), INV), (dict(scale=float("nan")), INV),
    (dict(d_head=96), UNS), (dict(kv_len=(1 << 29) + 1), UNS), (dict(batch=1 << 20, q_len=4096), UNS),
])
def test_attention_shapes(kw, want):
    base = dict(batch=2, q_heads=4, kv_heads=2, q_len=8, kv_len=8, d_head=64)
    with pytest.raises(mosa.MosaError) as e:
        ops.attn_scratch_size(ops.make_attn_shape(**{**base, **kw}))
    assert e.value.status == want


@pytest.mark.parametrize("kw,want", [
    (dict(batch=0), INV), (dict(kv_heads=0), INV), (dict(pages=0), INV), (dict(max_pages=0), INV),
    (dict(page_size=8), INV), (dict(page_size=24), INV), (dict(page_size=2048), INV), (dict(d_head=80), UNS),
    (dict(max_pages=1 << 26, page_size=16), UNS),
])
def test_cache_shapes(kw, want):
    base = dict(batch=2, kv_heads=2, d_head=64, pages=4, page_size=16, max_pages=2)
    with pytest.raises(mosa.MosaError) as e:
        ops.cache4_size(ops.make_cache_shape(**{**base, **kw}))
    assert e.value.status == want


def test_bad_dtype():
    for s, f in ((ops.make_norm_shape(1, 1, 1, 1, 64), ops.norm_scratch_size),
                 (ops.make_attn_shape(1, 1, 1, 1, 1, 64), ops.attn_scratch_size),
                 (ops.make_cache_shape(1, 1, 64, 1, 16, 1), ops.cache4_size)):
        s.dtype = 2
        with pytest.raises(mosa.MosaError):
            f(s)


def test_cache_size():
    # codes of K and V, and 4 bytes for every 32 values
    assert ops.cache4_size(ops.make_cache_shape(3, 2, 128, 5, 32, 2)) == 5 * 2 * 32 * 2 * (64 + 16)


BAD_ROWS = [dict(data=None), dict(data=A + 8), dict(row_stride=-64), dict(row_stride=68), dict(head_stride=4),
            dict(batch_stride=1 << 41)]


@pytest.mark.parametrize("bad", BAD_ROWS)
@pytest.mark.parametrize("at", range(4))
def test_norm_rows(at, bad):
    s = ops.make_norm_shape(2, 8, 4, 2, 64)
    r = [rows(2, 4, 8, 64), rows(2, 2, 8, 64), rows(2, 4, 8, 64), rows(2, 2, 8, 64)]
    for n, v in bad.items():
        setattr(r[at], n, v)
    assert status("mosa_qk_norm_rope", s, r[0], r[1], None, None, None, r[2], r[3], None) == INV


def test_outputs_may_not_overlap():
    s = ops.make_norm_shape(2, 8, 4, 2, 64)
    q, k = rows(2, 4, 8, 64), rows(2, 2, 8, 64)
    for over in (dict(row_stride=0), dict(row_stride=32), dict(head_stride=7 * 64), dict(batch_stride=0)):
        assert status("mosa_qk_norm_rope", s, q, k, None, None, None, rows(2, 4, 8, 64, **over), k, None) == INV


def test_norm_pointers_and_scratch():
    s = ops.make_norm_shape(2, 8, 4, 2, 64)
    q, k = rows(2, 4, 8, 64), rows(2, 2, 8, 64)
    assert status("mosa_qk_norm_rope", s, q, k, A + 2, None, None, q, k, None) == INV
    assert status("mosa_qk_norm_rope", s, q, k, None, None, A + 1, q, k, None) == INV
    assert status("mosa_qk_norm_rope", s, None, k, None, None, None, q, k, None) == INV

    def back(dwq, scratch, size):
        return status("mosa_qk_norm_rope_backward", s, q, k, A, A, None, q, k, q, k, dwq, None, scratch, size, None)
    need = ops.norm_scratch_size(s)
    assert back(A, None, need) == INV and back(A, A + 16, need) == INV
    assert back(A, A, need - 1) == WS and back(A + 4, A, need) == INV


def attention(s, q=None, k=None, v=None, ql=None, kl=None, out=None, lse=A, scratch=A, size=1 << 40):
    o = lambda r, H, T: rows(s.batch, H, T, s.d_head) if r is None else r
    return ("mosa_window_attention", s, o(q, s.q_heads, s.q_len), o(k, s.kv_heads, s.kv_len),
            o(v, s.kv_heads, s.kv_len), ql, kl, o(out, s.q_heads, s.q_len), lse, scratch, size, None)


def test_attention_pointers():
    s = ops.make_attn_shape(2, 4, 2, 8, 16, 64, window=4, sinks=1)
    for bad in BAD_ROWS:
        if "head_stride" in bad:
            continue
        for n, H, T in (("q", 4, 8), ("k", 2, 16), ("v", 2, 16), ("out", 4, 8)):
            assert status(*attention(s, **{n: rows(2, H, T, 64, **bad)})) == INV
    assert status(*attention(s, ql=A + 2)) == INV
    assert status(*attention(s, kl=A + 1)) == INV
    assert status(*attention(s, lse=A + 2)) == INV
    # broadcast inputs are taken, overlapping outputs are not
    assert status(*attention(s, out=rows(2, 4, 8, 64, head_stride=0))) == INV


def test_attention_scratch():
    s = ops.make_attn_shape(2, 4, 2, 1, 100000, 64)
    fwd, bwd = ops.attn_scratch_size(s)
    assert bwd >= 2 * 4 * 4
    if fwd:
        assert status(*attention(s, scratch=None)) == INV
        assert status(*attention(s, size=16)) == WS
    q, k = rows(2, 4, 1, 64), rows(2, 2, 100000, 64)

    def back(lse, scratch, size):
        return status("mosa_window_attention_backward", s, q, k, k, q, lse, q, None, None, q, k, k, scratch, size, None)
    assert back(None, A, bwd) == INV and back(A, None, bwd) == INV
    assert back(A, A + 64, bwd) == INV and back(A, A, bwd - 1) == WS


def test_cache_calls():
    s = ops.make_cache_shape(2, 2, 64, 4, 16, 2)
    k = rows(2, 2, 8, 64)
    for f in ("mosa_cache4_append", "mosa_cache4_read"):
        assert status(f, s, None, A, None, None, 8, k, k, None) == INV
        assert status(f, s, A + 16, A, None, None, 8, k, k, None) == INV
        assert status(f, s, A, None, None, None, 8, k, k, None) == INV
        assert status(f, s, A, A + 2, None, None, 8, k, k, None) == INV
        assert status(f, s, A, A, A + 2, None, 8, k, k, None) == INV
        assert status(f, s, A, A, None, A + 2, 8, k, k, None) == INV
        assert status(f, s, A, A, None, None, 0, k, k, None) == INV
        for bad in BAD_ROWS[:4]:
            assert status(f, s, A, A, None, None, 8, rows(2, 2, 8, 64, **bad), k, None) == INV
            assert status(f, s, A, A, None, None, 8, k, rows(2, 2, 8, 64, **bad), None) == INV
    assert status("mosa_cache4_read", s, A, A, None, None, 8, rows(2, 2, 8, 64, row_stride=0), k, None) == INV


def test_cache_attention_calls():
    c = ops.make_cache_shape(2, 2, 64, 4, 16, 2)
    q = rows(2, 4, 1, 64)

    def call(s, c=c, cache=A, table=A, kl=A, size=1 << 40):
        return status("mosa_cache4_attention", s, c, q, cache, table, None, kl, q, None, A, size, None)
    ok = dict(batch=2, q_heads=4, kv_heads=2, q_len=1, kv_len=32, d_head=64)
    for kw in (dict(batch=1), dict(kv_heads=1), dict(d_head=32), dict(kv_len=33), dict(dtype="f32")):
        assert call(ops.make_attn_shape(**{**ok, **kw})) == INV
    s = ops.make_attn_shape(**ok)
    assert call(s, cache=None) == INV and call(s, table=None) == INV and call(s, kl=None) == INV
    assert call(s, cache=A + 128) == INV
    if ops.attn_scratch_size(s)[0]:
        assert call(s, size=1) == WS


def test_binding_refuses_cpu_and_wrong_tensors():
    s = ops.make_norm_shape(1, 4, 2, 1, 64)
    q, k = torch.zeros(1, 2, 4, 64, dtype=torch.bfloat16), torch.zeros(1, 1, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU"):
        ops.qk_norm_rope(s, q, k)
    a = ops.make_attn_shape(1, 2, 1, 4, 4, 64)
    with pytest.raises(ValueError, match="GPU"):
        ops.window_attention(a, q, k, k)
    d = torch.device("cpu")
    with pytest.raises(TypeError):
        ops._rows(q, "q", (1, 2, 4, 64), torch.float32, d)
    with pytest.raises(ValueError):
        ops._rows(q, "q", (1, 4, 2, 64), torch.bfloat16, d)
    with pytest.raises(ValueError):
        ops._rows(q.transpose(2, 3), "q", (1, 2, 64, 4), torch.bfloat16, d)
    with pytest.raises(ValueError):
        ops._array(torch.zeros(3, dtype=torch.int32), "lens", torch.int32, 2, d)
    with pytest.raises(TypeError):
        ops._array(torch.zeros(2, dtype=torch.int64), "lens", torch.int32, 2, d)
    with pytest.raises(ValueError):
        ops._array(None, "kv_lens", torch.int32, 2, d, True)
    with pytest.raises(KeyError):
        ops.make_attn_shape(1, 2, 1, 4, 4, 64, dtype=torch.float16)


def test_structs_match_the_header():
    assert ctypes.sizeof(ops.Rows) == 32
    assert ctypes.sizeof(ops.NormShape) == 40
    assert ctypes.sizeof(ops.AttnShape) == 40
    assert ctypes.sizeof(ops.CacheShape) == 28


def test_extents_past_any_memory():
    """Sizes whose products pass 64 bits are refused, not taken modulo 2^64."""
    far = 1 << 40
    s = ops.make_norm_shape(2, 1 << 24, 1, 1, 64)
    k = rows(2, 1, 1 << 24, 64)
    assert status("mosa_qk_norm_rope", s, rows(2, 1, 1 << 24, 64, row_stride=far, batch_stride=64), k, None, None, None,
                  k, k, None) == INV
    assert status("mosa_qk_norm_rope", s, k, k, None, None, None, rows(2, 1, 1 << 24, 64, row_stride=far), k, None) == INV
    for kw in (dict(pages=(1 << 31) - 1, kv_heads=(1 << 31) - 1), dict(pages=1 << 30, kv_heads=1 << 24, page_size=1024)):
        with pytest.raises(mosa.MosaError) as e:
            ops.cache4_size(ops.make_cache_shape(**{**dict(batch=1, kv_heads=1, d_head=64, pages=1, page_size=16,
                                                           max_pages=1), **kw}))
        assert e.value.status == UNS
    # large ones that a device could hold are taken
    assert ops.cache4_size(ops.make_cache_shape(1, 8, 128, 1 << 17, 1024, 1024)) == (1 << 17) * 8 * 1024 * 160
