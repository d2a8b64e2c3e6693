"""Attention over the 4-bit cache: kv_len bounds positions of a table, no tensor of keys has that extent (no GPU needed)."""
import pytest

from paper_2505_00315_amd import mosa, ops
from test_ops_refusals import A, UNS, WS, rows, status


def shape(**kw):
    return ops.make_attn_shape(**{**dict(batch=256, q_heads=32, kv_heads=8, q_len=1, kv_len=1 << 20, d_head=128), **kw})


def test_long_tables_of_many_sequences():
    """256 sequences and 8 key heads with a table of 2^20 positions each: 2^31 of them together."""
    # 2048 blocks of rows fill the chip, so their keys are not cut into parts
    assert ops.attn_scratch_size(shape()) == (0, 0)


def test_the_longest_tables_of_few_sequences():
    s = shape(batch=4, q_heads=2, kv_heads=2, kv_len=1 << 29)
    forward, backward = ops.attn_scratch_size(s)
    assert forward > 0 and backward == 0
    c = ops.make_cache_shape(4, 2, 128, 4096, 1024, 1 << 19)
    # taken up to the scratch, which is checked last
    assert status("mosa_cache4_attention", s, c, rows(4, 2, 1, 128), A, A, None, A, rows(4, 2, 1, 128), None, A,
                  forward - 1, None) == WS


def test_rows_keep_their_limit():
    s = shape()
    q, k = rows(256, 32, 1, 128), rows(256, 8, 1 << 20, 128)
    assert status("mosa_window_attention", s, q, k, k, None, None, q, None, A, 1 << 40, None) == UNS
    assert status("mosa_window_attention_backward", s, q, k, k, q, A, q, None, None, q, k, k, A, 1 << 40, None) == UNS
    # the largest that rows may have: both directions have their scratch
    most = (1 << 31) // (256 * 8) - 128 - 1
    assert ops.attn_scratch_size(shape(kv_len=most))[1] > 0


@pytest.mark.parametrize("kw", [dict(q_len=1 << 19), dict(kv_len=(1 << 29) + 1)])
def test_limits_of_both(kw):
    with pytest.raises(mosa.MosaError) as e:
        ops.attn_scratch_size(shape(**kw))
    assert e.value.status == UNS
