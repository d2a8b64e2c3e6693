"""The dense heads' operators at the ends of their ranges of sizes."""
import pytest
import torch

from ops_util import rand_rows
from paper_2505_00315_amd import ops

pytestmark = pytest.mark.gpu


def test_tables_of_more_positions_than_rows_may_have():
    """256 sequences, 8 key heads, 2^20 positions of table each: the lengths in use decide, to the bit."""
    B, Hq, Hkv, dh, ps = 256, 16, 8, 32, 64
    g = torch.Generator().manual_seed(1)
    pages = torch.randperm(2 * B, generator=g).to(torch.int32).view(B, 2)
    k, v = (rand_rows(g, B, Hkv, 2 * ps, dh, torch.bfloat16) for _ in range(2))
    q = rand_rows(g, B, Hq, 1, dh, torch.bfloat16)
    lens = torch.randint(0, 2 * ps + 1, (B,), generator=g, dtype=torch.int32).cuda()
    got = []
    for entries in (2, (1 << 20) // ps):
        cs = ops.make_cache_shape(B, Hkv, dh, 2 * B, ps, entries)
        table = torch.full((B, entries), -1, dtype=torch.int32)
        table[:, :2] = pages
        table, cache = table.cuda(), ops.alloc_cache4(cs)
        ops.cache4_append(cs, cache, table, None, k, v, lens=lens)
        shape = ops.make_attn_shape(B, Hq, Hkv, 1, entries * ps, dh)
        got.append(ops.cache4_attention(shape, cs, q, cache, table, lens))
    assert bool(got[0].any()) and torch.equal(*got)
