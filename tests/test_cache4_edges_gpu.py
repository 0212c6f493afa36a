"""Edges of the 4-bit cache's calls, against the plain form in 64 bits."""
import numpy as np
import pytest
import torch

from tests import cache_ref as ref
from tests.test_cache4_gpu import D, check, expected, i32, make, random_pool, run_attend, tables
from tests.util import up

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("heads,group,lens,qlens,window", [(1, 1, [705], [1345], 258), (2, 1, [769, 30], [1921, 5], 256), (1, 4, [200], [500], 40)])
def test_many_more_queries_than_tokens_under_a_window(heads, group, lens, qlens, window, dtype):
    """Whole row tiles of queries stand in front of the first token: they see nothing and get 0 and -inf, the others what they see."""
    run_attend(np.random.default_rng(window), heads, group, 16, lens, qlens, window, dtype, garbage=False)


@pytest.mark.parametrize("queries,window", [(1, 0), (3, 0), (3, 100), (40, 0), (40, 100), (300, 170)])
def test_queries_that_stand_behind_the_tables_row(queries, window):
    """seq_len larger than a row of the table holds: the queries stand where it says, the tokens behind the row do not exist.  The plain
    form has them in blocks that do not exist."""
    rng = np.random.default_rng([queries, window])
    heads, group, block, width = 2, 4, 16, 15
    n_blocks, table = tables(rng, [width * block] * 4, block)
    lens, qlens = [width * block + 1, 300, 90, 5000], [queries, queries, min(queries, 7), queries]
    data = random_pool(rng, n_blocks, heads, block)
    c = make(n_blocks, heads, block, data)
    start = np.concatenate([[0], np.cumsum(qlens)])
    q = ref.to_bf16(rng.standard_normal((int(start[-1]), heads * group, D)).astype(np.float32))
    out, lse = c.attend(up(q), i32(start), i32(lens), i32(table), max_query=max(qlens), window=window, with_lse=True)
    longer = np.full((4, -(-max(lens) // block)), -1, dtype=np.int32)
    longer[:, :width] = table
    check(out, lse, expected(ref.widen(q).astype(np.float64), data, longer, lens, qlens, block, group, window, False, n_blocks))


def test_a_single_token_has_no_row_stride():
    """Tensors of one token whose first stride means nothing: 1, or an odd projection's width."""
    rng = np.random.default_rng(2)
    heads, group, block = 2, 4, 16
    c, other = make(3, heads, block, np.zeros((3, heads, 1, 2176), np.uint8)), make(3, heads, block, np.zeros((3, heads, 1, 2176), np.uint8))
    k, v, q = (up(ref.to_bf16(rng.standard_normal((1, heads * m, D)).astype(np.float32))) for m in (1, 1, group))
    wide = torch.zeros((1, 3 * heads * D + 3), dtype=torch.int16, device="cuda")
    wide[:, heads * D: 2 * heads * D] = v.flatten(1)
    odd_k, odd_v, odd_q = k[0].unsqueeze(-1).permute(2, 0, 1), wide.as_strided((1, heads, D), (wide.shape[1], D, 1), heads * D), q[0].unsqueeze(-1).permute(2, 0, 1)
    assert odd_k.stride(0) == 1 and odd_v.stride(0) % 8 and odd_q.stride(0) == 1
    table, lens, start, slots = i32([[2]]), i32([1]), i32([0, 1]), i32([2 * block])
    c.write(k, v, slots)
    other.write(odd_k, odd_v, slots)
    assert torch.equal(c.data, other.data) and bool(c.data.any())
    assert torch.equal(c.attend(q, start, lens, table), c.attend(odd_q, start, lens, table))
    pos, n_tok = i32(np.zeros((1, heads, 1))), i32(np.ones((1, heads)))
    assert torch.equal(c.attend_tokens(q, lens, table, pos, n_tok), c.attend_tokens(odd_q, lens, table, pos, n_tok))
