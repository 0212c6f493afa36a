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
