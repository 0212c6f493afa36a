"""GPU tests of calls of attention to sources whose tables are wide and whose requests are many, and of starts that do not ascend."""
import numpy as np
import pytest
import torch

from tests import cache_ref as ref
from tests import shared_ref as sh
from tests.test_cache4_gpu import check, i32, make, random_pool, tables
from tests.test_shared_gpu import bits
from tests.util import up

pytestmark = pytest.mark.gpu
D = 128


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_many_requests_behind_a_source_in_a_wide_table_without_hints(dtype):
    """900 single tokens of 16 heads a group, 8 KV heads, rows of 128 K tokens: what each request could have is counted once, by the step's tokens."""
    rng = np.random.default_rng(51)
    heads, group, block, n = 8, 16, 16, 900
    lens, qlens, source = [300] + [int(x) for x in rng.integers(1, 30, n)], [0] + [1] * n, [-1] + [0] * n
    n_blocks, table = tables(rng, lens, block)
    table = np.concatenate([table, np.full((n + 1, 8192 - table.shape[1]), -1, np.int32)], 1)
    data = random_pool(rng, n_blocks, heads, block)
    c, start = make(n_blocks, heads, block, data), np.concatenate([[0], np.cumsum(qlens)])
    q = bits(rng, n, heads * group, D)
    plan = i32(sh.sources(source, start, lens, n + 1, n))
    out, lse = c.attend_shared(up(q), i32(start), i32(source), plan, i32(lens), i32(table), out_dtype=dtype, with_lse=True)
    some = np.unique(rng.integers(0, n, 60))  # (the plain form takes a second for so many)
    rows = np.concatenate([[0], 1 + some])
    want = sh.attention(ref.widen(q[some]).astype(np.float64), data, table[rows], [lens[r] for r in rows], [0] + [1] * len(some), [-1] + [0] * len(some), block, group, 0,
                        dtype is torch.bfloat16, True)
    check(out[some], lse[some], want)


@pytest.mark.parametrize("requests", [6, 700])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("queries", [4, 40])
def test_starts_that_do_not_ascend_are_a_step_without_queries(queries, dtype, requests):
    """Requests whose queries overlap would count more work than a call of so many tokens has: rows are left as they were, and the next call is whole."""
    rng = np.random.default_rng([queries, requests])
    heads, group, block, tokens = 2, 4, 16, 3 * queries
    lens, source = [600] + [queries + 3] * (requests - 1), [-1] + [0] * (requests - 1)
    n_blocks, table = tables(rng, lens, block)
    data = random_pool(rng, n_blocks, heads, block)
    c = make(n_blocks, heads, block, data)
    q = bits(rng, tokens, heads * group, D)
    good = np.concatenate([[0, 0], np.minimum((np.arange(requests - 1) + 1) * queries, tokens)])
    bad = good.copy()
    bad[3] = queries - 1  # (behind [0, 0, queries, ...]: one request ends before it begins)
    plan = {name: i32(sh.sources(source, good, lens, requests, tokens)) for name in ("good", "bad")}
    plan["bad"][1] = tokens       # the source's queries end ...
    plan["bad"][2] = tokens - 1   # ... behind the next one's
    outs = []
    for start, listed in ((good, "bad"), (bad, "good"), (bad, "bad"), (good, "good")):
        out = torch.full((tokens, heads * group, D), 7.0, dtype=dtype, device="cuda")
        lse = torch.full((tokens, heads * group), 7.0, device="cuda")
        c.attend_shared(up(q), i32(start), i32(source), plan[listed], i32(lens), i32(table), max_query=queries, out=out, lse=lse)
        outs.append((out, lse))
    for out, lse in outs[:3]:
        assert bool((out == 7).all()) and bool((lse == 7).all())
    want = sh.attention(ref.widen(q).astype(np.float64), data, table, lens, list(np.diff(good)), source, block, group, 0, dtype is torch.bfloat16, True)
    check(*outs[3], want)
    # and attention to the sources alone
    cross = {name: i32(sh.sources(source, good, None, requests, tokens)) for name in ("good", "bad")}
    cross["bad"][1], cross["bad"][2] = tokens, tokens - 1
    for listed in ("bad", "good"):
        out = torch.full((tokens, heads * group, D), 7.0, dtype=dtype, device="cuda")
        lse = torch.full((tokens, heads * group), 7.0, device="cuda")
        c.attend_cross(up(q), cross[listed], i32(lens), i32(table), max_len=6000, out=out, lse=lse)
        if listed == "bad":
            assert bool((out == 7).all()) and bool((lse == 7).all())
    check(out, lse, sh.attention(ref.widen(q).astype(np.float64), data, table, lens, list(np.diff(good)), source, block, group, 0, dtype is torch.bfloat16, True, cross=True))
