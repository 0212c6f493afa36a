"""The 4-bit cache's attention where its work is cut most: many query rows over many workgroups, more requests than one launch takes,
steps captured into a graph.  Against the plain form in 64 bits, with the tolerances of cache_ref."""
import numpy as np
import pytest
import torch

from tests import cache_ref as ref
from tests.test_cache4_gpu import D, check, expected, i32, make, random_pool, run_attend, tables
from tests.util import up

pytestmark = pytest.mark.gpu

LONG = [  # heads, group, block, lengths, queries, window
    (1, 16, 64, [2500, 700], [301, 150], 0),       # 26 row tiles of one request, cut into as many pieces as there are workgroups
    (2, 16, 16, [1500, 40, 0], [260, 40, 3], 200),  # an odd number of row tiles under a window; as many queries as tokens
    (1, 4, 32, [1800], [49], 0),                  # two tiles, the second of four rows
    (1, 16, 16, [900, 3000, 17], [3, 13, 1], 0),    # 48, 208 and 16 rows: three requests, both kernels
    (1, 3, 64, [6000], [16], 100),                  # 48 rows under a window, all of it in one cut
    (2, 8, 16, [4000, 300], [6, 6], 0),             # 48 rows, cut
    (2, 6, 32, [2000, 900], [5, 2], 0),             # 30 rows, cut
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("case", range(len(LONG)))
def test_long_requests(case, dtype):
    heads, group, block, lens, qlens, window = LONG[case]
    run_attend(np.random.default_rng([17, case]), heads, group, block, lens, qlens, window, dtype, garbage=case % 2 == 1, fused=case % 2 == 0)


@pytest.mark.parametrize("queries", [1, 60])
def test_more_requests_than_one_launch_takes(queries):
    """1100 requests; the last ones have many queries, or one of them does."""
    rng = np.random.default_rng(queries)
    lens = [int(x) for x in rng.integers(0, 40, 1100)]
    qlens = [1] * 1100
    lens[1090], qlens[1090] = 700, queries
    run_attend(rng, 1, 2, 16, lens, qlens, 0, torch.float32, garbage=False, max_len=700)


def test_lists_of_more_requests_than_one_launch_takes():
    rng = np.random.default_rng(31)
    S, heads, group, block, most = 1100, 1, 2, 16, 9
    lens = [int(x) for x in rng.integers(1, 40, S)]
    n_blocks, table = tables(rng, lens, block)
    data = random_pool(rng, n_blocks, heads, block)
    c = make(n_blocks, heads, block, data)
    pos = rng.integers(0, np.array(lens)[:, None, None], (S, heads, most)).astype(np.int32)
    n_tok = rng.integers(0, most + 1, (S, heads)).astype(np.int32)
    q = ref.to_bf16(rng.standard_normal((S, heads * group, D)).astype(np.float32))
    out, lse = c.attend_tokens(up(q), i32(lens), i32(table), i32(pos), i32(n_tok), with_lse=True)
    res = []
    for s in range(S):
        p = pos[s, 0, : n_tok[s, 0]].astype(np.int64)
        k, v = ref.rows(data, table[s, p // block], p % block, 0)
        res.append(ref.softmax_rows(ref.widen(q[s]).astype(np.float64), k, v, np.ones((group, len(p)), dtype=bool), False))
    check(out, lse, [np.stack([r[i] for r in res]) for i in range(4)])


@pytest.mark.parametrize("group,longest,most", [(4, 9, 3), (8, 40, 25)])
def test_queries_beyond_the_most_are_left_as_they_were(group, longest, most):
    """max_query below a request's queries: its first max_query rows are those of the whole call, the others are not touched."""
    rng = np.random.default_rng(longest)
    heads, block, lens, qlens = 1, 16, [500, 60], [longest, 2]
    n_blocks, table = tables(rng, lens, block)
    c = make(n_blocks, heads, block, random_pool(rng, n_blocks, heads, block))
    q = up(ref.to_bf16(rng.standard_normal((longest + 2, heads * group, D)).astype(np.float32)))
    args = (q, i32([0, longest, longest + 2]), i32(lens), i32(table))
    want = expected(ref.widen(q.view(torch.int16).cpu().numpy().view(np.uint16)).astype(np.float64), c.data.cpu().numpy(), table, lens, qlens, block, group,
                    0, False, n_blocks)
    out = torch.full(tuple(q.shape), 7.0, device="cuda")
    lse = torch.full((longest + 2, heads * group), 7.0, device="cuda")
    c.attend(*args, max_query=most, out=out, lse=lse)
    assert bool((out[most:longest] == 7).all()) and bool((lse[most:longest] == 7).all())
    kept = [*range(most), longest, longest + 1]
    check(out[kept], lse[kept], [w[kept] for w in want])


def test_captured_chunks_and_lists_follow_their_lengths():
    """A chunk, a draft and a list attention captured in one graph; lengths, tables, queries and positions change between replays, with
    eager calls of another size in between.  Every replay is compared with an eager call on the same arrays, bit for bit."""
    rng = np.random.default_rng(23)
    heads, group, block, S, width = 2, 4, 16, 3, 40
    n_blocks = 3 * S * width
    c = make(n_blocks, heads, block, random_pool(rng, n_blocks, heads, block))
    tokens = 150
    q = torch.empty((tokens, heads * group, D), dtype=torch.int16, device="cuda")
    start, lens, table = i32(np.zeros(S + 1)), i32(np.zeros(S)), i32(np.zeros((S, width)))
    pos, n_tok = i32(np.zeros((S, heads, 1500))), i32(np.zeros((S, heads)))

    def feed():
        cut = np.sort(rng.integers(0, tokens + 1, S - 1))
        n = rng.integers(0, width * block + 1, S)
        for t, x in ((start, np.concatenate([[0], cut, [tokens]])), (lens, n), (table, rng.permutation(n_blocks)[: S * width].reshape(S, width)),
                     (pos, rng.integers(0, width * block, (S, heads, 1500))), (n_tok, rng.integers(0, 1501, (S, heads)))):
            t.copy_(i32(x))
        q.copy_(torch.from_numpy(ref.to_bf16(rng.standard_normal(tuple(q.shape)).astype(np.float32)).view(np.int16)))

    def calls():
        return [*c.attend(q, start, lens, table, with_lse=True), *c.attend(q, start, lens, table, window=70, out_dtype=torch.bfloat16, with_lse=True),
                *c.attend(q[:S], i32_start, lens, table, max_query=1, with_lse=True), *c.attend_tokens(q[:S], lens, table, pos, n_tok, with_lse=True)]
    i32_start = i32(np.arange(S + 1))
    feed()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = calls()
    with torch.cuda.graph(other):  # a second graph of the same calls has its own scratch
        got_other = calls()
    for i in range(6):
        feed()
        want = [t.clone() for t in calls()]
        for t in got + got_other:
            t.fill_(7.0)
        graph.replay()
        c.attend(q[: 2 * S], i32(2 * np.arange(S + 1)), lens, table, max_query=2)
        other.replay()
        torch.cuda.synchronize()
        for w, g, o in zip(want, got, got_other):
            assert torch.equal(w, g) and torch.equal(w, o), i


@pytest.mark.parametrize("group,queries,lens,dtype", [(2, 1, [150000, 140000, 160000, 147000], torch.float32), (8, 5, [90000, 120000, 105000, 98000], torch.bfloat16),
                                                      (16, 60, [41000, 40500, 41500, 43000], torch.float32)], ids=["few", "draft", "chunk"])
def test_as_many_long_pieces_as_there_are_workgroups(group, queries, lens, dtype):
    """Requests so long that the work is cut into pieces of two or three lengths.  Their blocks are shared: a small pool, long tables."""
    rng = np.random.default_rng(queries)
    heads, block, n_blocks = 1 if queries == 60 else 2, 64, 200
    table = rng.integers(0, n_blocks, (len(lens), -(-max(lens) // block))).astype(np.int32)
    data = random_pool(rng, n_blocks, heads, block)
    run_attend(rng, heads, group, block, lens, [queries] * len(lens), 0, dtype, garbage=False, data=data, table=table)


@pytest.mark.parametrize("requests,heads,most", [(256, 2, 3500), (384, 2, 4100)])
def test_long_lists_of_as_many_units_as_fill_the_card(requests, heads, most):
    """Two or three whole units for every CU, each of many steps: no unit is cut, each list is read to its end."""
    rng = np.random.default_rng(most)
    group, block, n_blocks, width = 1, 32, 150, 20
    data = random_pool(rng, n_blocks, heads, block)
    table = rng.integers(0, n_blocks, (requests, width)).astype(np.int32)
    lens = rng.integers(1, width * block + 1, requests)
    c = make(n_blocks, heads, block, data)
    pos = rng.integers(0, lens[:, None, None], (requests, heads, most)).astype(np.int32)
    n_tok = rng.integers(most - 700, most + 1, (requests, heads)).astype(np.int32)
    q = ref.to_bf16(rng.standard_normal((requests, heads * group, D)).astype(np.float32))
    out, lse = c.attend_tokens(up(q), i32(lens), i32(table), i32(pos), i32(n_tok), with_lse=True)
    res = []
    for s in range(requests):
        at = np.arange(lens[s])
        for h in range(heads):
            k, v = ref.rows(data, table[s, at // block], at % block, h)
            p = pos[s, h, : n_tok[s, h]]
            res.append(ref.softmax_rows(ref.widen(q[s, h: h + 1]).astype(np.float64), k[p], v[p], np.ones((1, len(p)), dtype=bool), False))
    check(out, lse, [np.stack([r[i] for r in res]).reshape(requests, heads, *res[0][i].shape[1:]) for i in range(4)])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("group,queries,window", [(4, 1, 0), (4, 2, 70), (16, 1, 0), (10, 3, 0), (8, 5, 300)])
def test_whole_units_of_many_requests(group, queries, window, dtype):
    """Enough (request, KV head) pairs, short enough, that none is cut: one workgroup each, no scratch; 4 to 40 rows."""
    rng = np.random.default_rng([group, queries])
    lens = [0, 1, queries, 1000] + [int(x) for x in rng.integers(0, 1000, 16)]
    run_attend(rng, 7, group, 16, lens, [queries] * 19 + [0], window, dtype, garbage=False, max_len=1000)
