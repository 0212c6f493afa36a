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


# ------------------------------------------------------------------------------------------------------------- what is refused
def _refusals():
    """(name, call on the good arguments g, the status): what the classes refuse, each a good call with one argument changed."""
    import paper_2604_10539_amd.binding as b
    shape, arg = b.ICE_ERR_SHAPE, b.ICE_ERR_INVALID_ARG

    def write(**change):
        return lambda g: g["cache"].write(**{**dict(k=g["k"], v=g["v"], slots=g["slots"]), **{n: f(g) for n, f in change.items()}})

    def read(**change):
        return lambda g: g["cache"].read(**{**dict(block_table=g["table"], seq_len=g["lens"], n_rows=5), **{n: f(g) for n, f in change.items()}})

    def attend(**change):
        return lambda g: g["cache"].attend(**{**dict(q=g["q"], query_start=g["start"], seq_len=g["lens"], block_table=g["table"], out=g["out"], lse=g["lse"]),
                                              **{n: f(g) for n, f in change.items()}})

    def tokens(**change):
        return lambda g: g["cache"].attend_tokens(**{**dict(q=g["q"], seq_len=g["lens"], block_table=g["table"], token_pos=g["pos"], n_tok=g["n_tok"], out=g["out"],
                                                            lse=g["lse"]), **{n: f(g) for n, f in change.items()}})
    shifted = lambda t: torch.zeros(t.numel() + 1, dtype=t.dtype, device="cuda")[1:].view(t.shape)  # noqa: E731
    rows = {"float32": lambda t: t.float(), "cpu": lambda t: t.cpu(), "64 values": lambda t: t[..., :64], "two dimensions": lambda t: t.flatten(1),
            "not a tensor": lambda t: 7, "none": lambda t: None, "heads apart": lambda t: t.transpose(0, 1).contiguous().transpose(0, 1),
            "values apart": lambda t: t.repeat_interleave(2, 2)[..., ::2], "the same row again": lambda t: t[:1].expand(t.shape)}
    ints = {"int64": lambda t: t.long(), "cpu": lambda t: t.cpu(), "longer": lambda t: torch.cat([t, t]), "apart": lambda t: t.repeat_interleave(2, -1)[..., ::2],
            "float": lambda t: t.float(), "none": lambda t: None}
    out = []
    for make_call, what, kinds in ((write, ("k", "v"), rows), (write, ("slots",), ints), (attend, ("q",), rows), (tokens, ("q",), rows),
                                   (attend, ("start", "lens", "table"), ints), (tokens, ("lens", "table", "pos", "n_tok"), ints), (read, ("lens", "table"), ints)):
        for n in what:
            name = {"start": "query_start", "lens": "seq_len", "table": "block_table", "pos": "token_pos"}.get(n, n)
            for kind, change in kinds.items():
                out.append(("%s %s %s" % (make_call.__name__, name, kind), make_call(**{name: lambda g, n=n, c=change: c(g[n])}), shape))
    for make_call, n in ((write, "k"), (write, "v"), (attend, "q"), (tokens, "q"), (attend, "out"), (tokens, "out")):
        out.append(("%s %s misaligned" % (make_call.__name__, n), make_call(**{n: lambda g, n=n: shifted(g[n])}), arg))
    for make_call in (attend, tokens):
        for n, kinds in (("out", {"float16": lambda t: t.half(), "cpu": lambda t: t.cpu(), "longer": lambda t: torch.cat([t, t]), "apart": lambda t: t.repeat_interleave(2, 2)[..., ::2]}),
                         ("lse", {"bf16": lambda t: t.bfloat16(), "cpu": lambda t: t.cpu(), "longer": lambda t: torch.cat([t, t]), "three": lambda t: t[..., None]})):
            for kind, change in kinds.items():
                out.append(("%s %s %s" % (make_call.__name__, n, kind), make_call(**{n: lambda g, n=n, c=change: c(g[n])}), shape))
        out.append(("%s out_dtype" % make_call.__name__, make_call(out_dtype=lambda g: torch.float16), shape))
        out.append(("%s heads" % make_call.__name__, make_call(q=lambda g: g["q"][:, :5].contiguous(), out=lambda g: None, lse=lambda g: None), shape))
        out.append(("%s 17 heads a group" % make_call.__name__, make_call(q=lambda g: g["q"].repeat(1, 5, 1)[:, :34].contiguous(), out=lambda g: None, lse=lambda g: None),
                    b.ICE_ERR_UNSUPPORTED))
    for n, v in (("window", -1), ("max_query", 0), ("max_query", -1), ("max_len", 0), ("max_len", 2 ** 30 + 1), ("window", 2 ** 31)):
        out.append(("attend %s %d" % (n, v), attend(**{n: lambda g, v=v: v}), shape))
    out.append(("tokens empty lists", tokens(token_pos=lambda g: g["pos"][..., :0].contiguous()), shape))
    out.append(("tokens more queries than requests", tokens(q=lambda g: g["q"].repeat(2, 1, 1), out=lambda g: None, lse=lambda g: None), shape))
    out.append(("write other heads", write(k=lambda g: g["k"][:, :1].contiguous(), v=lambda g: g["v"][:, :1].contiguous()), shape))
    for n, change in (("first", lambda g: i32([0])), ("first", lambda g: i32([0, 0, 0]).long()), ("n_rows", lambda g: -1), ("n_rows", lambda g: 2 ** 31),
                      ("out", lambda g: (None, torch.empty((3, 2, 5, D), device="cuda"))), ("out", lambda g: (torch.empty((3, 2, 4, D), dtype=torch.bfloat16, device="cuda"), None))):
        out.append(("read %s" % n, read(**{n: change}), shape))
    return out


def test_what_the_classes_refuse():
    """Nothing is enqueued, the outputs stay as they are, and the good call works afterwards."""
    from paper_2604_10539_amd import IceError
    rng = np.random.default_rng(12)
    heads, group, block, lens = 2, 4, 16, [20, 5, 40]
    n_blocks, table = tables(rng, lens, block)
    data = random_pool(rng, n_blocks, heads, block)
    q = ref.to_bf16(rng.standard_normal((3, heads * group, D)).astype(np.float32))
    bits = lambda h: up(ref.to_bf16(rng.standard_normal((3, h, D)).astype(np.float32)))  # noqa: E731
    g = dict(cache=make(n_blocks, heads, block, data), k=bits(heads), v=bits(heads), slots=i32([0, 17, 34]), table=i32(table), lens=i32(lens), q=up(q), start=i32([0, 1, 2, 3]),
             pos=i32(rng.integers(0, 5, (3, heads, 7))), n_tok=i32(np.full((3, heads), 7)), out=torch.full((3, heads * group, D), 7.0, device="cuda"),
             lse=torch.full((3, heads * group), 7.0, device="cuda"))
    for name, call, status in _refusals():
        try:
            call(g)
        except IceError as e:
            assert e.status == status, (name, e)
        else:
            raise AssertionError("%s: taken" % name)
    for bad in ((lambda: g["cache"].read(g["table"], g["lens"], 2.5)), (lambda: g["cache"].attend(g["q"], g["start"], g["lens"], g["table"], window=None))):
        with pytest.raises(TypeError):
            bad()
    assert bool((g["out"] == 7).all()) and bool((g["lse"] == 7).all()) and np.array_equal(g["cache"].data.cpu().numpy().reshape(data.shape), data)
    g["cache"].attend(g["q"], g["start"], g["lens"], g["table"], out=g["out"], lse=g["lse"])
    check(g["out"], g["lse"], expected(ref.widen(q).astype(np.float64), data, table, lens, [1, 1, 1], block, group, 0, False, n_blocks))


# ---------------------------------------------------------------------------------------------------- rows among others
FORMS = [(1, 4, [700, 90], [1, 1]), (2, 2, [300, 80], [4, 2]), (2, 4, [900, 40], [4, 3]), (1, 8, [600, 33], [3, 2]), (2, 8, [1500, 300], [6, 6]),
         (2, 4, [2000, 900, 70], [150, 1, 4])]  # rows of up to 5, 8, 16, 32 and 48; many beside few


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("form", range(len(FORMS)))
def test_queries_that_are_not_finite_stay_by_themselves(form, dtype):
    """A NaN or an infinity in a query makes its own row NaN and no other; scores of -inf alone give 0 and -inf."""
    heads, group, lens, qlens = FORMS[form]
    rng = np.random.default_rng([9, form])
    block = 16
    n_blocks, table = tables(rng, lens, block)
    data = random_pool(rng, n_blocks, heads, block)
    data[:, :, :, 64 * np.arange(16)] = data[:, :, :, 64 * np.arange(16)] & 0xF0 | 2  # dimension 0 of every key: its scale's 1
    start = np.concatenate([[0], np.cumsum(qlens)])
    q = ref.to_bf16(rng.standard_normal((int(start[-1]), heads * group, D)).astype(np.float32))
    last = int(start[-1]) - 1
    q[0, 0, 5], q[0, group * heads - 1, 77], q[last, 1, 100], q[start[1] - 1, 1, 3] = 0x7FC0, 0x7F80, 0xFF80, 0xFFFF
    nothing = [(start[1], 0), (start[1] - 1, group * heads - 2)]
    for t, h in nothing:
        q[t, h] = 0
        q[t, h, 0] = 0xFF80  # -inf
    c = make(n_blocks, heads, block, data)
    out, lse = c.attend(up(q), i32(start), i32(lens), i32(table), max_query=max(qlens), out_dtype=dtype, with_lse=True)
    with np.errstate(invalid="ignore"):
        want = expected(ref.widen(q).astype(np.float64), data, table, lens, qlens, block, group, 0, dtype is torch.bfloat16, n_blocks)
    for t, h in nothing:
        for w, x in zip(want, (0.0, -np.inf, 0.0, 1.0)):
            w[t, h] = x
        assert bool((out[t, h] == 0).all())
    want[2] = np.where(want[2] == 0, 1e-37, want[2])
    assert np.isnan(want[0][0, 0]).all() and np.isnan(want[0][last, 1]).all() and np.isfinite(want[0]).any()
    check(out, lse, want)


@pytest.mark.parametrize("window", [0, 60])
def test_requests_of_few_rows_beside_a_chunk_keep_two_terms(window):
    """bf16 outputs of requests with up to 16 rows in a call that has a chunk: their weights have 16 bits, and the bound is that of
    a call without the chunk."""
    rng = np.random.default_rng(window)
    heads, group, block, lens, qlens = 2, 4, 16, [800, 700, 40, 300, 90], [60, 1, 4, 2, 3]
    n_blocks, table = tables(rng, lens, block)
    data = random_pool(rng, n_blocks, heads, block)
    c = make(n_blocks, heads, block, data)
    start = np.concatenate([[0], np.cumsum(qlens)])
    q = ref.to_bf16(rng.standard_normal((int(start[-1]), heads * group, D)).astype(np.float32))
    out, lse = c.attend(up(q), i32(start), i32(lens), i32(table), max_query=max(qlens), window=window, out_dtype=torch.bfloat16, with_lse=True)
    few = slice(int(start[1]), int(start[-1]))  # (the plain form of these requests alone, with a bound for 16 rows)
    check(out[few], lse[few], expected(ref.widen(q[few]).astype(np.float64), data, table[1:], lens[1:], qlens[1:], block, group, window, True, n_blocks))
