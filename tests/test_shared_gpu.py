"""GPU tests of what requests of the 4-bit cache share: tokens that enter rotated, sorted queries, attention to a source and behind one; against
plain forms in numpy."""
import numpy as np
import pytest
import torch

from tests import cache_ref as ref
from tests import shared_ref as sh
from tests.test_cache4_gpu import check, i32, make, random_pool, tables
from tests.util import down, up

pytestmark = pytest.mark.gpu
D = 128


def bits(rng, *shape):
    return ref.to_bf16(rng.standard_normal(shape).astype(np.float32))


def angles(positions, rotated, base=500000.0):
    """float32 [positions, rotated]: cos and sin."""
    half = rotated // 2
    a = np.arange(positions, dtype=np.float64)[:, None] * base ** (-np.arange(half) / half)
    return np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)


# ---------------------------------------------------------------------------------------------------------------- append
APPEND = [  # heads, group, block, lengths, queries, sources, rotated, neighbours, rows of rope
    (1, 1, 16, [1], [1], [-1], 128, False, 40),
    (2, 4, 16, [20, 5, 0, 33, 16], [3, 5, 0, 1, 16], [-1, 3, 0, 99, 4], 128, False, 80),
    (3, 2, 32, [70, 64, 31], [70, 1, 2], [1, -5, 0], 64, False, 120),
    (2, 7, 64, [130, 1, 100], [10, 1, 33], [1, 2, -1], 32, True, 400),
    (8, 4, 16, [400, 300], [7, 200], [1, -1], 96, False, 350),     # positions beyond the table of rotations
    (5, 1, 16, [300, 90, 40], [45, 91, 12], [-1, 2, -1], 128, True, 1000),  # more queries than tokens
    (2, 16, 16, [90] * 70, [1] * 70, [3] * 70, 16, True, 300),     # more requests than a trip looks at
]


def run_append(rng, heads, group, block, lens, qlens, source, rotated, neighbours, positions, width=None, with_q=True, in_place=False, k=None, v=None, q=None):
    n_blocks, table = tables(rng, [min(n, (width or 10 ** 9) * block) for n in lens], block)
    if width:
        table = np.ascontiguousarray(table[:, :width])
    if len(lens) > 1:
        table[len(lens) // 2, -1] = n_blocks  # no such block
    total, behind = sum(qlens), 2
    before = rng.integers(0, 256, (n_blocks, heads, block // 16, 2176), dtype=np.uint8)
    c = make(n_blocks, heads, block, before)
    k, v = (bits(rng, total + behind, heads, D) if x is None else x for x in (k, v))
    q = bits(rng, total + behind, heads * group, D) if q is None else q
    fused = up(np.concatenate([x.reshape(total + behind, -1) for x in (q, k, v)], 1))
    edge = [0, heads * group * D, (heads * group + heads) * D, fused.shape[1]]
    qt, kt, vt = (fused[:, a:b].unflatten(1, ((b - a) // D, D)) for a, b in zip(edge, edge[1:]))
    rope = angles(positions, rotated) if rotated else None
    start = np.concatenate([[0], np.cumsum(qlens)])
    out = None if not with_q else qt if in_place else torch.full((total + behind, heads * group, D), 77, dtype=torch.int16, device="cuda")
    got = c.append(kt, vt, i32(start), i32(lens), i32(table), q=qt if with_q else None, out=out, rope=None if rope is None else up(rope), neighbours=neighbours,
                   source=None if source is None else i32(source))
    data, turned, done = sh.append(before, k, v, q if with_q else None, start, lens, source, table, rope, neighbours, block)
    assert np.array_equal(down(c.data), data)  # (bit for bit, and nothing else was touched)
    if not with_q:
        assert got is None
        return
    assert got is out
    got = down(got.contiguous())
    nan = np.isnan(turned)
    want = ref.to_bf16(np.where(nan, 0, turned))
    stay = q if in_place else np.full(q.shape, 77, np.uint16)
    want = np.where(done[:, None, None], want, stay)
    nan &= done[:, None, None]
    assert np.array_equal(np.isnan(ref.widen(got)) & done[:, None, None], nan) and np.array_equal(got[~nan], want[~nan])
    assert np.array_equal(down(fused)[:, edge[1]:], np.concatenate([k.reshape(total + behind, -1), v.reshape(total + behind, -1)], 1))


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("case", range(len(APPEND)))
def test_tokens_enter_rotated(case, in_place):
    run_append(np.random.default_rng([case, 1]), *APPEND[case], in_place=in_place)


@pytest.mark.parametrize("rotated,neighbours", [(128, False), (96, False), (64, False), (48, False), (32, False), (16, False), (128, True), (80, True), (16, True)])
def test_every_number_of_rotated_dimensions(rotated, neighbours):
    run_append(np.random.default_rng([rotated, 2]), 3, 2, 16, [50, 20], [9, 4], [1, -1], rotated, neighbours, 100)


def test_without_rotations_a_token_is_held_as_it_is():
    """... bit for bit as write() holds it, whatever the position."""
    rng = np.random.default_rng(6)
    run_append(rng, 2, 1, 16, [30, 7, 64], [5, 7, 30], [2, 0, -1], 0, False, 0, with_q=False)
    run_append(rng, 2, 1, 16, [30, 7, 64], [5, 7, 30], None, 64, False, 100, with_q=False)
    heads, block, n = 3, 16, 200
    k, v = (rng.integers(0, 65536, (n, heads, D), dtype=np.uint16) for _ in range(2))
    a, b = (make(16, heads, block, np.zeros((16, heads, 1, 2176), np.uint8)) for _ in range(2))
    table = rng.permutation(16).astype(np.int32)[None]
    slots = table[0, np.arange(n) // block] * block + np.arange(n) % block
    a.write(up(k), up(v), i32(slots))
    b.append(up(k), up(v), i32([0, n]), i32([n]), i32(table))
    assert torch.equal(a.data, b.data) and bool(a.data.any())


def test_rows_of_a_table_that_is_too_short():
    """Tokens behind the row's end are not held; their queries are rotated all the same."""
    run_append(np.random.default_rng(8), 2, 4, 16, [60, 40, 33], [30, 40, 2], [-1, 0, 1], 128, False, 200, width=2)


@pytest.mark.parametrize("neighbours", [False, True])
def test_keys_of_any_size(neighbours):
    """Subnormal to the largest, infinities and NaN: a block with one is held as NaN, a sum that overflows is one."""
    rng = np.random.default_rng(9)
    heads, tokens = 2, 90
    k, v = (rng.integers(0, 65536, (tokens + 2, heads, D), dtype=np.uint16) for _ in range(2))
    k[:40] = np.where((k[:40] & 0x7F80) == 0x7F80, k[:40] & 0xBFFF, k[:40])  # finite
    k[40:60, :, 0::3] = 0x7F7F  # the largest
    e = rng.integers(-126, 127, (20, heads, 4, 1)).astype(np.float64)
    k[60:80] = ref.to_bf16((rng.standard_normal((20, heads, 4, 32)) * np.exp2(e)).clip(-3e38, 3e38).astype(np.float32)).reshape(20, heads, D)
    run_append(rng, heads, 1, 16, [tokens + 50], [tokens], [-1], 128, neighbours, 300, k=k, v=v, q=k.copy())


@pytest.mark.parametrize("requests", [65, 4097, 9000])
def test_every_token_finds_its_request(requests):
    rng = np.random.default_rng(requests)
    heads, block = 1, 16
    gain = rng.choice([0, 1, 1, 2, 9], requests)
    lens = gain + rng.integers(0, 3, requests)
    start = np.concatenate([[0], np.cumsum(gain)])
    total = int(start[-1])
    k, v = bits(rng, total, heads, D), bits(rng, total, heads, D)
    c = make(requests, heads, block, np.zeros((requests, heads, 1, 2176), np.uint8))
    table = rng.permutation(requests).astype(np.int32)[:, None]
    rope = angles(16, 128)
    c.append(up(k), up(v), i32(start), i32(lens), i32(table), rope=up(rope))
    other = make(requests, heads, block, np.zeros((requests, heads, 1, 2176), np.uint8))
    owner = np.repeat(np.arange(requests), gain)
    place = lens[owner] - start[owner + 1] + np.arange(total)
    code, byte = sh.hold(sh.rotate(ref.widen(k), rope[place][:, None, :64], rope[place][:, None, 64:], False))
    other.write(up(k), up(v), i32(table[owner, 0] * block + place))
    want = down(other.data).copy()
    for t in range(total):
        ref.put(want, table[owner[t], 0], 0, place[t], 0, code[t, 0], byte[t, 0])
    assert np.array_equal(down(c.data), want)


# ------------------------------------------------------------------------------------------------------- sorted queries
@pytest.mark.parametrize("same", [True, False], ids=["same table", "another table"])
@pytest.mark.parametrize("requests,rows,most", [(1, 1, 1), (3, 3, 5), (17, 17, 1), (64, 64, 40), (300, 300, 9), (1025, 1025, 3), (8192, 8192, 2), (8192, 1, 1), (1, 8192, 3000),
                                                (5, 2, 2000)])
def test_queries_are_sorted_by_source(requests, rows, most, same):
    from paper_2604_10539_amd import ice_plan_sources
    rng = np.random.default_rng([requests, rows])
    if same:
        rows = requests
    gain = rng.integers(0, most + 1, requests) * (rng.random(requests) < 0.8)
    lens = gain + rng.integers(-most, 50, requests)
    few = rng.integers(0, rows, max(1, rows // 5))
    source = np.where(rng.random(requests) < 0.8, rng.choice(few, requests), rng.choice([-1, rows, 2 ** 31 - 1, -2 ** 31], requests))
    start = np.concatenate([[0], np.cumsum(gain)])
    tokens = int(start[-1]) + int(rng.integers(0, 200))
    plan = torch.full((2 * rows + 2 + 2 * tokens,), 7, dtype=torch.int32, device="cuda")
    ice_plan_sources(i32(source), i32(start), i32(lens) if same else None, plan, rows, tokens)
    assert np.array_equal(down(plan), sh.sources(source, start, lens if same else None, rows, tokens))


# ------------------------------------------------------------------------------------------------------------ attention
def spoil(rng, data, table, lens, block):
    """Garbage, NaN among it, behind every row's last token and in blocks that nobody owns."""
    n_blocks, heads = data.shape[:2]
    junk = random_pool(rng, n_blocks, heads, block, True)
    keep = np.zeros((n_blocks, block), dtype=bool)
    for s, n in enumerate(lens):
        for p in range(min(max(n, 0), table.shape[1] * block)):
            if 0 <= table[s, p // block] < n_blocks:
                keep[table[s, p // block], p % block] = True
    for b, p in np.argwhere(~keep):
        for side in (0, 1):
            at = np.concatenate([1024 * side + 64 * (p % 16) + np.arange(64), 2048 + 64 * side + ref.scale_at(p % 16, np.arange(4))])
            data[b, :, p // 16, at] = junk[b, :, p // 16, at]
            if p % 3 == 0:
                data[b, :, p // 16, 2048 + 64 * side + ref.scale_at(p % 16, np.arange(4))] = 255


def many_of(source, qlens, rows, group, same):
    count = {}
    for s, m in enumerate(qlens):
        r = sh.source_of(source, s, rows, same)
        if r >= 0:
            count[r] = count.get(r, 0) + m
    return max(list(count.values()) or [0])


def run_shared(rng, heads, group, block, lens, qlens, source, window, dtype, cross=False, hints=True, edit=None, data=None, table=None):
    from paper_2604_10539_amd import ice_plan_sources
    if table is None:
        n_blocks, table = tables(rng, [max(0, n) for n in lens], block)
        data = random_pool(rng, n_blocks, heads, block)
        spoil(rng, data, table, lens, block)
    if edit is not None:
        edit(data, table)
    c = make(data.shape[0], heads, block, data)
    total, behind, hq = sum(qlens), 3, heads * group
    q = bits(rng, total, hq, D)
    x = rng.integers(0, 65536, (total + behind, hq * D + 2 * heads * D), dtype=np.uint16)
    x[:total, : hq * D] = q.reshape(total, -1)
    qt = up(x)[:, : hq * D].unflatten(1, (hq, D))
    start = np.concatenate([[0], np.cumsum(qlens)])
    rows, tokens = len(lens), total + behind
    plan = torch.empty(2 * rows + 2 + 2 * tokens, dtype=torch.int32, device="cuda")
    ice_plan_sources(i32(source), i32(start), None if cross else i32(lens), plan, rows, tokens)
    out = torch.full((tokens, hq, D), 7.0, dtype=dtype, device="cuda")
    lse = torch.full((tokens, hq), 7.0, dtype=torch.float32, device="cuda")
    shared = many_of(source, qlens, rows, group, not cross)
    known = dict(max_shared=max(shared, 1), max_len=max(max(lens), 1)) if hints else {}
    if cross:
        c.attend_cross(qt, plan, i32(lens), i32(table), out=out, lse=lse, **known)
        most = shared if hints else tokens
    else:
        if hints:
            known.update(max_query=max(max(qlens), 1), max_source=max(max(lens), 1))
        c.attend_shared(qt, i32(start), i32(source), plan, i32(lens), i32(table), window=window, out=out, lse=lse, **known)
        most = max(shared, max(qlens)) if hints else tokens
    assert bool((out[total:] == 7).all()) and bool((lse[total:] == 7).all())
    want = sh.attention(ref.widen(q).astype(np.float64), data, table, lens, qlens, source, block, group, window, dtype is torch.bfloat16, most * group > 16, cross)
    want[2] = np.maximum(want[2], 1e-37)
    check(out[:total], lse[:total], want)


SHARED = [  # heads, group, block, lengths, queries, sources, window
    (1, 1, 16, [5, 1], [0, 1], [-1, 0], 0),
    (2, 4, 16, [40, 3, 1, 17], [0, 1, 1, 1], [-1, 0, 0, 0], 0),                         # rows of one source: 12
    (2, 4, 16, [700, 30, 0, 9, 300, 64, 1], [0, 1, 0, 1, 0, 1, 1], [-1, 0, 0, 4, -1, 0, 4], 0),  # two sources, two waiting
    (1, 16, 32, [900, 50, 40, 30, 1], [0, 1, 1, 1, 1], [-1, 0, 0, 0, 0], 0),             # 64 rows of a source, 16 of a request
    (2, 2, 64, [1000, 100, 65, 64, 63, 20], [0, 4, 4, 4, 3, 4], [-1, 0, 0, 0, 0, -1], 0),  # drafts; one request without a source
    (2, 8, 16, [333, 70, 30], [0, 40, 17], [-1, 0, 0], 0),                               # chunks: 456 rows of a source
    (1, 4, 16, [2000, 300, 200, 5], [0, 150, 1, 5], [-1, 0, 0, 0], 0),                   # chunks beside single tokens
    (1, 4, 16, [500, 60, 100, 5], [0, 2, 90, 5], [-1, 0, 0, 0], 80),                     # windows that end in the source, at its end, behind it
    (2, 2, 32, [600, 90, 40, 500, 7], [0, 3, 2, 0, 1], [-1, 0, 3, -1, 3], 64),
    (1, 1, 16, [300, 20, 10], [0, 1, 1], [-1, 0, 0], 1),                                 # a window of the query's own token
    (1, 3, 16, [50, 4, 0, 2], [0, 9, 3, 1], [-1, 0, 0, 2], 0),                           # more queries than tokens; a source without tokens
    (2, 4, 16, [100, 40, 30], [2, 1, 3], [0, 0, 1], 0),                                  # a row that names itself, a source with queries of its own, a source's source
    (1, 4, 64, [3000, 200] + [17] * 20, [0, 0] + [1] * 20, [-1, -1] + [0, 1] * 10, 0),
    (1, 2, 16, [4500, 1200, 33], [0, 100, 30], [-1, 0, 0], 900),
]


@pytest.mark.parametrize("hints", [True, False], ids=["hints", "none"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("case", range(len(SHARED)))
def test_attention_behind_a_source(case, dtype, hints):
    run_shared(np.random.default_rng([case, 3]), *SHARED[case], dtype, hints=hints)


CROSS = [  # heads, group, block, lengths of the sources, queries, sources
    (1, 1, 16, [1], [1], [0]),
    (2, 2, 16, [100, 7, 0], [1, 1, 1, 1, 1], [0, 1, 0, 2, -1]),
    (1, 8, 32, [1500], [1, 1, 1, 1, 1], [0] * 5),
    (3, 5, 64, [300, 129, 64], [3, 0, 4, 1], [2, 0, 0, 3]),
    (2, 4, 16, [200, 333], [40, 70, 11], [1, 1, 0]),
    (1, 16, 16, [77, 2000], [100, 3], [1, 0]),
    (2, 1, 16, [500] * 3, [1] * 200, [0, 1, 2, 0] * 50),
]


@pytest.mark.parametrize("hints", [True, False], ids=["hints", "none"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("case", range(len(CROSS)))
def test_attention_to_a_source(case, dtype, hints):
    heads, group, block, lens, qlens, source = CROSS[case]
    run_shared(np.random.default_rng([case, 4]), heads, group, block, lens, qlens, source, 0, dtype, cross=True, hints=hints)


def test_more_rows_than_one_launch_takes():
    rng = np.random.default_rng(11)
    n = 1500
    source = np.where(np.arange(n) % 7 == 3, -1, np.array([1400, 5])[np.arange(n) % 2])
    lens = [40 if s in (5, 1400) else int(x) for s, x in enumerate(rng.integers(1, 12, n))]
    qlens = [0 if s in (5, 1400) else 1 for s in range(n)]
    run_shared(rng, 1, 2, 16, lens, qlens, source, 0, torch.float32)
    run_shared(rng, 1, 2, 16, lens, qlens, source, 0, torch.float32, cross=True)


@pytest.mark.parametrize("cross", [False, True])
@pytest.mark.parametrize("queries", [1, 30])
def test_blocks_that_do_not_exist_and_values_held_as_nan(queries, cross):
    """A source's missing block is left out; a NaN among its values reaches the rows that see it (of a window, some do not)."""
    def edit(data, table):
        table[0, 1], table[0, 5], table[2, 0] = -1, data.shape[0], 2 ** 31 - 1
        data[table[0, 3], 0, 0, 2112 + ref.scale_at(9, 2)] = 255
        data[table[0, 7], -1, 0, 2048 + ref.scale_at(2, 1)] = 255
    lens, qlens, source = [160, 30, 40, 25], [0, queries, 1, 1], [-1, 0, 0, 0]
    for window in (0, 125) if not cross else (0,):
        run_shared(np.random.default_rng([queries, window]), 2, 4, 16, lens, qlens, source, window, torch.float32, cross=cross, edit=edit)


@pytest.mark.parametrize("group", [1, 3, 5, 6, 7, 9, 11, 13, 14, 16])
def test_row_tiles_of_whole_tokens(group):
    """Groups that do not divide a tile's 192 rows: a token's rows stay in one tile; one tile of up to 128 rows, several of them, chunks of a request's own."""
    rng = np.random.default_rng([group, 17])
    run_shared(rng, 1, group, 16, [300, 40, 9], [0, 100 // group, 1], [-1, 0, 0], 0, torch.float32)
    run_shared(rng, 2, group, 32, [450, 170, 60, 40], [0, 800 // group, 60 // group + 1, 2], [-1, 0, 0, -1], 0, torch.bfloat16)
    run_shared(rng, 1, group, 16, [270, 30], [700 // group, 3, 0], [1, 0, 0], 0, torch.float32, cross=True)


@pytest.mark.parametrize("longest,source", [(1, 1), (20, 200), (90000, 1), (1, 500000)])
def test_any_hint_of_the_lengths_gives_the_result(longest, source):
    rng = np.random.default_rng(longest)
    heads, group, block, lens, qlens, named = 2, 4, 16, [1500, 300, 33, 700, 5], [0, 1, 30, 2, 1], [-1, 0, 0, 0, -1]
    n_blocks, table = tables(rng, lens, block)
    data = random_pool(rng, n_blocks, heads, block)
    c, start = make(n_blocks, heads, block, data), np.concatenate([[0], np.cumsum(qlens)])
    q = bits(rng, int(start[-1]), heads * group, D)
    plan = i32(sh.sources(named, start, lens, 5, int(start[-1])))
    want = sh.attention(ref.widen(q).astype(np.float64), data, table, lens, qlens, named, block, group, 0, False, True)
    check(*c.attend_shared(up(q), i32(start), i32(named), plan, i32(lens), i32(table), max_len=longest, max_source=source, with_lse=True), want)
    plan = i32(sh.sources(named, start, None, 5, int(start[-1])))
    want = sh.attention(ref.widen(q).astype(np.float64), data, table, lens, qlens, named, block, group, 0, False, True, cross=True)
    check(*c.attend_cross(up(q), plan, i32(lens), i32(table), max_len=source, with_lse=True), want)


@pytest.mark.parametrize("max_query,max_shared", [(2, 9), (9, 4), (3, 5), (70, 40), (20, 90), (30, 30)])
def test_queries_beyond_the_most_are_left_as_they_were(max_query, max_shared):
    """Of a request those behind its first max_query, of a source those behind the first max_shared of its list; the others get their results."""
    rng = np.random.default_rng([max_query, max_shared])
    many = max(max_query, max_shared) > 12
    heads, group, block, lens = 2, 4, 16, [400, 90, 120, 64]
    qlens, named = ([0, 60, 40, 25] if many else [0, 3, 5, 4]), [-1, 0, 0, -1]
    n_blocks, table = tables(rng, lens, block)
    data = random_pool(rng, n_blocks, heads, block)
    c, start = make(n_blocks, heads, block, data), np.concatenate([[0], np.cumsum(qlens)])
    total = int(start[-1])
    q = bits(rng, total, heads * group, D)
    place = np.arange(total) - np.repeat(start[:-1], qlens)
    in_list = np.where(np.arange(total) < start[3], np.arange(total), 0)  # (the two requests behind row 0 stand one after the other)
    for cross in (False, True):
        plan = i32(sh.sources(named, start, None if cross else lens, 4, total))
        out, lse = torch.full((total, heads * group, D), 7.0, device="cuda"), torch.full((total, heads * group), 7.0, device="cuda")
        if cross:
            c.attend_cross(up(q), plan, i32(lens), i32(table), max_shared=max_shared, out=out, lse=lse)
            there = in_list < max_shared
        else:
            c.attend_shared(up(q), i32(start), i32(named), plan, i32(lens), i32(table), max_query=max_query, max_shared=max_shared, out=out, lse=lse)
            there = (place < max_query) & (in_list < max_shared)
        want = sh.attention(ref.widen(q).astype(np.float64), data, table, lens, qlens, named, block, group, 0, False, True, cross)
        want[2] = np.maximum(want[2], 1e-37)
        assert there.any()
        at = torch.from_numpy(there).cuda()
        check(out[at], lse[at], [w[there] for w in want])
        assert bool((out[~at] == 7).all()) and bool((lse[~at] == 7).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("group,queries,window", [(4, 1, 0), (2, 2, 700), (4, 1, 4500), (1, 3, 0), (3, 1, 5000), (2, 1, 4999)])
def test_few_rows_of_a_source_in_a_call_that_is_not_small(group, queries, window, dtype):
    """Two sources of 17 to 48 rows, requests of up to six; eight KV heads."""
    n = 12
    lens = [5000, 4700] + [40 + 53 * i % 300 for i in range(n)]
    run_shared(np.random.default_rng([group, queries, window]), 8, group, 16, lens, [0, 0] + [queries] * n, [-1, -1] + [0] * 7 + [1] * 5, window, dtype)


@pytest.mark.parametrize("requests", [3, 70])
def test_rows_in_front_of_the_first_request_are_nobodys(requests):
    """A step whose first rows belong to other work: the rest is as if they were not there, and they stay as they were."""
    rng = np.random.default_rng(requests)
    heads, group, block, front, behind = 2, 4, 16, 5, 3
    lens, qlens, named = [100] + [20] * (requests - 1), [0] + [2] * (requests - 1), [-1] + [0, -1] * requests
    named = named[:requests]
    n_blocks, table = tables(rng, lens, block)
    data = random_pool(rng, n_blocks, heads, block)
    start = np.concatenate([[0], np.cumsum(qlens)]) + front
    total = int(start[-1]) + behind
    k, v, q = bits(rng, total, heads, D), bits(rng, total, heads, D), bits(rng, total, heads * group, D)
    rope = up(angles(200, 128))

    def step(rows, start, out, lse):
        c = make(n_blocks, heads, block, data)
        args = i32(start), i32(lens), i32(table)
        turned = up(q[rows])
        c.append(up(k[rows]), up(v[rows]), *args, q=turned, out=turned, rope=rope, source=i32(named))
        plan = i32(sh.sources(named, start, lens, requests, len(turned)))
        c.attend_shared(turned, args[0], i32(named), plan, *args[1:], max_query=2, max_shared=2 * requests, out=out, lse=lse)
        return c.data, turned

    full = [torch.full((total, heads * group, *d), 7.0, device="cuda") for d in ((D,), ())]
    less = [x[front:].clone() for x in full]
    data0, q0 = step(slice(None), start, *full)
    data1, q1 = step(slice(front, None), start - front, *less)
    assert torch.equal(data0, data1) and torch.equal(q0[front:], q1) and np.array_equal(down(q0[:front].contiguous()), q[:front])
    for x, y in zip(full, less):
        assert torch.equal(x[front:].view(torch.int32), y.view(torch.int32)) and bool((x[:front] == 7).all()) and bool((x[-behind:] == 7).all())


def test_a_negative_number_of_rows_is_refused():
    from paper_2604_10539_amd import IceBlocks, IceError
    b = IceBlocks(8, 16, 2, 64)
    for n in (-1, -100):
        with pytest.raises(IceError):
            b.plan_sources(i32([-1, 0]), n)


def test_units_of_few_rows_beside_a_chunk_keep_two_terms():
    """bf16 outputs of requests and sources with up to 16 rows in a call that has a chunk: their weights have 16 bits."""
    rng = np.random.default_rng(18)
    heads, group, block, lens, qlens, named = 2, 4, 16, [500, 700, 90, 300, 40, 200], [0, 0, 1, 2, 1, 60], [-1, -1, 0, 0, 0, 1]
    n_blocks, table = tables(rng, lens, block)
    data = random_pool(rng, n_blocks, heads, block)
    c, start = make(n_blocks, heads, block, data), np.concatenate([[0], np.cumsum(qlens)])
    q = bits(rng, 64, heads * group, D)
    for cross in (False, True):
        plan = i32(sh.sources(named, start, None if cross else lens, 6, 64))
        got = c.attend_cross(up(q), plan, i32(lens), i32(table), out_dtype=torch.bfloat16, with_lse=True) if cross else \
            c.attend_shared(up(q), i32(start), i32(named), plan, i32(lens), i32(table), out_dtype=torch.bfloat16, with_lse=True)
        want = sh.attention(ref.widen(q).astype(np.float64), data, table, lens, qlens, named, block, group, 0, True, False, cross)
        check(got[0][:4], got[1][:4], [w[:4] for w in want])


@pytest.mark.parametrize("group,queries,requests,longest,dtype", [(16, 1, 6, 102000, torch.bfloat16), (1, 1, 3, 150000, torch.float32), (4, 40, 3, 35000, torch.bfloat16)])
def test_a_long_source(group, queries, requests, longest, dtype):
    """As many long pieces as there are workgroups, of the two lengths that two to a CU get, or the three of three."""
    rng = np.random.default_rng([queries, requests])
    heads, block = 8, 64
    lens = [longest] + [int(x) for x in rng.integers(queries, 200, requests)]
    n_blocks, table = tables(rng, lens, block)
    data = rng.integers(0, 256, (n_blocks, heads, 4, 2176), dtype=np.uint8)
    data[..., 2048:] = 124 + data[..., 2048:] % 3  # scales of 1 / 8 to 1 / 2
    run_shared(rng, heads, group, block, lens, [0] + [queries] * requests, [-1] + [0] * requests, 0, dtype, data=data, table=table)


def test_sources_that_are_longer_than_the_tables_row():
    """Queries stand behind the source's length all the same; its tokens behind the row do not exist."""
    rng = np.random.default_rng(13)
    heads, block, width = 2, 16, 6
    n_blocks, table = tables(rng, [width * block] * 3, block)
    data = random_pool(rng, n_blocks, heads, block)
    for window in (0, 60):
        run_shared(rng, heads, 4, block, [130, 50, 96], [0, 3, 20], [-1, 0, 0], window, torch.float32, data=data, table=table)
    run_shared(rng, heads, 4, block, [130, 50, 96], [0, 3, 20], [-1, 0, 1], 0, torch.float32, cross=True, data=data, table=table)


def test_equal_to_one_long_request():
    """A request behind a source, and the same text in one row by attend: both within the bounds of the one plain form."""
    rng = np.random.default_rng(14)
    heads, group, block, before, own, m = 2, 4, 16, 96, 40, 5
    n_blocks, table = tables(rng, [before, own], block)
    data = random_pool(rng, n_blocks, heads, block)
    c = make(n_blocks, heads, block, data)
    q = bits(rng, m, heads * group, D)
    from paper_2604_10539_amd import ice_plan_sources
    source, start, lens = i32([-1, 0]), i32([0, 0, m]), i32([before, own])
    plan = torch.empty(2 * 2 + 2 + 2 * m, dtype=torch.int32, device="cuda")
    ice_plan_sources(source, start, lens, plan, 2, m)
    one = np.concatenate([table[0, : before // block], table[1, : -(-own // block)]])[None]
    for window in (0, 50):
        want = sh.attention(ref.widen(q).astype(np.float64), data, one, [before + own], [m], [-1], block, group, window, False, True)
        check(*c.attend_shared(up(q), start, source, plan, lens, i32(table), window=window, with_lse=True), want)
        check(*c.attend(up(q), i32([0, m]), i32([before + own]), i32(one), window=window, with_lse=True), want)


def test_a_pool_beyond_32_bit_offsets():
    rng = np.random.default_rng(15)
    heads, block = 2, 64
    n_blocks = 2 ** 32 // (heads * 4 * 2176) + 400
    from paper_2604_10539_amd import IceCache, ice_plan_sources
    c = IceCache(n_blocks, heads, block)
    c.data[-8:] = 0
    table = np.array([[n_blocks - 1, n_blocks - 3], [n_blocks - 2, n_blocks - 5]], dtype=np.int32)
    lens, qlens, source = [100, 70], [100, 70], [-1, 0]
    k, v, q = bits(rng, 170, heads, D), bits(rng, 170, heads, D), bits(rng, 170, heads * 2, D)
    start, rope = np.concatenate([[0], np.cumsum(qlens)]), angles(200, 128)
    got = c.append(up(k), up(v), i32(start), i32(lens), i32(table), q=up(q), rope=up(rope), source=i32(source))
    small, turned, _ = sh.append(np.zeros((8, heads, 4, 2176), np.uint8), k, v, q, start, lens, source, table - (n_blocks - 8), rope, False, block)
    assert np.array_equal(down(c.data[-8:]), small) and np.array_equal(down(got), ref.to_bf16(turned))
    plan = torch.empty(2 * 2 + 2 + 2 * 170, dtype=torch.int32, device="cuda")
    ice_plan_sources(i32(source), i32(start), i32(lens), plan, 2, 170)
    out, lse = c.attend_shared(got, i32(start), i32(source), plan, i32(lens), i32(table), with_lse=True)
    want = sh.attention(ref.widen(ref.to_bf16(turned)).astype(np.float64), small, table - (n_blocks - 8), lens, qlens, source, block, 2, 0, False, True)
    check(out, lse, want)


@pytest.mark.parametrize("shape", [(0, 128), (0, 0), (5, 0)])
def test_an_empty_table_of_rotations_is_refused(shape):
    """Nothing is held: without the refusal keys would enter as they are."""
    import paper_2604_10539_amd.binding as b
    from paper_2604_10539_amd import IceError
    rng = np.random.default_rng(52)
    c = make(4, 2, 16)
    c.data.fill_(9)
    k, v, q = up(bits(rng, 3, 2, D)), up(bits(rng, 3, 2, D)), up(bits(rng, 3, 4, D))
    for queries in (None, q):
        with pytest.raises(IceError) as e:
            c.append(k, v, i32([0, 3]), i32([3]), i32([[1]]), q=queries, rope=torch.empty(shape, device="cuda"))
        assert e.value.status == b.ICE_ERR_SHAPE
    assert bool((c.data == 9).all())


# ---------------------------------------------------------------------------------------------------------- as they are used
class Server:
    """Two layers' caches, a shared prompt in row 0, requests behind it, and the same in numpy."""

    def __init__(self, seed, requests=5, heads=2, group=4, block=16):
        from paper_2604_10539_amd import IceBlocks, IceCache
        self.rng, self.n, self.heads, self.group, self.block = np.random.default_rng(seed), requests, heads, group, block
        self.blocks = IceBlocks(64, block, requests, 400)
        self.caches = [IceCache(64, heads, block) for _ in range(2)]
        for c in self.caches:
            c.data.zero_()
        self.data = [down(c.data).copy() for c in self.caches]
        self.rope = angles(900, 128)
        self.rope_gpu = up(self.rope)
        self.room = 48
        self.new_len, self.source = i32([0] * requests), i32([-1] + [0] * (requests - 1))
        shape = (self.room, (group + 2) * heads, D)
        self.x = [torch.zeros(shape, dtype=torch.int16, device="cuda") for _ in self.caches]
        self.out = [torch.zeros((self.room, group * heads, D), device="cuda") for _ in self.caches]
        self.lse = [torch.zeros((self.room, group * heads), device="cuda") for _ in self.caches]

    def feed(self, gain):
        self.x_np = [bits(self.rng, *x.shape) for x in self.x]
        for x, y in zip(self.x, self.x_np):
            x.copy_(up(y))
        self.new_len.copy_(i32(gain))

    def step(self):
        hq, h = self.group * self.heads, self.heads
        start, _, _ = self.blocks.plan(self.new_len, self.room)
        plan = self.blocks.plan_sources(self.source, self.room)
        for c, x, out, lse in zip(self.caches, self.x, self.out, self.lse):
            q = c.append(x[:, hq: hq + h], x[:, hq + h:], start, self.blocks.seq_len, self.blocks.block_table, q=x[:, :hq], rope=self.rope_gpu, source=self.source)
            c.attend_shared(q, start, self.source, plan, self.blocks.seq_len, self.blocks.block_table, out=out, lse=lse)

    def check(self):
        hq, h = self.group * self.heads, self.heads
        start, lens, table, source = (down(x) for x in (self.blocks.query_start, self.blocks.seq_len, self.blocks.block_table, self.source))
        qlens = np.diff(start)
        for i, x in enumerate(self.x_np):
            self.data[i], turned, _ = sh.append(self.data[i], x[:, hq: hq + h], x[:, hq + h:], x[:, :hq], start, lens, source, table, self.rope, False, self.block)
            assert np.array_equal(down(self.caches[i].data), self.data[i])
            total = int(start[-1])
            want = sh.attention(ref.widen(ref.to_bf16(turned))[:total].astype(np.float64), self.data[i], table, lens, list(qlens), source, self.block, self.group, 0,
                                False, True)
            check(self.out[i][:total], self.lse[i][:total], want)


GAINS = [[40, 0, 0, 0, 0], [0, 9, 1, 17, 3], [0, 1, 1, 1, 1], [5, 1, -1, 1, 1], [0, 1, 1, -400, 4], [0, 1, 1, 20, 1]]


def test_steps_behind_a_shared_prompt():
    s = Server(21)
    for gain in GAINS:
        s.feed(gain)
        s.step()
        s.check()
    assert down(s.blocks.seq_len)[3] == 20 and int(s.blocks.info[3]) == 0


def test_a_captured_step_is_replayed():
    """Two graphs of the same step, replayed in turn beside eager steps: each step's results are those of the plain form."""
    s = Server(22)
    s.feed(GAINS[0])
    s.step()
    s.check()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        s.new_len.zero_()
        with torch.cuda.graph(g):
            s.step()
        graphs.append(g)
    for i, gain in enumerate(GAINS[1:] + GAINS[1:3]):
        s.feed(gain)
        if i == 2:
            s.step()
        else:
            graphs[i % 2].replay()
        torch.cuda.synchronize()
        s.check()


def test_calls_on_two_streams_at_once():
    servers = [Server(23), Server(24)]
    streams = [torch.cuda.Stream() for _ in servers]
    for gain in GAINS[:3]:
        for s in servers:
            s.feed(gain)
        torch.cuda.synchronize()
        for s, stream in zip(servers, streams):
            with torch.cuda.stream(stream):
                s.step()
        torch.cuda.synchronize()
        for s in servers:
            s.check()


def test_a_stream_that_is_handed_over():
    s, stream = Server(25), torch.cuda.Stream()
    s.feed(GAINS[0])
    s.step()
    s.check()
    s.feed(GAINS[1])
    torch.cuda.synchronize()
    hq, h = s.group * s.heads, s.heads
    start, _, _ = s.blocks.plan(s.new_len, s.room, stream=stream)
    plan = s.blocks.plan_sources(s.source, s.room, stream=stream.cuda_stream)
    for c, x, out, lse in zip(s.caches, s.x, s.out, s.lse):
        q = c.append(x[:, hq: hq + h], x[:, hq + h:], start, s.blocks.seq_len, s.blocks.block_table, q=x[:, :hq], rope=s.rope_gpu, source=s.source, stream=stream)
        c.attend_shared(q, start, s.source, plan, s.blocks.seq_len, s.blocks.block_table, out=out, lse=lse, stream=stream)
        other = torch.zeros_like(out)
        c.attend_cross(q, plan, s.blocks.seq_len, s.blocks.block_table, out=other, stream=stream)
    torch.cuda.synchronize()
    s.check()
    total = int(start[-1])
    turned = ref.widen(down(q))[:total].astype(np.float64)
    want = sh.attention(turned, s.data[1], down(s.blocks.block_table), down(s.blocks.seq_len), list(np.diff(down(start))), down(s.source), s.block, s.group, 0, False,
                        True, cross=True)
    check(other[:total], torch.from_numpy(want[1]), want)


def test_the_same_call_gives_the_same_bits():
    rng = np.random.default_rng(31)
    heads, group, block = 8, 4, 64
    lens, qlens = [5000] + [int(x) for x in rng.integers(1, 700, 40)], [0] + [1] * 38 + [30, 7]
    n_blocks, table = tables(rng, lens, block)
    c = make(n_blocks, heads, block, random_pool(rng, n_blocks, heads, block))
    q = up(bits(rng, sum(qlens), heads * group, D))
    from paper_2604_10539_amd import ice_plan_sources
    source, start, lens_t, table_t = i32([-1] + [0] * 40), i32(np.concatenate([[0], np.cumsum(qlens)])), i32(lens), i32(table)
    plan = torch.empty(2 * 41 + 2 + 2 * sum(qlens), dtype=torch.int32, device="cuda")
    ice_plan_sources(source, start, lens_t, plan, 41, sum(qlens))
    for dtype in (torch.float32, torch.bfloat16):
        first = c.attend_shared(q, start, source, plan, lens_t, table_t, out_dtype=dtype, with_lse=True)
        for _ in range(5):
            again = c.attend_shared(q, start, source, plan, lens_t, table_t, out_dtype=dtype, with_lse=True)
            assert all(torch.equal(x, y) for x, y in zip(first, again))


# ------------------------------------------------------------------------------------------------------- what is refused
def test_what_the_classes_refuse():
    """Nothing is enqueued, outputs and cache stay as they are, and the good calls work afterwards."""
    import paper_2604_10539_amd.binding as b
    from paper_2604_10539_amd import IceBlocks, IceError
    rng = np.random.default_rng(41)
    heads, group, block, lens, qlens = 2, 4, 16, [20, 5, 40], [1, 1, 1]
    n_blocks, table = tables(rng, lens, block)
    data = random_pool(rng, n_blocks, heads, block)
    c = make(n_blocks, heads, block, data)
    rows = lambda h: up(bits(rng, 3, h, D))  # noqa: E731
    plan = sh.sources([-1, 0, 0], [0, 1, 2, 3], lens, 3, 3)
    g = dict(q=rows(heads * group), k=rows(heads), v=rows(heads), query_start=i32([0, 1, 2, 3]), seq_len=i32(lens), block_table=i32(table), source=i32([-1, 0, 0]),
             plan=i32(plan), rope=up(angles(70, 64)), out=torch.full((3, heads * group, D), 7.0, device="cuda"), lse=torch.full((3, heads * group), 7.0, device="cuda"))
    turned = torch.full((3, heads * group, D), 7, dtype=torch.int16, device="cuda")
    calls = {"append": (c.append, ("k", "v", "query_start", "seq_len", "block_table", "q", "rope", "source"), dict(out=turned)),
             "attend_cross": (c.attend_cross, ("q", "plan", "seq_len", "block_table", "out", "lse"), {}),
             "attend_shared": (c.attend_shared, ("q", "query_start", "source", "plan", "seq_len", "block_table", "out", "lse"), {})}
    row_kinds = {"float32": lambda t: t.float(), "cpu": lambda t: t.cpu(), "64 values": lambda t: t[..., :64], "two dimensions": lambda t: t.flatten(1), "a number": lambda t: 7,
                 "heads apart": lambda t: t.transpose(0, 1).contiguous().transpose(0, 1), "the same row again": lambda t: t[:1].expand(t.shape)}
    int_kinds = {"int64": lambda t: t.long(), "cpu": lambda t: t.cpu(), "longer": lambda t: torch.cat([t, t]), "apart": lambda t: t.repeat_interleave(2, -1)[..., ::2],
                 "none": lambda t: None}
    out_kinds = {"float16": lambda t: t.half(), "cpu": lambda t: t.cpu(), "longer": lambda t: torch.cat([t, t]), "apart": lambda t: t.repeat_interleave(2, -1)[..., ::2]}
    rope_kinds = {"float64": lambda t: t.double(), "cpu": lambda t: t.cpu(), "apart": lambda t: t.repeat_interleave(2, -1)[..., ::2], "one dimension": lambda t: t.flatten(),
                  "130 wide": lambda t: torch.zeros((70, 130), device="cuda")}

    def refused(call, status, **k):
        try:
            call(**k)
        except IceError as e:
            assert e.status == status, (k.keys(), e)
            return
        raise AssertionError("taken")
    for name, (call, names, more) in calls.items():
        for n in names:
            kinds = row_kinds if n in ("q", "k", "v") else out_kinds if n in ("out", "lse") else rope_kinds if n == "rope" else int_kinds
            for kind, change in kinds.items():
                if (n, kind) == ("source", "none") and name == "append":
                    continue
                refused(call, b.ICE_ERR_SHAPE, **{**{x: g[x] for x in names}, **more, n: change(g[n])})
    good = {x: g[x] for x in calls["append"][1]}
    for change, status in ((dict(rope=None), b.ICE_ERR_INVALID_ARG), (dict(q=None), b.ICE_ERR_SHAPE), (dict(rope=up(angles(70, 64))[:0]), b.ICE_ERR_SHAPE),
                           (dict(rope=torch.zeros((70, 24), device="cuda")), b.ICE_ERR_UNSUPPORTED), (dict(q=g["q"][:2]), b.ICE_ERR_SHAPE), (dict(k=g["k"][:, :1], v=g["v"][:, :1]), b.ICE_ERR_SHAPE),
                           (dict(out=turned[:2]), b.ICE_ERR_SHAPE), (dict(out=turned.float()), b.ICE_ERR_SHAPE)):
        refused(c.append, status, **{**good, "out": turned, **change})
    for name in ("attend_cross", "attend_shared"):
        call, names, _ = calls[name]
        good = {x: g[x] for x in names}
        for change in (dict(max_shared=0), dict(max_len=0), dict(max_len=2 ** 30 + 1), dict(out_dtype=torch.float16), dict(plan=g["plan"][:-2].contiguous())):
            refused(call, b.ICE_ERR_SHAPE, **{**good, **change})
        refused(call, b.ICE_ERR_UNSUPPORTED, **{**good, "q": g["q"].repeat(1, 5, 1)[:, :34].contiguous(), "out": None, "lse": None})
    good = {x: g[x] for x in calls["attend_shared"][1]}
    for change in (dict(max_query=0), dict(max_source=0), dict(window=-1)):
        refused(c.attend_shared, b.ICE_ERR_SHAPE, **{**good, **change})
    blocks = IceBlocks(16, 16, 3, 64)
    for bad in (dict(source=i32([0, 1])), dict(source=i32([0, 1, 2]).cpu()), dict(source=i32([0, 1, 2]).long()), dict(n_tokens=-1), dict(plan=i32([0] * 9))):
        refused(blocks.plan_sources, b.ICE_ERR_SHAPE, **{**dict(source=i32([0, 1, 2]), n_tokens=3, plan=i32([0] * 14)), **bad})
    assert bool((g["out"] == 7).all()) and bool((g["lse"] == 7).all()) and bool((turned == 7).all()) and np.array_equal(down(c.data), data)
    c.attend_shared(**good)
    check(g["out"], g["lse"], sh.attention(ref.widen(down(g["q"])).astype(np.float64), data, table, lens, qlens, [-1, 0, 0], block, group, 0, False, True))
