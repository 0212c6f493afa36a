"""How the 4-bit cache's attention cuts its work, on the host with the kernels' own arithmetic: every query row's keys are taken once, by workgroups
that follow each other, and every place that the kernels write or the merge reads is one that somebody has written and the workspace holds."""
import numpy as np
import pytest

CHUNK, RECORD, FEW = 192, 528, 48  # rows of a unit of the kernel for many queries, bytes of a record's row, the most rows of the other kernel


def cut(heads, group, lens, qlens, window=0, max_query=None, max_keys=None, block=16, width=None):
    """The parts of a call, as a dict of arrays, and its workspace's bytes."""
    import paper_2604_10539_amd as p
    from paper_2604_10539_amd import binding as b
    c = p.make_cache_desc(None, 1, heads, block)
    start = np.concatenate([[0], np.cumsum(qlens)])
    most = max(max(qlens), 1) if max_query is None else max_query
    width = width or max(1, -(-max(lens) // block))
    keys = max(1, max(lens)) if max_keys is None else max_keys
    parts = b.ice_debug_cache_cut(c, group, len(lens), start, int(start[-1]), most, lens, keys, width, window)
    return dict(zip(b.CUT_FIELDS, parts.T)), p.ice_cache_attend_bytes(c, group, len(lens), most, keys), width * block


def check_units(x, nbytes, heads, expected, room):
    """x: parts; expected: {(kernel, request, base): (rows, low, high)}, the same for every KV head; room: rows of a record, by kernel."""
    order = np.lexsort((x["now"], x["base"], x["head"], x["request"], x["many"]))
    x = {k: v[order].astype(np.int64) for k, v in x.items()}
    n = len(order)
    if n == 0:
        assert not expected
        return
    same = np.zeros(n, dtype=bool)  # the same unit as the part before
    same[1:] = np.all([x[k][1:] == x[k][:-1] for k in ("many", "request", "head", "base")], 0)
    firsts, lasts = np.flatnonzero(~same), np.flatnonzero(~np.append(same[1:], False))
    got = {}
    for i in firsts:
        got.setdefault((x["many"][i], x["request"][i], x["base"][i]), []).append(x["head"][i])
    assert set(got) == set(expected) and all(h == list(range(heads)) for h in got.values()), "units missing, or others than there are"
    want = np.array([expected[x["many"][i], x["request"][i], x["base"][i]] for i in range(n)]).reshape(n, 3)
    assert np.array_equal(x["rows"], want[:, 0])
    # in the flat work: from the unit's start to its end without a gap, by workgroups that follow each other
    assert np.array_equal(x["now"][firsts], x["u0"][firsts]) and np.array_equal(x["stop"][lasts], x["u1"][lasts])
    for k in ("u0", "u1"):
        assert np.array_equal(x[k][same], x[k][np.flatnonzero(same) - 1])
    rest = np.flatnonzero(same)
    assert np.array_equal(x["now"][rest], x["stop"][rest - 1]) and np.all(x["stop"] > x["now"])
    assert np.array_equal(x["workgroup"][rest], x["workgroup"][rest - 1] + 1)
    # keys: the parts that have any cover what the rows see, once
    some = np.flatnonzero(x["to"] > x["from"])
    assert np.all((x["from"][some] >= want[some, 1]) & (x["to"][some] <= want[some, 2]))
    unit = np.cumsum(~same) - 1
    taken = np.zeros(len(firsts), dtype=np.int64)
    np.add.at(taken, unit[some], x["to"][some] - x["from"][some])
    assert np.array_equal(taken, np.maximum(want[firsts, 2] - want[firsts, 1], 0))
    follow = some[1:][unit[some[1:]] == unit[some[:-1]]]
    before = some[:-1][unit[some[1:]] == unit[some[:-1]]]
    assert np.all(x["from"][follow] >= x["to"][before])
    # records: of every part of a unit that was cut and of no other, the first part's by itself; one note, by the workgroup with the end
    is_cut = (x["now"] > x["u0"]) | (x["stop"] < x["u1"])
    assert np.array_equal(x["record"], np.where(is_cut, 2 * x["workgroup"] + (x["now"] == x["u0"]), -1))
    ends = is_cut & (x["stop"] == x["u1"])
    assert np.array_equal(x["note"], np.where(ends, x["workgroup"][firsts][unit], -1))
    for kernel in (0, 1):
        for launch in np.unique(x["first"]):
            here = (x["many"] == kernel) & (x["first"] == launch)
            r = x["record"][here & is_cut]
            assert len(np.unique(r)) == len(r)
            notes = x["workgroup"][here & ends]
            assert len(np.unique(notes)) == len(notes)
            if len(r):
                assert (x["workgroup"][here].max() + 1) * (2 * room[kernel] * RECORD + 32) <= nbytes


def check(heads, group, lens, qlens, window=0, max_query=None, max_keys=None, block=16, width=None):
    x, nbytes, capacity = cut(heads, group, lens, qlens, window, max_query, max_keys, block, width)
    most = max(max(qlens), 1) if max_query is None else max_query
    rows_most = most * group
    room = next(r for r in (5, 8, 16, 32, FEW, 1 << 30) if rows_most <= r)
    few = 16 if rows_most > FEW else room
    expected = {}
    for s, (length, n) in enumerate(zip(lens, qlens)):
        rows = min(n, most) * group
        many = rows_most > FEW and rows > 16
        for base in range(0, rows, CHUNK if many else 1 << 30):
            here = min(rows - base, CHUNK) if many else rows
            seen = [length - n + t + 1 for t in (base // group, (base + here - 1) // group)]  # keys up to the query's own position
            low = max(seen[0] - window, 0) if window else 0
            expected[int(many), s, base] = (here, min(low, capacity), min(max(seen[1], 0), capacity))
    check_units(x, nbytes, heads, expected, (few, min(CHUNK, rows_most)))


def test_row_tiles_that_see_nothing_in_front_of_a_window():
    """More queries than tokens: the first row tiles see nothing, and the last but one sees more than the last."""
    check(1, 1, [705], [1345], window=258)
    check(2, 1, [769], [1921], window=256)


@pytest.mark.parametrize("seed", range(12))
def test_chunks_of_any_shape(seed):
    rng = np.random.default_rng(seed)
    for _ in range(60):
        S, group = int(rng.integers(1, 5)), int(rng.choice([1, 2, 3, 4, 7, 8, 16]))
        qlens = [int(np.exp(rng.uniform(0, np.log(2500)))) if rng.random() < 0.8 else 0 for _ in range(S)]
        lens = [int(np.exp(rng.uniform(0, np.log(4000)))) if rng.random() < 0.6 else int(n + rng.integers(-1000, 3000)) for n in qlens]
        lens = [max(n, 0) for n in lens]
        window = int(rng.choice([0, 1, 64, 127, 128, 129, int(rng.integers(1, 1500))]))
        most = None if rng.random() < 0.7 else int(rng.integers(1, max(qlens) + 2))
        keys = None if rng.random() < 0.5 else int(rng.integers(1, 5000))
        check(int(rng.integers(1, 4)), group, lens, qlens, window, most, keys)


@pytest.mark.parametrize("seed", range(6))
def test_few_queries_of_any_shape(seed):
    rng = np.random.default_rng([seed, 1])
    for _ in range(40):
        S, group = int(rng.choice([1, 2, 16, 40, 130])), int(rng.choice([1, 2, 4, 5, 8, 16]))
        most = int(rng.integers(1, FEW // group + 1))
        qlens = [int(rng.integers(0, most + 1)) for _ in range(S)]
        lens = [int(np.exp(rng.uniform(0, np.log(200000 // S + 2)))) - 1 for _ in range(S)]
        check(int(rng.choice([1, 2, 8])), group, lens, qlens, int(rng.choice([0, 0, 1, 100, 4096])), most, None if rng.random() < 0.7 else int(rng.integers(1, 9000)))


@pytest.mark.parametrize("group,queries,lens", [(2, 1, [150000, 140000, 160000, 147000]), (8, 5, [90000, 120000, 105000, 98000]), (16, 60, [41000, 40500, 41500, 43000]),
                                                (4, 2048, [32768, 31000])])
def test_pieces_of_two_or_three_lengths(group, queries, lens):
    check(2, group, lens, [queries] * len(lens), block=64)


def test_the_measured_cases():
    from perf import operators
    for case in operators.listed():
        if case["kind"] == "attend":
            cached, gain = operators._lengths(case)
            check(case["heads"], case["group"], [c + g for c, g in zip(cached, gain)], gain, case["window"], block=case["block"])


@pytest.mark.parametrize("queries", [1, 60])
def test_more_requests_than_one_launch_takes(queries):
    rng = np.random.default_rng(queries)
    lens = [int(x) for x in rng.integers(0, 3000, 2500)]
    check(2, 4, lens, [1] * 2400 + [queries] * 100)


@pytest.mark.parametrize("group,queries", [(2, 2), (2, 40), (4, 700)])
def test_lengths_beyond_the_table_keep_the_queries_positions(group, queries):
    """seq_len says where the queries stand, the table's row how many tokens there are: queries behind the row see all of it, or with a window
    what it leaves them."""
    for length in (150, 159, 160, 161, 161 + queries, 400, 2 ** 31 - 1):
        for window in (0, 1, 50, 300, 2 ** 31 - 1):
            check(2, group, [length, 90], [queries, 1], window, max_keys=300, width=10)


def test_records_have_room_for_the_rows_that_there_can_be_and_no_more():
    """A call of many queries keeps 512 workgroups' records; a unit of it has 192 rows, or all that a request may have."""
    import paper_2604_10539_amd as p
    c = p.make_cache_desc(None, 1, 8, 16)
    for rows in (49, 64, 191, 192, 193, 5000):
        assert p.ice_cache_attend_bytes(c, 1, 16, rows, 32768) == 512 * (2 * min(rows, CHUNK) * RECORD + 32)


@pytest.mark.parametrize("requests,heads,most", [(1, 1, 1), (1, 8, 256), (1, 8, 2500), (3, 2, 5000), (16, 8, 1024), (40, 1, 700), (256, 2, 3500), (384, 2, 4100), (1100, 1, 2100)])
def test_lists(requests, heads, most):
    import paper_2604_10539_amd as p
    from paper_2604_10539_amd import binding as b
    rng = np.random.default_rng(most)
    c = p.make_cache_desc(None, 1, heads, 16)
    n_tok = rng.integers(-1, most + 9, (requests, heads))
    parts = b.ice_debug_cache_cut(c, 4, requests, None, 0, 1, n_tok, most, 100)
    x = dict(zip(b.CUT_FIELDS, parts.T))
    nbytes = p.ice_cache_attend_tokens_bytes(c, 4, requests, most)
    for h in range(heads):  # (a head's lists are its own: one head at a time)
        here = {k: v[x["head"] == h] for k, v in x.items()}
        here["head"] = np.zeros_like(here["head"])
        check_units(here, nbytes, 1, {(0, s, 0): (4, 0, min(max(int(n_tok[s, h]), 0), most)) for s in range(requests)}, (5, CHUNK))
    if nbytes:
        r = x["record"][x["record"] >= 0]
        assert len(np.unique(np.stack([x["first"][x["record"] >= 0], r]), axis=1).T) == len(r)


def test_the_hook_refuses():
    import paper_2604_10539_amd as p
    from paper_2604_10539_amd import binding as b
    c = p.make_cache_desc(None, 1, 2, 16)
    good = dict(group_size=4, n_requests=1, query_start=[0, 1], n_tokens=1, max_query=1, length=[5], max_keys=5, max_blocks=1)
    for change, status in ((dict(group_size=17), b.ICE_ERR_UNSUPPORTED), (dict(n_requests=0), b.ICE_ERR_SHAPE), (dict(max_blocks=0), b.ICE_ERR_SHAPE),
                           (dict(n_requests=1024, query_start=[0] * 1025, length=[0] * 1024, max_query=2 ** 24, max_blocks=2 ** 20), b.ICE_ERR_UNSUPPORTED),
                           (dict(window=-1), b.ICE_ERR_SHAPE), (dict(max_query=0), b.ICE_ERR_SHAPE), (dict(max_blocks=2 ** 27), b.ICE_ERR_SHAPE)):
        with pytest.raises(p.IceError) as e:
            b.ice_debug_cache_cut(c, **{**good, **change})
        assert e.value.status == status
    assert b.lib().ice_debug_cache_cut(None, 1, 1, None, 1, 1, None, 1, 1, 0, None, 0, None) == b.ICE_ERR_INVALID_ARG
