"""Sources of the 4-bit cache without a GPU: how attention to them cuts its work, and what the calls refuse."""
import numpy as np
import pytest
import torch

from tests.test_cache4_cpu import FAKE, status
from tests import shared_ref as sh
from tests.test_cache4_cut_cpu import CHUNK, FEW, check_units


def tiles(queries, group):
    """First rows of the tiles of the kernel for many queries: whole tokens, as evenly as they go, at most 192 rows."""
    n = -(-queries // (CHUNK // group))
    step = -(-queries // n)
    return [(at * group, min(step, queries - at) * group) for at in range(0, queries, step)]


def check(heads, group, lens, counts, max_shared=None, max_keys=None, block=16, width=None):
    """counts: queries (tokens) of each source."""
    import paper_2604_10539_amd as p
    from paper_2604_10539_amd import binding as b
    c = p.make_cache_desc(None, 1, heads, block)
    start = np.concatenate([[0], np.cumsum(counts), [sum(counts) + 3]])
    most = max(max(counts), 1) if max_shared is None else max_shared
    width = width or max(1, -(-max(lens) // block))
    keys = max(1, max(lens)) if max_keys is None else max_keys
    parts = b.ice_debug_cross_cut(c, group, len(lens), start, int(start[-1]), most, lens, keys, width)
    nbytes = p.ice_cache_attend_cross_bytes(c, group, len(lens), most, keys)
    many = most * group > FEW
    expected = {}
    for s, (length, n) in enumerate(zip(lens, counts)):
        n = min(n, most)
        for base, rows in tiles(n, group) if many and n else [(0, n * group)] if n else []:
            expected[int(many), s, base] = (rows, 0, min(length, width * block))
    check_units(dict(zip(b.CUT_FIELDS, parts.T)), nbytes, heads, expected, (next(r for r in (5, 8, 16, 32, FEW, 1 << 30) if most * group <= r), min(CHUNK, most * group)))


def check_shared(heads, group, lens, qlens, source, window=0, max_query=None, max_shared=None, max_keys=None, max_source=None, block=16, width=None):
    import paper_2604_10539_amd as p
    from paper_2604_10539_amd import binding as b
    c = p.make_cache_desc(None, 1, heads, block)
    n, start = len(lens), np.concatenate([[0], np.cumsum(qlens)])
    tokens = int(start[-1]) + 2
    plan = sh.sources(source, start, lens, n, tokens)
    counts, lowest = np.diff(plan[: n + 1]), plan[n + 2: 2 * n + 2]
    most = [max(max(x), 1) if m is None else m for x, m in ((qlens, max_query), (counts, max_shared))]
    width = width or max(1, -(-max(lens) // block))
    keys = [max(1, max(lens)) if k is None else k for k in (max_keys, max_source)]
    parts = b.ice_debug_shared_cut(c, group, n, start, plan, tokens, *most, lens, *keys, width, window)
    nbytes = p.ice_cache_attend_shared_bytes(c, group, n, tokens, *most, *keys) - tokens * heads * (32 + 1056 * group)
    quanta, capacity = heads * (n * -(-keys[0] // 128) + -(-keys[1] // 128)), width * block
    many = max(most) * group > (16 if quanta > 512 else FEW)
    expected = {}
    for e in range(2 * n):
        s = e % n
        m = min(counts[s], most[1]) if e < n else min(qlens[s], most[0])
        for base, rows in tiles(m, group) if many and m else [(0, m * group)] if m else []:
            if e < n:  # every tile of a source takes what the lowest query's window leaves
                low = max(lens[s] + int(lowest[s]) + 1, 0) - window if window else 0
                seen = (min(max(low, 0), capacity, lens[s]), min(lens[s], capacity))
            else:
                ends = [lens[s] - qlens[s] + t + 1 for t in (base // group, (base + rows - 1) // group)]
                low = max(max(ends[0], 0) - window, 0) if window else 0
                seen = (min(low, capacity, lens[s]), min(max(ends[1], 0), capacity))
            expected[int(many), e, base] = (rows, *seen)
    room = next(r for r in (5, 8, 16, 32, FEW, 1 << 30) if max(most) * group <= r)
    x = dict(zip(b.CUT_FIELDS, parts.T))
    nbytes += 32 * (int(x["workgroup"].max(initial=-1)) + 1)  # (there are no notes by workgroup here)
    check_units(x, nbytes, heads, expected, (room, min(CHUNK // group, max(most)) * group))


@pytest.mark.parametrize("seed", range(16))
def test_requests_behind_sources_of_any_shape(seed):
    rng = np.random.default_rng([seed, 6])
    for _ in range(40):
        n, group = int(rng.choice([1, 2, 5, 40, 130])), int(rng.choice([1, 2, 3, 4, 5, 7, 8, 11, 16]))
        top = 1500 if rng.random() < 0.5 else max(1, FEW // group)
        qlens = [int(np.exp(rng.uniform(0, np.log(top)))) if rng.random() < 0.6 else 0 for _ in range(n)]
        lens = [int(np.exp(rng.uniform(0, np.log(40000 // n + 2)))) - 1 if rng.random() < 0.5 else max(0, int(m + rng.integers(-500, 900))) for m in qlens]
        source = rng.choice([-1, int(rng.integers(0, n)), int(rng.integers(0, n))], n)
        window = int(rng.choice([0, 0, 1, 127, 128, int(rng.integers(1, 1500))]))
        some = lambda most: None if rng.random() < 0.7 else int(rng.integers(1, most))  # noqa: E731
        check_shared(int(rng.choice([1, 2, 8])), group, lens, qlens, source, window, some(max(qlens) + 2), some(sum(qlens) + 2), some(9000), some(9000),
                     width=None if rng.random() < 0.8 else max(1, max(lens) // 40))


def test_more_rows_than_the_table_of_sums_has_places():
    for n, queries in ((513, 1), (1500, 1), (3000, 60), (8192, 1)):
        check_shared(1, 2, [9] * 7 + [500] + [20] * (n - 8), [queries if i % 3 else 0 for i in range(n)], np.where(np.arange(n) % 5 == 4, -1, 7))


@pytest.mark.parametrize("seed", range(12))
def test_sources_of_any_shape(seed):
    rng = np.random.default_rng([seed, 5])
    for _ in range(50):
        rows, group = int(rng.choice([1, 2, 7, 40, 130])), int(rng.choice([1, 2, 3, 4, 7, 8, 16]))
        top = 2500 if rng.random() < 0.5 else max(1, FEW // group)
        counts = [int(np.exp(rng.uniform(0, np.log(top)))) if rng.random() < 0.6 else 0 for _ in range(rows)]
        lens = [int(np.exp(rng.uniform(0, np.log(100000 // rows + 2)))) - 1 for _ in range(rows)]
        most = None if rng.random() < 0.7 else int(rng.integers(1, max(counts) + 2))
        width = None if rng.random() < 0.8 else max(1, max(lens) // 40)
        check(int(rng.choice([1, 2, 8])), group, lens, counts, most, None if rng.random() < 0.5 else int(rng.integers(1, 9000)), width=width)


def test_one_source_among_many_rows_and_more_rows_than_a_launch_takes():
    check(8, 4, [32768] + [900] * 32, [32] + [0] * 32, block=64)
    check(2, 4, [300] * 1030, [3] * 1030)
    check(1, 2, [300] * 2100, [0, 40, 0] * 700)


def test_the_measured_cases():
    from perf import more_operators
    for case in more_operators.listed():
        if case["kind"] not in ("cross", "shared"):
            continue
        source, _, gain, lengths = more_operators._batch(case)
        counts = [0] * len(lengths)
        for s, g in zip(source, gain):
            if s >= 0:
                counts[s] += g
        if case["kind"] == "cross":
            check(case["heads"], case["group"], lengths, counts, block=case["block"])
        else:
            check_shared(case["heads"], case["group"], lengths, gain, source, case["window"], block=case["block"])


def test_the_hook_refuses():
    import paper_2604_10539_amd as p
    from paper_2604_10539_amd import binding as b
    c, e = p.make_cache_desc(None, 1, 2, 16), np.zeros(4, np.int32)
    for change in (dict(n_rows=0), dict(n_rows=8193), dict(n_tokens=-1), dict(max_shared=0), dict(max_keys=0), dict(max_blocks=0), dict(max_blocks=2 ** 27)):
        args = dict(cache=c, group_size=4, n_rows=1, start=e, n_tokens=1, max_shared=1, length=e, max_keys=16, max_blocks=1)
        assert status(b.ice_debug_cross_cut, **{**args, **change}) == b.ICE_ERR_SHAPE, change
    e = np.zeros(8, np.int32)
    for change in (dict(n_requests=0), dict(n_requests=8193), dict(n_tokens=-1), dict(max_query=0), dict(max_shared=0), dict(max_keys=0), dict(max_source_keys=0),
                   dict(max_blocks=0), dict(window=-1)):
        args = dict(cache=c, group_size=4, n_requests=1, query_start=e, plan=e, n_tokens=1, max_query=1, max_shared=1, length=e, max_keys=16, max_source_keys=16,
                    max_blocks=1)
        assert status(b.ice_debug_shared_cut, **{**args, **change}) == b.ICE_ERR_SHAPE, change


# ------------------------------------------------------------------------------------------------------------- what is refused
def test_sorting_refuses():
    from paper_2604_10539_amd import binding as b
    good = dict(n=4, rows=4, tokens=10, source=FAKE, start=FAKE, seq_len=FAKE, plan=FAKE)

    def call(**change):
        return b.lib().ice_plan_sources(*{**good, **change}.values(), None)
    for name in ("source", "start", "plan"):
        assert call(**{name: None}) == b.ICE_ERR_INVALID_ARG
    for change in (dict(n=0), dict(n=8193), dict(rows=0), dict(rows=8193), dict(tokens=-1), dict(tokens=2 ** 30 + 1)):
        assert call(**change) == b.ICE_ERR_SHAPE, change


def test_appending_refuses():
    import paper_2604_10539_amd as p
    from paper_2604_10539_amd import binding as b
    c = p.make_cache_desc(FAKE, 10, 2, 16)
    good = dict(q=FAKE, qs=1024, qh=8, out=FAKE, os=1024, k=FAKE, v=FAKE, ks=256, vs=256, tokens=4, n=2, start=FAKE, sl=FAKE, source=FAKE, table=FAKE, mb=4,
                rope=FAKE, positions=100, rotated=128, neighbours=0)
    go = lambda **change: status(p.ice_cache_append, c, *{**good, **change}.values())  # noqa: E731
    for name in ("out", "k", "v", "start", "sl", "table", "rope"):
        assert go(**{name: None}) == b.ICE_ERR_INVALID_ARG, name
    for name in ("q", "out", "k", "v", "rope"):
        assert go(**{name: FAKE + 8}) == b.ICE_ERR_INVALID_ARG, name
    for change in (dict(qs=1028), dict(qs=1016), dict(os=1028), dict(os=1016), dict(ks=252), dict(ks=248), dict(vs=260), dict(vs=0), dict(tokens=-1), dict(n=0),
                   dict(n=65536), dict(mb=0), dict(mb=2 ** 27), dict(positions=0), dict(qh=0)):
        assert go(**change) == b.ICE_ERR_SHAPE, change
    for rotated in (0, 8, 24, 144, -16):
        assert go(rotated=rotated) == b.ICE_ERR_UNSUPPORTED
    assert go(neighbours=2) == b.ICE_ERR_INVALID_ARG
    assert go(tokens=2 ** 30) == b.ICE_ERR_UNSUPPORTED
    p.ice_cache_append(c, *{**good, "tokens": 0, "k": None, "v": None, "out": None}.values())  # nothing to do
    assert b.lib().ice_cache_append(None, *good.values(), None) == b.ICE_ERR_INVALID_ARG


def test_an_empty_table_of_rotations_is_not_none():
    """(A fresh tensor of no values has no address, which would read as no rotations.)"""
    import paper_2604_10539_amd as p
    from paper_2604_10539_amd import binding as b
    c = p.make_cache_desc(FAKE, 10, 2, 16)
    for q, out in ((FAKE, FAKE), (None, None)):
        for shape in ((0, 128), (0, 0), (5, 0)):
            assert status(p.ice_cache_append, c, q, 1024, 8, out, 1024, FAKE, FAKE, 256, 256, 4, 2, FAKE, FAKE, FAKE, FAKE, 4, torch.empty(shape), *shape, 0) == b.ICE_ERR_SHAPE


def test_attention_to_sources_refuses():
    import paper_2604_10539_amd as p
    from paper_2604_10539_amd import binding as b
    c = p.make_cache_desc(FAKE, 1000, 2, 16)
    cross = dict(q=FAKE, qs=1024, G=4, rows=2, plan=FAKE, tokens=2, shared=1, sl=FAKE, keys=4096, table=FAKE, mb=256, out=FAKE, ot=0, lse=None, ws=FAKE, wb=1 << 30)
    both = dict(q=FAKE, qs=1024, G=4, n=2, start=FAKE, source=FAKE, plan=FAKE, tokens=2, query=1, shared=2, sl=FAKE, keys=64, source_keys=4096, table=FAKE, mb=256,
                window=0, out=FAKE, ot=0, lse=None, ws=FAKE, wb=1 << 30)
    need = {p.ice_cache_attend_cross: p.ice_cache_attend_cross_bytes(c, 4, 2, 1, 4096),
            p.ice_cache_attend_shared: p.ice_cache_attend_shared_bytes(c, 4, 2, 2, 1, 2, 64, 4096)}
    assert need[p.ice_cache_attend_shared] > 2 * 8 * 1056  # (every row's sums over both sides' tokens, and scratch)
    for call, good, count in ((p.ice_cache_attend_cross, cross, "rows"), (p.ice_cache_attend_shared, both, "n")):
        go = lambda **change: status(call, c, *{**good, **change}.values())  # noqa: E731, B023
        for name in [x for x in ("q", "start", "source", "plan", "sl", "table", "out", "ws") if x in good]:
            assert go(**{name: None}) == b.ICE_ERR_INVALID_ARG, name
        for change in (dict(q=FAKE + 8), dict(out=FAKE + 8), dict(ws=FAKE + 8), dict(ot=2)):
            assert go(**change) == b.ICE_ERR_INVALID_ARG
        for name, values in ((count, (0, 8193)), ("tokens", (-1,)), ("shared", (0, 2 ** 24 + 1)), ("keys", (0, 2 ** 30 + 1)), ("mb", (0, 2 ** 27)), ("qs", (1020, 1016)),
                             ("query", (0, 2 ** 24 + 1)), ("source_keys", (0,)), ("window", (-1,))):
            for v in values if name in good else ():
                assert go(**{name: v}) == b.ICE_ERR_SHAPE, (name, v)
        for G in (0, -1, 17):
            assert go(G=G) == b.ICE_ERR_UNSUPPORTED
        assert go(wb=need[call] - 1) == b.ICE_ERR_CAPACITY and "workspace" in p.ice_last_error()
        assert go(**{count: 8192, "shared": 2 ** 24}) == b.ICE_ERR_UNSUPPORTED
        call(c, *{**good, "tokens": 0}.values())
    assert status(p.ice_cache_attend_shared, c, *{**both, "tokens": 5 * 10 ** 6 + 1}.values()) == b.ICE_ERR_UNSUPPORTED
    for args in ((c, 17, 2, 1, 4096), (c, 4, 0, 1, 4096), (c, 4, 8193, 1, 4096), (c, 4, 2, 0, 4096)):
        assert p.ice_cache_attend_cross_bytes(*args) == 0
    assert p.ice_cache_attend_shared_bytes(c, 4, 2, -1, 1, 2, 64, 4096) == 0 and p.ice_cache_attend_shared_bytes(c, 4, 8193, 2, 1, 2, 64, 4096) == 0


def test_sorting_takes_arrays_on_a_gpu_only():
    import paper_2604_10539_amd as p
    from paper_2604_10539_amd import binding as b
    e = lambda n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    args = [e(2), e(3), e(2), e(2 * 2 + 2 + 2 * 5), 2, 5]
    assert status(p.ice_plan_sources, *args) == b.ICE_ERR_INVALID_ARG
    for i, bad in ((0, e(3)), (1, e(2)), (2, e(1)), (3, e(15)), (0, torch.zeros(2)), (1, None), (3, torch.zeros(32, dtype=torch.int32)[::2])):
        assert status(p.ice_plan_sources, *[bad if j == i else x for j, x in enumerate(args)]) == b.ICE_ERR_SHAPE, i


@pytest.mark.parametrize("current", [0, 1])
def test_sorting_goes_to_the_device_of_its_arrays(monkeypatch, current):
    """Rows of another table are sorted by ice_plan_sources itself: on the arrays' device and its current stream, whatever the current device is."""
    from paper_2604_10539_amd import binding as b
    state, calls = {"device": current}, []

    class Under:
        def __init__(self, device):
            self.device = getattr(device, "index", device)

        def __enter__(self):
            self.before, state["device"] = state["device"], self.device

        def __exit__(self, *_):
            state["device"] = self.before

    class OnSecond(torch.Tensor):
        is_cuda = True

        def get_device(self):
            return 1

    class Native:
        def plan_sources(self, stream, *args):
            calls.append((state["device"], stream, args))
    monkeypatch.setattr(torch.cuda, "device", Under)
    monkeypatch.setattr(b, "_current_device", lambda: state["device"])
    monkeypatch.setattr(b, "_extension", lambda: Native())
    monkeypatch.setattr(b, "_stream", lambda stream: 100 + state["device"] if stream is None else stream)
    arrays = [torch.zeros(n, dtype=torch.int32).as_subclass(OnSecond) for n in (2, 3, 2, 16)]
    b.ice_plan_sources(*arrays, 2, 5)
    b.ice_plan_sources(*arrays, 2, 5, stream=7)
    assert [x[:2] for x in calls] == [(1, 101), (1, 7)] and all(x[2][0] is arrays[0] and x[2][4:] == (2, 5) for x in calls) and state["device"] == current
