"""The cut of attention behind a source on the host is the kernels' own: how many quanta every unit has, with the hints that calls give."""
import numpy as np
import pytest

from tests import shared_ref as sh
from tests.test_cache4_cut_cpu import CHUNK, FEW
from tests.test_shared_cpu import tiles


def cut_of(heads, group, lens, qlens, source, window=0, hints=(None,) * 4, block=16):
    """The parts of attention behind a source, as a dict of arrays, and the plan; hints: max_query, max_shared, max_keys, max_source."""
    import paper_2604_10539_amd as p
    from paper_2604_10539_amd import binding as b
    c = p.make_cache_desc(None, 1, heads, block)
    n, start = len(lens), np.concatenate([[0], np.cumsum(qlens)])
    tokens = int(start[-1])
    plan = sh.sources(source, start, lens, n, tokens)
    counts = np.diff(plan[: n + 1])
    full = max(max(qlens), 1), max(int(counts.max()), 1), max(1, max(lens)), max(1, max(lens))
    query, shared, keys, source_keys = (f if h is None else h for f, h in zip(full, hints))
    parts = b.ice_debug_shared_cut(c, group, n, start, plan, tokens, query, shared, lens, keys, source_keys, max(1, -(-max(lens) // block)), window)
    return dict(zip(b.CUT_FIELDS, parts.T.astype(np.int64))), plan


def check_quanta(heads, group, lens, qlens, source, window=0, hints=(None,) * 4, block=16):
    """Every unit is as long in the flat work as the kernel counts it from its lengths: quanta that its keys lie in, one at least, and in the
    kernel for many queries what a unit costs beside them.  (Own tokens of several row tiles lie there in pairs: left out.)"""
    x, plan = cut_of(heads, group, lens, qlens, source, window, hints, block)
    n = len(lens)
    counts, lowest = np.diff(plan[: n + 1]), plan[n + 2: 2 * n + 2]
    seen = 0
    for many, e, base, u0, u1 in sorted(set(zip(*(x[k].tolist() for k in ("many", "request", "base", "u0", "u1"))))):
        s, gathered = e % n, e < n
        queries = int(counts[s] if gathered else qlens[s])
        assert queries, "a unit without queries"
        low, high = 0, lens[s]
        if not gathered:
            low, high = lens[s] - queries + 1, lens[s]
        elif window:
            low = lens[s] + int(lowest[s]) + 1
        low = min(max(max(low, 0) - window, 0), lens[s]) if window else 0
        quantum, beside = 128, 0
        if many:
            parts = tiles(queries, group)
            if len(parts) > 1 and not gathered:
                continue
            quantum = 512 if queries * group <= 16 else 256 if parts[0][1] <= 64 else 128
            beside = 1 if queries * group <= 16 else 2
        assert u1 - u0 == max(-(-high // quantum) - low // quantum, 1) + beside, (many, e, base)
        seen += 1
    assert seen >= heads
    return x


def test_a_few_samples_of_one_prompt_are_cut_by_their_lengths():
    """(Short texts of the requests' own do not make the source's unit whole.)"""
    x = check_quanta(2, 4, [2048, 130, 60, 7, 129], [0, 1, 1, 1, 1], [-1, 0, 0, 0, 0], hints=(1, 4, 130, 2048))
    source = x["request"] == 0
    assert np.all(x["u1"][source] - x["u0"][source] == 16) and len(x["now"]) == 2 * (16 + 2 + 1 + 1 + 2)
    y = check_quanta(2, 4, [2048, 130, 60, 7, 129], [0, 1, 1, 1, 1], [-1, 0, 0, 0, 0], hints=(1, 4, 2048, 2048))
    assert np.array_equal(x["u1"] - x["u0"], y["u1"] - y["u0"])


def test_the_measured_cases_with_the_hints_that_their_calls_give():
    from perf import more_operators
    for case in more_operators.listed():
        if case["kind"] != "shared":
            continue
        source, _, gain, lengths = more_operators._batch(case)
        rows = [s for s, g in zip(source, gain) for _ in range(g)]
        hints = (max(gain), max([rows.count(s) for s in set(rows) if s >= 0] or [1]), max(x for x, g in zip(lengths, gain) if g),
                 max([lengths[s] for s in set(rows) if s >= 0] or [1]))
        check_quanta(case["heads"], case["group"], lengths, gain, source, case["window"], hints, case["block"])


@pytest.mark.parametrize("seed", range(8))
def test_requests_of_any_length_behind_sources(seed):
    rng = np.random.default_rng([seed, 12])
    for _ in range(30):
        n, group = int(rng.choice([2, 5, 40, 130, 600])), int(rng.choice([1, 2, 4, 7, 16]))
        top = 500 if rng.random() < 0.3 else max(1, min(FEW, CHUNK) // group // 4)
        qlens = [int(np.exp(rng.uniform(0, np.log(top)))) if rng.random() < 0.6 else 0 for _ in range(n)]
        qlens[-1] = 1
        lens = [m + int(rng.integers(0, 500)) for m in qlens]
        lens[0] += 3000
        source = rng.choice([-1, 0, 0, int(rng.integers(0, n))], n)
        check_quanta(int(rng.choice([1, 2, 8])), group, lens, qlens, source, int(rng.choice([0, 0, 100, 700])),
                     (None, None, max(lens[1:]), None if rng.random() < 0.5 else lens[0]))
