"""How much work a call of attention to sources may have: queries of all requests are n_tokens at most, however they lie."""
import numpy as np
import pytest

from tests import shared_ref as sh
from tests.test_cache4_cpu import FAKE, status


def shared_call(c, group, n, tokens, query, shared, width, lens=None, qlens=None, source=None):
    """Status of the call itself, up to the check of its workspace, and the largest quantum of its cut on the host (None: refused)."""
    import paper_2604_10539_amd as p
    from paper_2604_10539_amd import binding as b
    cap = min(width * c.block_size, 1 << 30)
    need = p.ice_cache_attend_shared_bytes(c, group, n, tokens, query, shared, cap, cap)
    assert need
    st = status(p.ice_cache_attend_shared, c, FAKE, 1 << 20, group, n, FAKE, FAKE, FAKE, tokens, query, shared, FAKE, cap, cap, FAKE, width, 0, FAKE, 0, None, FAKE, need - 1)
    start = np.concatenate([[0], np.cumsum(qlens)])
    plan = sh.sources(source, start, lens, n, tokens)
    try:
        parts = b.ice_debug_shared_cut(c, group, n, start, plan, tokens, query, shared, lens, cap, cap, width)
    except b.IceError as e:
        assert e.status == st == b.ICE_ERR_UNSUPPORTED
        return st, None
    x = dict(zip(b.CUT_FIELDS, parts.T.astype(np.int64)))
    assert np.all(x["now"] >= 0) and np.all(x["stop"] > x["now"])
    return st, int(x["u1"].max())


@pytest.mark.parametrize("requests, queries, block, heads, group", [
    (3000, 1, 16, 8, 4), (8191, 1, 16, 8, 4), (128, 256, 16, 8, 4), (500, 300, 16, 8, 4), (8000, 5, 64, 8, 8), (64, 1000, 16, 1, 16)])
def test_requests_behind_a_source_that_can_be_counted(requests, queries, block, heads, group):
    """A table of 128 K tokens a row, and no hints: nobody has more queries than the step's tokens."""
    import paper_2604_10539_amd as p
    from paper_2604_10539_amd import binding as b
    c = p.make_cache_desc(FAKE, 8192, heads, block)
    width, tokens = (1 << 17) // block, requests * queries
    lens = [1 << 17] + [queries + 300] * requests
    st, most = shared_call(c, group, requests + 1, tokens, tokens, tokens, width, lens, [0] + [queries] * requests, [-1] + [0] * requests)
    assert st == b.ICE_ERR_CAPACITY and 0 < most < 2 ** 31


def test_answers_to_many_sources_that_can_be_counted():
    import paper_2604_10539_amd as p
    from paper_2604_10539_amd import binding as b
    c, width = p.make_cache_desc(FAKE, 8192, 8, 16), 8192
    for rows, tokens in ((3000, 30000), (8192, 100000), (1, 10 ** 6)):
        need = p.ice_cache_attend_cross_bytes(c, 4, rows, tokens, 1 << 17)
        assert status(p.ice_cache_attend_cross, c, FAKE, 1 << 20, 4, rows, FAKE, tokens, tokens, FAKE, 1 << 17, FAKE, width, FAKE, 0, None, FAKE,
                      need - 1) == b.ICE_ERR_CAPACITY
        count = tokens // rows
        start = np.concatenate([np.arange(rows + 1) * count, [tokens]])
        parts = b.ice_debug_cross_cut(c, 4, rows, start, tokens, tokens, [1 << 17] * rows, 1 << 17, width)
        x = dict(zip(b.CUT_FIELDS, parts.T.astype(np.int64)))
        assert np.all(x["now"] >= 0) and np.all(x["stop"] > x["now"])


def test_the_edge_of_what_can_be_counted():
    """Rows of 2^30 tokens: 2^23 + 4 quanta a tile of 48 tokens, 8 KV heads, so 31 tiles at most, of two rows' own queries and of as many sources'."""
    import paper_2604_10539_amd as p
    from paper_2604_10539_amd import binding as b
    c = p.make_cache_desc(FAKE, 8192, 8, 64)
    width = (1 << 30) // 64
    lens = [(1 << 30) - 4] * 2
    st, most = shared_call(c, 4, 2, 671, 671, 671, width, lens, [0, 671], [-1, 0])
    assert st == b.ICE_ERR_CAPACITY and 2 ** 30 < most < 2 ** 31  # (14 tiles of one row's own, and 14 of its source's)
    st, most = shared_call(c, 4, 2, 672, 672, 672, width, lens, [0, 672], [-1, 0])
    assert st == b.ICE_ERR_UNSUPPORTED and most is None
    for tokens, want in ((1439, b.ICE_ERR_CAPACITY), (1488, b.ICE_ERR_CAPACITY), (1489, b.ICE_ERR_UNSUPPORTED)):
        need = p.ice_cache_attend_cross_bytes(c, 4, 1, tokens, 1 << 30)
        assert status(p.ice_cache_attend_cross, c, FAKE, 1 << 20, 4, 1, FAKE, tokens, tokens, FAKE, 1 << 30, FAKE, width, FAKE, 0, None, FAKE, need - 1) == want


@pytest.mark.parametrize("queries", [1, 60])
def test_starts_that_do_not_ascend_have_no_parts(queries):
    """As in the kernels.  Every second request with all of the step's queries would be more quanta than 32 bits count (300 of 2^24 tokens, 32 heads, two tiles)."""
    import paper_2604_10539_amd as p
    from paper_2604_10539_amd import binding as b
    n = 600
    c = p.make_cache_desc(FAKE, 8192, 32, 64)
    width, lens = 1 << 18, [1 << 24] * n
    good = np.minimum(np.arange(n + 1), queries)
    bad = np.arange(n + 1) % 2 * queries
    plan = {name: np.concatenate([start, [queries], np.zeros(n, int), np.arange(queries), np.zeros(queries, int)]) for name, start in (("good", good), ("bad", bad))}
    cut = lambda start, listed: b.ice_debug_shared_cut(c, 4, n, start, plan[listed], queries, queries, queries, lens, 1 << 24, 1 << 24, width)  # noqa: E731
    assert len(cut(good, "good")) > 0
    for start, listed in ((good, "bad"), (bad, "good"), (bad, "bad")):
        assert len(cut(start, listed)) == 0
    for start in (good, bad):
        parts = b.ice_debug_cross_cut(c, 4, n, np.concatenate([start, [queries]]), queries, queries, lens, 1 << 24, width)
        assert (len(parts) > 0) == (start is good)


def test_a_most_that_a_step_cannot_have_counts_as_it_is_given():
    import paper_2604_10539_amd as p
    from paper_2604_10539_amd import binding as b
    c = p.make_cache_desc(FAKE, 8192, 8, 16)
    call = lambda tokens, query, shared: status(  # noqa: E731
        p.ice_cache_attend_shared, c, FAKE, 1 << 20, 4, 3000, FAKE, FAKE, FAKE, tokens, query, shared, FAKE, 64, 64, FAKE, 8192, 0, FAKE, 0, None, FAKE, 0)
    assert call(3000, 3000, 3000) == b.ICE_ERR_CAPACITY
    assert call(3000, 1, 1 << 20) == b.ICE_ERR_UNSUPPORTED and call(3000, 1 << 20, 1) == b.ICE_ERR_UNSUPPORTED
