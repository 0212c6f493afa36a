"""GPU tests of the 4-bit cache: its plan, writing and reading, and attention over it, against plain numpy in 64 bits."""
import numpy as np
import pytest
import torch

from tests import cache_ref as ref
from tests.util import down, up

pytestmark = pytest.mark.gpu
D = 128


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def make(n_blocks, heads, block, fill=None):
    from paper_2604_10539_amd import IceCache
    c = IceCache(n_blocks, heads, block)
    if fill is not None:
        c.data.copy_(torch.from_numpy(fill).reshape(c.data.shape))
    return c


def random_pool(rng, n_blocks, heads, block, garbage=False):
    """Tiles whose rows are N(0, 1) values as the cache holds them, or any bytes at all."""
    tiles = block // 16
    if garbage:
        return rng.integers(0, 256, (n_blocks, heads, tiles, 2176), dtype=np.uint8)
    data = np.zeros((n_blocks, heads, tiles, 2176), dtype=np.uint8)
    for side in (0, 1):
        x = rng.standard_normal((n_blocks, heads, tiles, 16, D)).astype(np.float32) * np.exp(0.5 * rng.standard_normal((heads, 1, 1, D))).astype(np.float32)
        code, byte = ref.encode(ref.to_bf16(x))
        data[..., 1024 * side: 1024 * side + 1024] = (code[..., 0::2] | code[..., 1::2] << 4).reshape(n_blocks, heads, tiles, 1024)
        t, j = np.arange(16)[:, None], np.arange(4)
        at = 2048 + 64 * side + ref.scale_at(t, j)
        data[..., at] = byte
    return data


def tables(rng, lens, block, spare=3):
    need = [-(-n // block) for n in lens]
    ids = rng.permutation(sum(need) + spare).astype(np.int32)
    table = np.full((len(lens), max(1, max(need))), -1, dtype=np.int32)
    at = 0
    for s, k in enumerate(need):
        table[s, :k] = ids[at: at + k]
        at += k
    return len(ids), table


# ------------------------------------------------------------------------------------------------------ writing and reading
def _rows_of_bits(rng, kind, n):
    if kind == "normal":
        return ref.to_bf16(rng.standard_normal((n, D)).astype(np.float32))
    if kind == "any":  # every bit pattern, infinities and NaN among them
        return rng.integers(0, 65536, (n, D), dtype=np.uint16)
    if kind == "exponents":  # finite, magnitudes from subnormal to the largest
        b = rng.integers(0, 65536, (n, D), dtype=np.uint16)
        return np.where((b & 0x7F80) == 0x7F80, b & 0xBFFF, b).astype(np.uint16)
    if kind == "narrow":  # each block's magnitudes within a few powers of two of a random one: every border of the scale
        e = rng.integers(-120, 126, (n, 4, 1)).astype(np.float64)
        x = rng.standard_normal((n, 4, 32)) * np.exp2(e)
        return ref.to_bf16(np.clip(x, -3.3e38, 3.3e38).astype(np.float32).reshape(n, D))
    # ties: halves and quarters between the levels of the scale that a largest value of 6 or 4 gives
    x = rng.integers(-24, 25, (n, 4, 32)) / 4.0
    x[..., 0] = rng.choice([4.0, 6.0, 7.0, 7.25, 7.5], (n, 4))
    return ref.to_bf16((x * np.exp2(rng.integers(-20, 20, (n, 4, 1)))).astype(np.float32).reshape(n, D))


@pytest.mark.parametrize("kind", ["normal", "any", "exponents", "narrow", "ties"])
@pytest.mark.parametrize("tokens,heads,block", [(1, 1, 16), (17, 3, 32), (200, 2, 64)])
def test_rows_are_held_bit_for_bit(kind, tokens, heads, block):
    rng = np.random.default_rng([tokens, heads, len(kind)])
    n_blocks = -(-tokens // block) + 2
    before = rng.integers(0, 256, (n_blocks, heads, block // 16, 2176), dtype=np.uint8)
    c = make(n_blocks, heads, block, before)
    slots = rng.permutation(n_blocks * block)[:tokens].astype(np.int32)
    drop = rng.random(tokens) < 0.2
    slots[drop] = rng.choice([-1, -7, n_blocks * block, 2 ** 31 - 1], int(drop.sum()))
    k, v = (_rows_of_bits(rng, kind, tokens * heads).reshape(tokens, heads, D) for _ in range(2))
    # rows of a fused projection: queries, keys, values side by side
    fused = rng.integers(0, 65536, (tokens, 4 * heads * D), dtype=np.uint16)
    fused[:, 2 * heads * D: 3 * heads * D] = k.reshape(tokens, -1)
    fused[:, 3 * heads * D:] = v.reshape(tokens, -1)
    x = up(fused)
    c.write(x[:, 2 * heads * D: 3 * heads * D].unflatten(1, (heads, D)), x[:, 3 * heads * D:].unflatten(1, (heads, D)), i32(slots))
    want = before.copy()
    for side, rows in ((0, k), (1, v)):
        code, byte = ref.encode(rows)
        for t, s in enumerate(slots):
            if 0 <= s < n_blocks * block:
                for h in range(heads):
                    ref.put(want, s // block, h, s % block, side, code[t, h], byte[t, h])
    assert np.array_equal(down(c.data), want)  # (and nothing else was touched)


def test_reading_gives_the_held_values_and_zeros_where_there_is_no_token():
    rng = np.random.default_rng(4)
    heads, block, lens = 3, 32, [75, 0, 200, 33]
    n_blocks, table = tables(rng, lens, block)
    data = random_pool(rng, n_blocks, heads, block)
    data[table[2, 1], 1, 0, 2048 + ref.scale_at(3, 2)] = 255  # a key block that is held as NaN
    table[3, 1] = n_blocks  # no such block
    table[0, 1] = -1
    lens[3] = 4000          # longer than its row of the table
    c = make(n_blocks, heads, block, data)
    first = np.array([-3, 5, 20, 1], dtype=np.int32)
    for first_, n_rows in ((None, 1), (first, 77), (first, 210)):
        K, V = c.read(i32(table), i32(lens), n_rows, first=None if first_ is None else i32(first_))
        K, V = K.float().cpu().numpy(), V.float().cpu().numpy()
        for s in range(len(lens)):
            pos = np.arange(n_rows) + (0 if first_ is None else int(first_[s]))
            ok = (pos >= 0) & (pos < min(lens[s], table.shape[1] * block))
            blk = np.where(ok, table[s, np.clip(pos // block, 0, table.shape[1] - 1)], 0)
            ok &= (blk >= 0) & (blk < n_blocks)
            for h in range(heads):
                k, v = ref.rows(data, np.clip(blk, 0, n_blocks - 1), np.clip(pos, 0, None) % block, h)
                assert np.array_equal(K[s, h], np.where(ok[:, None], k, 0).astype(np.float32), equal_nan=True)
                assert np.array_equal(V[s, h], np.where(ok[:, None], v, 0).astype(np.float32), equal_nan=True)
    K, V = c.read(i32(table), i32(lens), 0)
    assert K.numel() == 0


# -------------------------------------------------------------------------------------------------------------- plan
@pytest.mark.parametrize("requests,block,n_slots", [(1, 16, 1), (3, 64, 300), (5, 32, 5000), (40, 16, 4096), (1024, 16, 9000), (1025, 32, 700), (2500, 16, 20000),
                                                    (5000, 16, 4500)])
def test_plans_follow_each_other(requests, block, n_slots):
    from paper_2604_10539_amd import IceBlocks, ice_plan_blocks
    rng = np.random.default_rng([requests, block])
    width = 400 if requests <= 5 else 12
    n_blocks = max(8, min(requests * width, requests * 5 + 200))
    b = IceBlocks(n_blocks, block, requests, width * block)
    table, free_ids, n_free, lens = down(b.block_table).copy(), down(b.free_ids).copy(), n_blocks, np.zeros(requests, dtype=np.int64)
    seen = set()
    for step in range(8):
        gain = np.ones(requests, dtype=np.int64)
        x = rng.random(requests)
        few = max(1, (n_slots - requests) // max(1, requests // 4))
        gain[x < 0.3] = rng.integers(0, min(few, width * block // 3) + 1, int((x < 0.3).sum()))
        gain[x > 0.8] = -rng.integers(0, 3 * block, int((x > 0.8).sum()))
        ends = x > 0.95
        gain[ends] = rng.choice([-lens.max() - 1, -2 ** 31], int(ends.sum()))
        if step == 6:
            gain[:] = -1
        want = ref.plan(gain, lens, table, free_ids, n_free, block, n_slots)
        # the same step into arrays of its own, from copies
        copy = [t.clone() for t in (b.seq_len, b.block_table, b.free_ids, b.n_free)]
        e = lambda n: torch.full((n,), 77, dtype=torch.int32, device="cuda")  # noqa: E731
        apart = [e(requests), copy[1], copy[2], e(1), e(requests + 1), e(n_slots), e(4)]
        ice_plan_blocks(i32(gain), copy[0], apart[0], copy[1], copy[2], copy[3], apart[3], apart[4], apart[5], apart[6], block)
        start, slots, info = b.plan(i32(gain), n_slots)
        for x, y in zip(apart, (b.seq_len, b.block_table, b.free_ids, b.n_free, start, slots, info)):
            assert torch.equal(x, y)
        got = [down(t) for t in (b.seq_len, b.block_table, b.free_ids, b.n_free, start, slots, info)]
        assert np.array_equal(got[6], want[6]), (step, got[6], want[6])
        for name, g, w in zip(("seq_len", "table", "free_ids", "n_free", "query_start", "slots"), got, want):
            assert np.array_equal(g.reshape(-1), np.asarray(w).reshape(-1)), (step, name)
        lens, table, free_ids, n_free = want[:4]
        seen.add(int(want[6][3]))
        live = [set(table[s, : -(-int(lens[s]) // block)]) for s in range(requests)]
        assert sum(map(len, live)) == len(set().union(*live)) and n_free + sum(map(len, live)) == n_blocks
    assert 0 in seen


@pytest.mark.parametrize("requests", [2, 1100])
def test_a_step_that_cannot_be_is_refused_whole(requests):
    from paper_2604_10539_amd import ice_plan_blocks
    rng = np.random.default_rng(1)
    block, width, n_blocks = 16, 4, requests * 2 + 6
    lens = np.full(requests, 20)
    table = np.full((requests, width), -1)
    ids = rng.permutation(n_blocks)
    table[:, :2] = ids[: 2 * requests].reshape(requests, 2)
    free = np.full(n_blocks, -1)
    free[:6] = ids[2 * requests:]
    one = np.zeros(requests, dtype=np.int64)

    def step(gain, cached=lens, n_free=6, n_slots=89):
        want = ref.plan(gain, cached, table, free, n_free, block, n_slots)
        t, f = i32(table), i32(free)
        e = lambda n: torch.full((n,), 77, dtype=torch.int32, device="cuda")  # noqa: E731
        seq_len, left, start, slots, info = e(requests), e(1), e(requests + 1), e(n_slots), e(4)
        ice_plan_blocks(i32(gain), i32(cached), seq_len, t, f, i32([n_free]), left, start, slots, info, block)
        got = [down(x).reshape(-1) for x in (seq_len, t, f, left, start, slots, info)]
        for g, w in zip(got, want):
            assert np.array_equal(g, np.asarray(w).reshape(-1)), (got[6], want[6])
        return int(want[6][3])

    def gains(**at):
        g = one.copy()
        for i, x in at.items():
            g[int(i[1:])] = x
        return g
    last = "r%d" % (requests - 1)
    assert step(gains(r0=28)) == 0
    assert step(gains(**{"r0": 44, last: 44})) == 0
    assert step(gains(**{"r0": 44, last: 45})) == 2
    assert step(gains(r0=44), n_free=1) == 1
    assert step(gains(**{"r0": 44, last: -20}), n_free=1) == 0       # the blocks given back are taken
    assert step(gains(**{"r0": 44, last: -3}), n_free=1) == 1
    assert step(gains(r0=44), n_slots=43) == 4
    assert step(gains(r0=2 ** 31 - 1)) == 7
    assert step(np.full(requests, 2 ** 31 - 1)) == 7
    assert step(one, n_free=-1) == 8 and step(one, n_free=n_blocks + 1) == 8
    assert step(gains(r0=-20), n_free=n_blocks) == 8                  # more blocks than there are
    bad = lens.copy()
    bad[-1] = -5
    assert step(one, cached=bad) == 8
    bad[-1] = width * block + 1
    assert step(one, cached=bad) == 8
    assert step(gains(r0=-2 ** 31)) == 0


# ------------------------------------------------------------------------------------------------------------- attention
def check(got, lse, want):
    out, z, tol, ztol = want
    got, lse = got.double().cpu().numpy(), lse.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(out)), "NaN at other places: %s" % np.argwhere(np.isnan(got) != np.isnan(out))[:4]
    off = np.abs(np.nan_to_num(got) - np.nan_to_num(out)) / np.nan_to_num(tol, nan=1.0)
    assert off.max(initial=0) <= 1, "output off by %.2f of its tolerance at %s" % (off.max(), np.unravel_index(off.argmax(), off.shape))
    inf = np.isneginf(z)
    assert np.array_equal(np.isneginf(lse), inf) and np.array_equal(np.isnan(lse), np.isnan(z))
    offz = np.where(inf | np.isnan(z), 0, np.abs(np.where(inf, 0, lse) - np.where(inf, 0, z))) / ztol
    assert np.nan_to_num(offz).max(initial=0) <= 1, "lse off by %.2f of its tolerance" % offz.max()


def expected(q, data, table, lens, qlens, block, group, window, bf16_out, n_blocks):
    """Query rows in order: (out, lse, tol, lse_tol), [tokens, heads, ...]."""
    heads = data.shape[1]
    parts = []
    at = 0
    for s, (n, m) in enumerate(zip(lens, qlens)):
        if m == 0:
            continue
        n_ = int(min(max(n, 0), table.shape[1] * block))
        pos = np.arange(n_)
        blk = table[s, pos // block]
        there = (blk >= 0) & (blk < n_blocks)
        qpos = n_ - m + np.arange(m)
        seen = (pos[None] <= qpos[:, None]) & there[None]
        if window:
            seen &= pos[None] > qpos[:, None] - window
        res = []
        for h in range(heads):
            k, v = ref.rows(data, np.where(there, blk, 0), pos % block, h)
            k, v = np.where(there[:, None], k, 0), np.where(there[:, None], v, 0)
            for j in range(group):
                res.append(ref.softmax_rows(q[at: at + m, h * group + j], k, v, seen, bf16_out, max(qlens) * group > 16))
        parts.append([np.stack([r[i] for r in res], 1) for i in range(4)])
        at += m
    return [np.concatenate([p[i] for p in parts]) for i in range(4)]


def run_attend(rng, heads, group, block, lens, qlens, window, dtype, garbage=True, data=None, table=None, fused=True, max_len=None, edit=None):
    if table is None:
        n_blocks, table = tables(rng, [max(0, n) for n in lens], block)
    else:
        n_blocks = data.shape[0]
    if data is None:
        data = random_pool(rng, n_blocks, heads, block)
    if garbage:  # what lies behind a request's last token, and in blocks that nobody owns
        junk = random_pool(rng, n_blocks, heads, block, True)
        keep = np.zeros((n_blocks, block), dtype=bool)
        for s, n in enumerate(lens):
            for p in range(min(max(n, 0), table.shape[1] * block)):
                if 0 <= table[s, p // block] < n_blocks:
                    keep[table[s, p // block], p % block] = True
        for b, p in np.argwhere(~keep):
            for side in (0, 1):
                t = p % 16
                at = np.concatenate([1024 * side + 64 * t + np.arange(64), 2048 + 64 * side + ref.scale_at(t, np.arange(4))])
                data[b, :, p // 16, at] = junk[b, :, p // 16, at]
            if p % 3 == 0:
                data[b, :, p // 16, 2048 + ref.scale_at(p % 16, np.arange(4))] = 255
                data[b, :, p // 16, 2112 + ref.scale_at(p % 16, np.arange(4))] = 255
    if edit is not None:
        edit(data, table)
    c = make(n_blocks, heads, block, data)
    total, hq = sum(qlens), heads * group
    q = ref.to_bf16(rng.standard_normal((total, hq, D)).astype(np.float32))
    behind = 3  # rows behind the last request
    x = rng.integers(0, 65536, (total + behind, hq * D * (3 if fused else 1)), dtype=np.uint16)
    x[:total, : hq * D] = q.reshape(total, -1)
    qt = up(x)[:, : hq * D].unflatten(1, (hq, D))
    start = np.concatenate([[0], np.cumsum(qlens)])
    out = torch.full((total + behind, hq, D), 7.0, dtype=dtype, device="cuda")
    lse = torch.full((total + behind, hq), 7.0, dtype=torch.float32, device="cuda")
    c.attend(qt, i32(start), i32(lens), i32(table), max_query=max(qlens), max_len=max_len, window=window, out=out, lse=lse)
    assert bool((out[total:] == 7).all()) and bool((lse[total:] == 7).all())
    want = expected(ref.widen(q).astype(np.float64), data, table, lens, qlens, block, group, window, dtype is torch.bfloat16, n_blocks)
    check(out[:total], lse[:total], want)
    return c, qt[:total], start, table


CASES = [  # heads, group, block, lengths, queries, window
    (1, 1, 16, [1], [1], 0),
    (2, 4, 16, [1, 15, 16, 17, 31, 32, 33, 0], [1, 1, 1, 1, 1, 1, 1, 1], 0),
    (2, 4, 64, [63, 64, 65, 257, 1000], [1, 1, 1, 1, 1], 0),
    (3, 7, 32, [300, 5, 129], [1, 1, 1], 0),
    (1, 16, 16, [500, 40], [1, 2], 0),
    (2, 8, 32, [513, 90, 4, 0], [5, 5, 4, 2], 0),          # drafts; a request with more queries than tokens
    (2, 8, 32, [700, 90, 40], [5, 3, 1], 64),
    (1, 4, 16, [2000], [1], 1),                             # a window of the query's own token
    (2, 3, 16, [333, 70, 0, 200, 17], [40, 70, 0, 1, 17], 0),
    (1, 5, 64, [400, 350], [130, 1], 50),
    (1, 4, 32, [5000], [1], 0),
    (1, 2, 16, [3000, 10], [37, 10], 1000),
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention_over_the_cache(case, dtype):
    heads, group, block, lens, qlens, window = CASES[case]
    rng = np.random.default_rng([7, case])
    run_attend(rng, heads, group, block, lens, qlens, window, dtype, fused=case % 2 == 0, max_len=max(lens) if case % 3 else None)


@pytest.mark.parametrize("requests,heads,max_len", [(1, 1, 4000), (1, 1, 100), (40, 8, 300), (130, 8, 300)])
def test_any_cut_of_the_keys_gives_the_result(requests, heads, max_len):
    """max_len only cuts the work: too small a hint, many requests and few give the same."""
    rng = np.random.default_rng(requests)
    lens = [3000] + [int(x) for x in rng.integers(0, 300, requests - 1)]
    run_attend(rng, heads, 2, 64, lens, [1] * requests, 0, torch.float32, garbage=requests < 10, max_len=max_len)


@pytest.mark.parametrize("queries", [4, 40])
def test_nan_reaches_only_the_rows_that_see_it(queries):
    """A value or key block held as NaN in a token that only the later queries of a chunk see."""
    rng = np.random.default_rng(3)
    lens, block = [200, 100], 16

    def edit(data, table):
        for s, p, side, j in ((0, 198, 1, 1), (0, 199, 0, 2), (1, 30, 1, 3)):
            data[table[s, p // block], 0, 0, 2048 + 64 * side + ref.scale_at(p % 16, j)] = 255
    run_attend(rng, 2, 4, block, lens, [queries, queries], 0, torch.float32, edit=edit)
    run_attend(rng, 2, 4, block, lens, [queries, queries], 20, torch.bfloat16, edit=edit)


@pytest.mark.parametrize("queries", [1, 33])
def test_blocks_that_do_not_exist_are_left_out(queries):
    rng = np.random.default_rng(5)
    heads, block, lens = 2, 16, [250, 80, 10000]
    n_blocks, table = tables(rng, [250, 80, 100], block)
    data = random_pool(rng, n_blocks, heads, block)
    table[0, 3], table[0, 4], table[0, 15], table[1, :] = -1, n_blocks, -2 ** 31, 2 ** 31 - 1
    table[2, 7:] = -1
    run_attend(rng, heads, 4, block, lens, [queries] * 3, 0, torch.float32, garbage=False, data=data, table=table)


def test_scores_of_any_size():
    """Queries so large that all but one weight vanish, and rows whose scores all lie far below zero."""
    rng = np.random.default_rng(6)
    heads, block, lens = 1, 16, [90, 90]
    n_blocks, table = tables(rng, lens, block)
    data = random_pool(rng, n_blocks, heads, block)
    for s in (0, 1):
        for p in range(90):
            data[table[s, p // block], 0, 0, 2048 + ref.scale_at(p % 16, np.arange(4))] += 12 if s else 6
    run_attend(rng, heads, 4, block, lens, [1, 3], 0, torch.float32, garbage=False, data=data, table=table)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("requests,heads,group,block,most", [(1, 1, 1, 16, 1), (2, 3, 4, 16, 33), (3, 2, 7, 64, 300), (1, 8, 4, 32, 2500), (5, 2, 16, 16, 31)])
def test_attention_over_listed_tokens(requests, heads, group, block, most, dtype):
    rng = np.random.default_rng([requests, most])
    lens = [int(x) for x in rng.integers(1, 900, requests)]
    n_blocks, table = tables(rng, lens, block)
    data = random_pool(rng, n_blocks, heads, block)
    c = make(n_blocks, heads, block, data)
    pos = rng.integers(0, np.array(lens)[:, None, None], (requests, heads, most)).astype(np.int32)
    pos[..., 1::5] = pos[..., 0:1]                                        # the same token again
    bad = rng.random(pos.shape) < 0.1
    pos[bad] = rng.choice([-1, -2 ** 31, 2 ** 31 - 1, max(lens) + 5000], int(bad.sum()))
    n_tok = rng.integers(0, most + 1, (requests, heads)).astype(np.int32)
    n_tok[0, 0] = most
    if requests > 1:
        n_tok[1, 0], n_tok[-1, -1] = 0, most + 9                         # no tokens; more than the list holds
        pos[1, 1, :] = -1                                                # none that exists
    q = ref.to_bf16(rng.standard_normal((requests, heads * group, D)).astype(np.float32))
    out, lse = c.attend_tokens(up(q), i32(lens), i32(table), i32(pos), i32(n_tok), out_dtype=dtype, with_lse=True)
    res = []
    for s in range(requests):
        for h in range(heads):
            p = pos[s, h, : min(max(n_tok[s, h], 0), most)].astype(np.int64)
            p = p[(p >= 0) & (p < lens[s])]
            k, v = ref.rows(data, table[s, p // block], p % block, h)
            res.append(ref.softmax_rows(ref.widen(q[s, h * group: (h + 1) * group]).astype(np.float64), k, v, np.ones((group, len(p)), dtype=bool),
                                        dtype is torch.bfloat16))
    want = [np.stack([r[i] for r in res]).reshape(requests, heads * group, *res[0][i].shape[1:]) for i in range(4)]
    check(out, lse, want)


# ----------------------------------------------------------------------------------------------------- together, and apart
def test_layers_beside_an_index():
    """A decode step as the calls are used together: an anchor layer's index selects, a layer behind it attends to the selected
    tokens of its 4-bit cache, a dense layer to all of its own; plans, writes and reads on the way.  On the values that the cache
    holds the index's own attention over the selected pages is the same."""
    import datagen
    from paper_2604_10539_amd import IceBlocks, IceCache, IceIndex
    heads, group, n, page = 2, 4, 700, 16
    w = datagen.small(n_tokens=n, n_clusters=12, n_kv_heads=heads, n_components=12, seed=5)
    K, V = datagen.keys_values(w)  # [1, heads, n, 128]
    blocks = IceBlocks(64, 16, 1, 1024)
    cache = IceCache(64, heads, 16)
    start, slots, info = blocks.plan(i32([n]), 1024)
    k = up(K)[0].transpose(0, 1).contiguous()
    v = up(V)[0].transpose(0, 1).contiguous()
    cache.write(k, v, slots[:n].contiguous())
    Kh, Vh = cache.read(blocks.block_table, blocks.seq_len, n)
    ix = IceIndex(1, heads, group, n + 64, page, 12, kmeans_iters=3, init_idx=up(datagen.init_indices(w)))
    ix.build_index(Kh, Vh)
    st = datagen.DecodeStream(w)
    for step in range(3):
        k1, v1, q1 = st.next()
        q = up(q1)
        start, slots, info = blocks.plan(i32([1]), 16)
        cache.write(up(k1).expand(1, -1, -1), up(v1).expand(1, -1, -1), slots[:1].contiguous())
        assert down(info).tolist()[3] == 0 and int(blocks.seq_len[0]) == n + step + 1
        ids, n_sel, _ = ix.select(q, 160)
        pos, n_tok = ix.selected_tokens(ids, n_sel)
        dense = ix.attend(q, ids, n_sel)
        reused = cache.attend_tokens(q, blocks.seq_len, blocks.block_table, pos, n_tok)
        assert float((dense - reused).abs().max()) <= 2e-4  # (the guard of this repository's attention against its own oracle)
        full, lse = cache.attend(q, start, blocks.seq_len, blocks.block_table, max_query=1, with_lse=True)
        Kn, Vn = cache.read(blocks.block_table, blocks.seq_len, n + step + 1)
        data = down(cache.data)
        want = expected(ref.widen(q1).astype(np.float64), data, down(blocks.block_table), [n + step + 1], [1], 16, group, 0, False, 64)
        check(full, lse, want)
        assert torch.equal(Kn[:, :, :n], Kh) and torch.equal(Vn[:, :, :n], Vh)


def test_a_captured_step_is_replayed():
    """plan -> write -> attend in one graph, lengths and free blocks moving on in place, between eager calls of another size."""
    from paper_2604_10539_amd import IceBlocks, IceCache
    rng = np.random.default_rng(8)
    S, heads, group, block = 3, 2, 4, 16

    def fresh():
        b, c = IceBlocks(200, block, S, 640), IceCache(200, heads, block)
        start, slots, _ = b.plan(i32([100, 20, 300]), 512)
        x = torch.from_numpy(ref.to_bf16(np.random.default_rng(1).standard_normal((2, 420, heads, D)).astype(np.float32)).view(np.int16)).cuda()
        c.write(x[0], x[1], slots[:420].contiguous())
        return b, c
    gain = i32([1, 1, 1])
    q, k, v = (torch.empty((S, heads * m, D), dtype=torch.int16, device="cuda") for m in (group, 1, 1))

    def step(b, c, slots, out, lse):
        start, s, _ = b.plan(gain, S, slots=slots)
        c.write(k, v, s)
        c.attend(q, start, b.seq_len, b.block_table, max_query=1, max_len=640, out=out, lse=lse)
    inputs = [[torch.from_numpy(ref.to_bf16(rng.standard_normal(tuple(t.shape)).astype(np.float32)).view(np.int16)).cuda() for t in (q, k, v)] for _ in range(20)]

    def feed(i):
        for t, x in zip((q, k, v), inputs[i]):
            t.copy_(x)
    buf = lambda: (torch.empty(S, dtype=torch.int32, device="cuda"), torch.empty((S, heads * group, D), device="cuda"),  # noqa: E731
                   torch.empty((S, heads * group), device="cuda"))
    eb, ec = fresh()
    eager = []
    for i in range(20):
        feed(i)
        o = buf()
        step(eb, ec, *o)
        eager.append([t.clone() for t in o])
    gb, gc = fresh()
    other_b, other_c = fresh()
    state = [t.clone() for t in (gb.seq_len, gb.block_table, gb.free_ids, gb.n_free)]
    go = buf()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(gb, gc, *go)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(gb, gc, *go)
    for t, x in zip((gb.seq_len, gb.block_table, gb.free_ids, gb.n_free), state):
        t.copy_(x)
    for i in range(20):
        feed(i)
        graph.replay()
        got = [t.clone() for t in go]
        step(other_b, other_c, *buf())  # eager work of its own in between
        torch.cuda.synchronize()
        for g, e in zip(got, eager[i]):
            assert torch.equal(g, e), i
    assert torch.equal(gb.block_table, eb.block_table) and torch.equal(gb.free_ids, eb.free_ids)


def test_calls_on_two_streams_at_once():
    rng = np.random.default_rng(9)
    c, q, start, table = run_attend(rng, 2, 4, 32, [3000, 2000], [1, 1], 0, torch.float32, garbage=False)
    args = (q, i32(start), i32([3000, 2000]), i32(table))
    want = c.attend(*args, max_query=1)
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    got = []
    for _ in range(8):
        got += [c.attend(*args, max_query=1, stream=one), c.attend(*args, max_query=1, stream=two.cuda_stream)]
    torch.cuda.synchronize()
    assert all(torch.equal(g, want) for g in got)


def test_a_pool_beyond_32_bit_offsets():
    """Blocks whose bytes lie behind 4 GiB of a pool."""
    rng = np.random.default_rng(10)
    heads, block, n_blocks, lens = 8, 64, 70000, [150, 70]
    from paper_2604_10539_amd import IceCache
    c = IceCache(n_blocks, heads, block)
    table = np.array([[n_blocks - 1, 5, n_blocks - 3], [n_blocks - 2, 65000, -1]], dtype=np.int32)
    small = random_pool(rng, 5, heads, block)
    where = [n_blocks - 1, 5, n_blocks - 3, n_blocks - 2, 65000]
    near = np.array([[0, 1, 2], [3, 4, -1]], dtype=np.int32)
    q = ref.to_bf16(rng.standard_normal((2, heads * 4, D)).astype(np.float32))
    x = ref.to_bf16(rng.standard_normal((2, 220, heads, D)).astype(np.float32))
    slots = np.concatenate([table[s, np.arange(n) // block] * block + np.arange(n) % block for s, n in enumerate(lens)])
    c.write(up(x[0]), up(x[1]), i32(slots))
    for b, i in zip(where, range(5)):
        small[i] = down(c.data[b])
    code, byte = ref.encode(x[0, 100])
    k, _ = ref.rows(small, np.array([1]), np.array([100 - 64]), 3)
    assert np.array_equal(k[0], ref.decode(code[3], byte[3]))
    out, lse = c.attend(up(q), i32([0, 1, 2]), i32(lens), i32(table), max_query=1, with_lse=True)
    check(out, lse, expected(ref.widen(q).astype(np.float64), small, near, lens, [1, 1], block, 4, 0, False, 5))
    pos = rng.integers(0, 70, (2, heads, 40)).astype(np.int32)
    pos[0] += 80
    n_tok = np.full((2, heads), 40, dtype=np.int32)
    out, lse = c.attend_tokens(up(q), i32(lens), i32(table), i32(pos), i32(n_tok), with_lse=True)
    res = []
    for s in range(2):
        for h in range(heads):
            k, v = ref.rows(small, near[s, pos[s, h] // block], pos[s, h] % block, h)
            res.append(ref.softmax_rows(ref.widen(q[s, 4 * h: 4 * h + 4]).astype(np.float64), k, v, np.ones((4, 40), dtype=bool), False))
    check(out, lse, [np.stack([r[i] for r in res]).reshape(2, heads * 4, *res[0][i].shape[1:]) for i in range(4)])
    K, _ = c.read(i32(table), i32(lens), 150)
    k, _ = ref.rows(small, near[0, np.arange(150) // block], np.arange(150) % block, 7)
    assert np.array_equal(K[0, 7].float().cpu().numpy(), k.astype(np.float32))
