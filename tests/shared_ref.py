"""Plain forms in numpy of what requests of the 4-bit cache share: rotated tokens that are held, sorted queries, attention behind a source."""
import numpy as np

from tests import cache_ref as ref

D, NONE = 128, 2 ** 31 - 1


def hold(x):
    """float32 values [..., 128] -> codes [..., 128], scale bytes [..., 4]: cache_ref.encode for values that are not bf16."""
    y = x.reshape(*x.shape[:-1], 4, 32)
    bad = ~np.isfinite(y).all(-1)
    y = np.where(bad[..., None], 0, y).astype(np.float64)
    top = np.abs(y).max(-1)
    e = np.frexp(np.where(top == 0, 1.0, top))[1] - 1
    e = np.where(top == 0, -1000, e + (top > 1.75 * np.exp2(e.astype(np.float64))))
    byte = np.clip(e - 2, -100, 125) + 127
    m = np.abs(y) / np.exp2(byte - 127.0)[..., None]
    code = np.zeros(m.shape, dtype=np.uint8)
    for i, mid in enumerate((ref.LEVELS[1:] + ref.LEVELS[:-1]) / 2):  # a tie goes to the even code
        code += (m >= mid) if i % 2 else (m > mid)
    code |= np.where(np.signbit(x.reshape(y.shape)), 8, 0).astype(np.uint8)
    code[bad] = 0
    return code.reshape(x.shape), np.where(bad, 255, byte).astype(np.uint8)


def rotate(x, cos, sin, neighbours):
    """float32 rows x [..., 128]; cos, sin float32 [..., half]: products and sums each rounded."""
    x = x.astype(np.float32).copy()
    half = cos.shape[-1]
    a, b = (x[..., 0: 2 * half: 2].copy(), x[..., 1: 2 * half: 2].copy()) if neighbours else (x[..., :half].copy(), x[..., half: 2 * half].copy())
    with np.errstate(invalid="ignore", over="ignore"):
        c, d = a * cos - b * sin, a * sin + b * cos
    assert c.dtype == np.float32
    if neighbours:
        x[..., 0: 2 * half: 2], x[..., 1: 2 * half: 2] = c, d
    else:
        x[..., :half], x[..., half: 2 * half] = c, d
    return x


def source_of(source, s, rows, same):
    r = int(source[s])
    return r if 0 <= r < rows and not (same and r == s) else -1


def sources(source, start, lens, n_rows, n_tokens):
    """The plan as the header states it; lens None: the sources are rows of another table."""
    n = len(source)
    to = np.array([source_of(source, s, n_rows, lens is not None) for s in range(n)])
    to = np.where(to < 0, n_rows, to)
    many = np.diff(np.asarray(start))
    at = np.maximum(np.asarray(lens), 0) - many if lens is not None else np.zeros(n, int)
    begin, lowest = np.zeros(n_rows + 2, int), np.full(n_rows + 1, NONE)
    np.add.at(begin, to + 1, many)
    np.minimum.at(lowest, to[many > 0], at[many > 0])
    token, place = [], []
    for s in np.argsort(to, kind="stable"):
        token += range(int(start[s]), int(start[s + 1]))
        place += range(int(at[s]), int(at[s] + many[s])) if lens is not None else [0] * int(many[s])
    rest = [-1] * (n_tokens - len(token))
    return np.concatenate([np.cumsum(begin), lowest[:n_rows], token, rest, place, rest]).astype(np.int64)


def append(data, k, v, q, start, lens, source, table, rope, neighbours, block):
    """(data, rotated q as float32, rows of q that are written) after the step; k, v, q bf16 bits [tokens, heads, 128]."""
    data = data.copy()
    n, n_blocks = len(lens), data.shape[0]
    out, done = None if q is None else np.zeros(q.shape, np.float32), np.zeros(len(k), bool)
    for s in range(n):
        r = source_of(source, s, n, True) if source is not None else -1
        for t in range(int(start[s]), int(start[s + 1])):
            place = max(int(lens[s]), 0) - int(start[s + 1]) + t
            pos = place + (max(int(lens[r]), 0) if r >= 0 else 0)
            row = ref.widen(k[t])
            if rope is not None:
                if not 0 <= pos < len(rope):
                    continue
                half = rope.shape[1] // 2
                cos, sin = rope[pos, :half], rope[pos, half:]
                row = rotate(row, cos, sin, neighbours)
                if q is not None:
                    out[t] = rotate(ref.widen(q[t]), cos, sin, neighbours)
                    done[t] = True
            if not 0 <= place < table.shape[1] * block:
                continue
            b = int(table[s, place // block])
            if not 0 <= b < n_blocks:
                continue
            for side, x in ((0, row), (1, ref.widen(v[t]))):
                code, byte = hold(x)
                for h in range(data.shape[1]):
                    ref.put(data, b, h, place % block, side, code[h], byte[h])
    return data, out, done


def held_rows(data, table_row, length, block, h):
    """Float64 keys and values of the first tokens of a row, and which of them exist."""
    pos = np.arange(int(min(max(length, 0), len(table_row) * block)))
    blk = table_row[pos // block]
    there = (blk >= 0) & (blk < data.shape[0])
    k, v = ref.rows(data, np.where(there, blk, 0), pos % block, h)
    return np.where(there[:, None], k, 0), np.where(there[:, None], v, 0), there


def attention(q, data, table, lens, qlens, source, block, group, window, bf16_out, many, cross=False):
    """Query rows in order: (out, lse, tol, lse_tol), [tokens, heads, ...].  cross: table and lens are the sources'."""
    heads, parts, at, kept = data.shape[1], [], 0, {}

    def of_source(r, h):
        if (r, h) not in kept:
            kept[r, h] = held_rows(data, table[r], lens[r], block, h)
        return kept[r, h]
    for s, m in enumerate(qlens):
        if m == 0:
            continue
        r = source_of(source, s, len(lens), not cross)
        before = max(int(lens[r]), 0) if r >= 0 else 0
        res = []
        for h in range(heads):
            rows = [of_source(r, h) + (0,)] if r >= 0 else []
            if not cross:
                rows.append(held_rows(data, table[s], lens[s], block, h) + (before,))
            if rows:
                k, v, there = (np.concatenate([x[i] for x in rows]) for i in range(3))
                pos = np.concatenate([x[3] + np.arange(len(x[0])) for x in rows])
            else:
                k, v, there, pos = np.zeros((0, D)), np.zeros((0, D)), np.zeros(0, bool), np.zeros(0, int)
            seen = np.repeat(there[None], m, 0)
            if not cross:
                own = before + max(int(lens[s]), 0) - m + np.arange(m)[:, None]
                seen &= pos[None] <= own
                if window:
                    seen &= pos[None] > own - window
            rows = ref.softmax_rows(q[at: at + m, h * group: (h + 1) * group].reshape(m * group, D), k, v, np.repeat(seen, group, 0), bf16_out, many)
            res.append([x.reshape(m, group, *x.shape[1:]) for x in rows])
        parts.append([np.concatenate([x[i] for x in res], 1) for i in range(4)])
        at += m
    return [np.concatenate([p[i] for p in parts]) for i in range(4)]
