"""Plain forms of the 4-bit cache in numpy and 64 bits, for its tests: holding a row, the tiles' layout, a step's plan, attention."""
import numpy as np

D, TILE, TILE_BYTES = 128, 16, 2176
LEVELS = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=np.float64)


def widen(bits):
    return (np.ascontiguousarray(bits, dtype=np.uint16).astype(np.uint32) << 16).view(np.float32)


def to_bf16(x):
    b = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32)
    return ((b + np.uint32(0x7FFF) + ((b >> np.uint32(16)) & np.uint32(1))) >> np.uint32(16)).astype(np.uint16)


def encode(bits):
    """bf16 bits [..., 128] -> codes [..., 128], scale bytes [..., 4]."""
    x = widen(bits).astype(np.float64).reshape(*bits.shape[:-1], 4, 32)
    top = np.abs(x).max(-1)
    bad = ~np.isfinite(x).all(-1)
    e = np.frexp(np.where(bad | (top == 0), 1.0, top))[1] - 1
    e = np.where(top == 0, -1000, e + (top > 1.75 * np.exp2(e.astype(np.float64))))
    byte = np.clip(e - 2, -100, 125) + 127
    y = np.abs(np.where(bad[..., None], 0, x)) / np.exp2(byte - 127.0)[..., None]
    mid = (LEVELS[1:] + LEVELS[:-1]) / 2
    code = np.zeros(y.shape, dtype=np.uint8)
    for i, m in enumerate(mid):  # a tie goes to the even code
        code += (y >= m) if i % 2 else (y > m)
    code |= np.where(np.signbit(x), 8, 0).astype(np.uint8)
    code[bad] = 0
    byte = np.where(bad, 255, byte).astype(np.uint8)
    return code.reshape(bits.shape), byte


def decode(code, byte):
    v = LEVELS[code & 7] * np.where(code & 8, -1.0, 1.0)
    s = np.where(byte == 255, np.nan, np.exp2(byte.astype(np.float64) - 127))
    return (v.reshape(*byte.shape, 32) * s[..., None]).reshape(code.shape)


def scale_at(t, j):
    return 16 * (t % 4) + 4 * j + t // 4


def put(data, block, head, place, side, code, byte):
    """Stores one row in data [blocks, heads, tiles, 2176]."""
    tile, t = data[block, head, place // TILE], place % TILE
    tile[1024 * side + 64 * t: 1024 * side + 64 * t + 64] = code[0::2] | code[1::2] << 4
    for j in range(4):
        tile[2048 + 64 * side + scale_at(t, j)] = byte[j]


def rows(data, blocks, places, head):
    """Keys and values, float64 [n, 128] each, of the listed places."""
    t = places % TILE
    tiles = data[blocks, head, places // TILE].reshape(len(places), TILE_BYTES)
    out = []
    for side in (0, 1):
        at = 1024 * side + 64 * t[:, None] + np.arange(64)
        b = np.take_along_axis(tiles, at, 1)
        code = np.stack([b & 15, b >> 4], -1).reshape(len(t), D)
        at = 2048 + 64 * side + scale_at(t[:, None], np.arange(4))
        out.append(decode(code, np.take_along_axis(tiles, at, 1)))
    return out


def plan(new_len, cached_len, table, free_ids, n_free, block, n_slots):
    """The step as the header states it: (seq_len, table, free_ids, n_free_left, query_start, slots, info)."""
    table, free_ids = table.copy(), free_ids.copy()
    n, width = table.shape
    after = [max(int(c) + int(g), 0) for c, g in zip(cached_len, new_len)]
    held, need = [-(-int(c) // block) for c in cached_len], [-(-a // block) for a in after]
    taken, back = sum(max(b - a, 0) for a, b in zip(held, need)), sum(max(a - b, 0) for a, b in zip(held, need))
    fresh = sum(max(int(g), 0) for g in new_len)
    err = 0
    bad = [not 0 <= int(c) <= width * block for c in cached_len]
    if any(bad) or not 0 <= n_free <= len(free_ids) or n_free + back > len(free_ids):
        err |= 8
    elif taken > n_free + back:
        err |= 1
    if any(a > width * block and not x for a, x in zip(after, bad)):
        err |= 2
    if fresh > n_slots:
        err |= 4
    if err:
        return np.array(cached_len), table, free_ids, n_free, np.zeros(n + 1, int), np.full(n_slots, -1), np.array([0, 0, 0, err])
    for s in range(n):
        for j in range(need[s], held[s]):
            free_ids[n_free] = table[s, j]
            n_free += 1
    for s in range(n):
        for j in range(held[s], need[s]):
            n_free -= 1
            table[s, j] = free_ids[n_free]
    start, slots = [0], []
    for s in range(n):
        g = max(int(new_len[s]), 0)
        start.append(start[-1] + g)
        slots += [int(table[s, p // block]) * block + p % block for p in range(after[s] - g, after[s])]
    slots += [-1] * (n_slots - len(slots))
    return np.array(after), table, free_ids, n_free, np.array(start), np.array(slots), np.array([fresh, taken, back, 0])


def softmax_rows(q, k, v, seen, bf16_out, many=False):
    """(out, lse, tolerance of out, tolerance of lse) of query rows q [r, 128] against keys [n, 128], seen [r, n], in 64 bits.

    Tolerance.  A score is a chain of 128 exact products in fp32 and a multiplication: off by at most 130 * 2^-23 of the sum of
    the products' magnitudes (an addition is taken to be off by a whole unit of the last place), times log2(e) / sqrt(128) in powers of two;
    the exponent subtracts the reference (one more rounding of a number of the scores' size) and exp2 is taken to be good to 2^-21.  With d the
    largest such error among a row's scores in natural units, every weight and their sum are off by a factor within e^(+-d): 2 d between them.  Sums of n
    weighted values in fp32, rescaled now and then and joined: (n + 64) 2^-23 of the sum of their magnitudes, for the denominator
    likewise.  Weights in three bf16 terms: 2^-24; in two (bf16 outputs): 2^-16; a bf16 output is rounded by at most 2^-8.  A bf16 output of a
    call with more than 16 query rows per request (`many`) may come from weights rounded to bf16 once: each is off by at most half a step, 2^-8 of itself, so
    the sum by at most 2^-8 of the sum of the magnitudes (the denominator is summed from the weights before they are rounded)."""
    n = k.shape[0]
    s = q @ np.where(np.isnan(k), 0, k).T / np.sqrt(128.0)
    s = np.where(np.isnan(k).any(1)[None], np.nan, s)
    mag = np.abs(q) @ np.abs(np.where(np.isnan(k), 0, k)).T / np.sqrt(128.0)
    s = np.where(seen, s, -np.inf)
    any_seen = seen.any(1)
    top = np.where(any_seen, np.max(s, axis=1, initial=-np.inf), 0.0)
    with np.errstate(invalid="ignore"):
        p = np.exp(s - top[:, None])
    total = p.sum(1)
    p = p / np.where(any_seen, total, 1.0)[:, None]
    clean = np.where(np.isnan(v), 0, v)
    out = p @ clean
    # a NaN among the values of a dimension reaches the rows that see its token
    out = np.where((seen.astype(float) @ np.isnan(v).astype(float)) > 0, np.nan, out)
    with np.errstate(divide="ignore"):
        lse = top + np.log(total)
    d = np.where(seen, 130 * 2.0 ** -23 * mag, 0).max(1, initial=0) + 2.0 ** -21 + 2.0 ** -23 * np.where(any_seen, np.abs(np.where(np.isfinite(s), s, 0)).max(1, initial=0), 0) * 2
    weight = 2 * d + 2 * (n + 64) * 2.0 ** -23 + (2.0 ** -8 if bf16_out and many else 2.0 ** -16 if bf16_out else 2.0 ** -24)
    tol = weight[:, None] * (p @ np.abs(clean)) + (2.0 ** -8 * np.abs(out) if bf16_out else 0) + 1e-37
    lse_tol = d + (n + 64) * 2.0 ** -23 + 2.0 ** -22 * np.abs(np.where(any_seen, lse, 0))
    return out, lse, tol, lse_tol
