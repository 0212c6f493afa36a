"""What requests of a 4-bit KV cache share, and tokens that enter it with their positions rotated, as callable cases.

Four operators beside those of perf/operators.py, on the same cache:

  append   a step's queries, keys and values take their positions' rotation; keys and values go into the cache, queries come back
  sources  the step's queries sorted by the row of the block table that their requests share, once for all layers
  cross    attention of every query to all tokens of its request's source, a row of another table: an encoder's states, read once for all of them
  shared   causal attention of requests whose texts begin with a source's tokens: the common part is read once for all of them

Places and positions.  A source is a row of the block table.  Request s holds the tokens behind its source (source[s], -1: it has none): its
j-th of n queries stands at place seq_len[s] - n + j of its own row, and at position place + seq_len[source[s]] of its text.

Rotation.  Row p of the table `rope` holds cos and then sin of rot / 2 angles.  Pair i of a head's first rot dimensions, (i, i + rot / 2) or
(2 i, 2 i + 1), becomes (a cos - b sin, a sin + b cos): products and sums in 32 bits, each rounded; then queries are rounded to
bf16 and keys are held.

Held values.  A row of 128 values is four blocks of 32 with a scale 2^(b - 127) each, b a byte, and codes for +-{0, 0.5, 1, 1.5, 2, 3, 4, 6}.
With e = floor(log2(max |x|)) the scale is 2^(e - 2), twice that where max |x| > 1.75 * 2^e, and never below 2^-100 or above 2^125; a code is the nearest of the
sixteen to x / scale, to the even one on a tie; a block with a value that is not finite is held as NaN (b = 255).

Layout.  The cache is [block][KV head][tile of 16 tokens][2176 bytes]: 1024 bytes of key codes (64 per token, dimension 2i in the low half of
byte i), 1024 of value codes, 64 of key scales, 64 of value scales; the scale of token t's block j is at byte 16 (t mod 4) + 4 j + t / 4.

Sorted queries.  One int32 array for R rows and T tokens: start [R + 2], where in the list each row's queries begin, those of requests without a source at
start[R], and their number; first [R], the lowest place of a row's queries (2^31 - 1: it has none); token [T] and place [T] of the listed ones,
requests with one source in their own order, -1 behind the last.
"""
import math
import random
import zlib

import torch

own = False  # the plain forms; true: the calls of paper_2604_10539_amd

D = 128
TILE = 16
TILE_BYTES = 2176
ROW_BYTES = 136  # a token's keys and values of one KV head: half of it codes and scales of the keys
DEV = "cuda"
NONE = 2 ** 31 - 1
PART = 1 << 26  # values that the input makers and exact() touch at a time


def listed():
    return [
        # one decode step of a batch, out of the fused projection's output
        {"name": "append_step_16", "kind": "append", "requests": 16, "heads": 8, "group": 4, "block": 64, "ctx": 32768, "new": 1, "mix": 0,
         "sources": 0, "shared": 0, "rot": 128, "pairs": "halves"},
        # two prompts of 16k tokens
        {"name": "append_prompt_2x16k", "kind": "append", "requests": 2, "heads": 8, "group": 4, "block": 64, "ctx": 16384, "new": 16384, "mix": 0,
         "sources": 0, "shared": 0, "rot": 128, "pairs": "halves"},
        # chunks beside single tokens behind three documents of up to 100k tokens, half of a head's dimensions rotated
        {"name": "append_mixed_64", "kind": "append", "requests": 64, "heads": 8, "group": 2, "block": 16, "ctx": 8192, "new": 500, "mix": 1,
         "sources": 3, "shared": 100000, "rot": 64, "pairs": "neighbours"},
        # a decode step of a batch with two common system prompts
        {"name": "sources_32", "kind": "sources", "requests": 32, "ctx": 4096, "new": 1, "mix": 0, "sources": 2, "shared": 2048},
        # a busy server's step: chunks, single tokens and requests that wait, forty common texts
        {"name": "sources_mixed_2000", "kind": "sources", "requests": 2000, "ctx": 8192, "new": 700, "mix": 1, "sources": 40, "shared": 8192},
        # the smallest: one token that reads 1500 encoded frames
        {"name": "cross_1x1500", "kind": "cross", "requests": 1, "heads": 8, "group": 2, "block": 16, "sources": 1, "shared": 1500, "query": 1, "mix": 0,
         "out": "bfloat16"},
        # a step of beam search, five beams to each of sixteen recordings
        {"name": "cross_beams_16x5", "kind": "cross", "requests": 80, "heads": 8, "group": 2, "block": 16, "sources": 16, "shared": 1500, "query": 1,
         "mix": 0, "out": "float32"},
        # answers that are scored as a whole against long encoded documents
        {"name": "cross_answers_8x4k", "kind": "cross", "requests": 8, "heads": 8, "group": 4, "block": 64, "sources": 8, "shared": 4096, "query": 450,
         "mix": 0, "out": "bfloat16"},
        # the smallest: four samples of one prompt, two KV heads on this GPU
        {"name": "shared_4x2k", "kind": "shared", "requests": 4, "heads": 2, "group": 4, "block": 16, "sources": 1, "shared": 2048, "ctx": 130, "query": 1,
         "mix": 0, "window": 0, "out": "float32"},
        # a batch's decode step behind one document of 32k tokens
        {"name": "shared_32x32k", "kind": "shared", "requests": 32, "heads": 8, "group": 4, "block": 64, "sources": 1, "shared": 32768, "ctx": 1024,
         "query": 1, "mix": 0, "window": 0, "out": "bfloat16"},
        # four drafted tokens per request are checked, six system prompts, a layer with a sliding window; merged with an index's outputs
        {"name": "shared_draft_48x8k", "kind": "shared", "requests": 48, "heads": 8, "group": 2, "block": 32, "sources": 6, "shared": 8192, "ctx": 2048,
         "query": 4, "mix": 0, "window": 4096, "out": "float32"},
        # questions of 500 tokens about one document, beside requests that answer already
        {"name": "shared_chunk_6x32k", "kind": "shared", "requests": 6, "heads": 8, "group": 4, "block": 64, "sources": 1, "shared": 32768, "ctx": 1500,
         "query": 500, "mix": 1, "window": 0, "out": "bfloat16"},
    ]


def _near(rng, low, high):
    """A whole number between the two, spread over the logarithm."""
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    kind = rng.choice(["append", "append", "sources", "cross", "cross", "shared", "shared", "shared"])
    heads, group = rng.choice([(1, 1), (1, 8), (2, 1), (2, 4), (2, 16), (5, 1), (5, 2), (5, 7), (8, 2), (8, 4)])
    block, mix, requests = rng.choice([16, 32, 64]), rng.choice([0, 1]), _near(rng, 1, 64)
    sources = min(requests, rng.choice([1, 1, _near(rng, 1, 16)]))
    if kind == "sources":
        return {"kind": kind, "requests": _near(rng, 1, 2000), "ctx": _near(rng, 1, 8192), "new": _near(rng, 1, 700) if mix else 1, "mix": mix,
                "sources": _near(rng, 1, 200), "shared": _near(rng, 1, 131072)}
    if kind == "append":
        new = _near(rng, 1, 32768 // requests)
        return {"kind": kind, "requests": requests, "heads": heads, "group": group, "block": block, "ctx": new + _near(rng, 1, 8192), "new": new,
                "mix": mix, "sources": rng.choice([0, sources]), "shared": _near(rng, 1, 131072), "rot": rng.choice([32, 64, 96, 128]),
                "pairs": rng.choice(["halves", "neighbours"])}
    # (query row, key) pairs are what the plain forms write out: no more of them than in the largest case
    room = 1.0e9 / (requests * heads * group)
    if kind == "cross":
        query = rng.choice([1, 1, _near(rng, 2, 500)])
        length = max(1, min(_near(rng, 1, 32768), int(room / query)))
        return {"kind": kind, "requests": requests, "heads": heads, "group": group, "block": block, "sources": sources, "shared": length, "query": query,
                "mix": int(query > 1 and mix), "out": rng.choice(["float32", "bfloat16"])}
    query = rng.choice([1, 1, 1, _near(rng, 2, 8), _near(rng, 16, 500)])
    ctx = query + _near(rng, 1, 2048)
    shared = max(1, min(_near(rng, 64, 65536), int(room / query) - ctx))
    query = max(1, min(query, int(room / (shared + ctx))))
    return {"kind": kind, "requests": requests, "heads": heads, "group": group, "block": block, "sources": sources, "shared": shared, "ctx": ctx,
            "query": query, "mix": int(query > 1 and mix), "window": rng.choice([0, 0, 0, max(1, (shared + ctx) // 3)]),
            "out": rng.choice(["float32", "bfloat16"])}


# ---------------------------------------------------------------------------------------------------------------- inputs
def _batch(case):
    """(source, cached, gain) of each row of the step, and the lengths of the rows that sources name: fixed by the case.  For `cross` these are
    rows of another table; else the sources are rows among the requests' own, which gain nothing."""
    r = random.Random(zlib.crc32(repr(sorted((k, v) for k, v in case.items() if k != "name")).encode()))
    n, m, kind = case["requests"], case["sources"], case["kind"]
    lengths = [case["shared"]] + [r.randint(max(1, case["shared"] // 2), case["shared"]) for _ in range(m - 1)] if m else []
    most = case.get("new", case.get("query"))
    if case["mix"]:  # chunks beside single tokens and requests that wait
        gain = [most] + [r.choice([1, 1, r.randint(0, most)]) for _ in range(n - 1)]
    else:
        gain = [most] * n if most <= 16 or kind == "append" else [most] + [r.randint(most // 2, most) for _ in range(n - 1)]
    # every source has a request, and where there are enough one in 16 requests has none
    named = [i if i < m else (r.randrange(m) if r.random() > 0.0625 else -1) for i in range(n)] if m else [-1] * n
    r.shuffle(named)
    if kind == "cross":
        return named, [0] * n, gain, lengths
    rows = n + m
    at = sorted(r.sample(range(rows), m))  # rows that are sources
    source, cached, new, i = [], [], [], 0
    for row in range(rows):
        if row in at:
            source.append(-1)
            cached.append(lengths[at.index(row)])
            new.append(0)
            continue
        source.append(at[named[i]] if named[i] >= 0 else -1)
        total = case["ctx"] if i == 0 else r.randint(1, case["ctx"])
        new.append(gain[i])
        cached.append(max(0, total - gain[i]))
        i += 1
    return source, cached, new, [c + g for c, g in zip(cached, new)]


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _starts(gain):
    start = [0]
    for g in gain:
        start.append(start[-1] + g)
    return start


def _pool(block, lengths, gen):
    """A pool with room to spare and the rows' block table, blocks in no order: (n_blocks, table)."""
    need = [-(-x // block) for x in lengths]
    n_blocks = sum(need) + 8
    ids = torch.randperm(n_blocks, generator=gen, device=DEV, dtype=torch.int32)
    place = torch.full((len(need), max(1, max(need))), -1, dtype=torch.int32)
    at = 0
    for s, k in enumerate(need):
        place[s, :k] = torch.arange(at, at + k, dtype=torch.int32)
        at += k
    place = place.to(DEV)
    return n_blocks, torch.where(place >= 0, ids[place.clamp(min=0).long()], -1).to(torch.int32)


def _filled(heads, block, n_blocks, gen):
    """A cache whose every slot holds a token: keys with a few strong channels, values N(0, 1)."""
    data = torch.empty((n_blocks, heads, block // TILE, TILE_BYTES), dtype=torch.uint8, device=DEV)
    channel = torch.exp(0.5 * torch.randn((heads, 1, 1, D), generator=gen, device=DEV))
    step = max(1, PART // (heads * block * D))
    for at in range(0, n_blocks, step):
        part = data[at: at + step]
        shape = (part.shape[0], heads, block // TILE, TILE, D)
        for side, scale in ((0, channel), (1, 1.0)):
            codes, scales = _encode(torch.randn(shape, generator=gen, device=DEV) * scale)
            part[..., 1024 * side: 1024 * side + 1024] = codes.reshape(*shape[:3], 1024)
            # token t = 4 i + g: the scales lie as [g][block of 32][i]
            part[..., 2048 + 64 * side: 2112 + 64 * side] = scales.reshape(*shape[:3], 4, 4, 4).permute(0, 1, 2, 4, 5, 3).reshape(*shape[:3], 64)
    return data


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    kind = case["kind"]
    source, cached, gain, lengths = _batch(case)
    start = _starts(gain)
    state = {"case": case, "source": _i32(source), "query_start": _i32(start), "n_tokens": start[-1]}
    if kind == "sources":
        state["seq_len"] = _i32(lengths)
        state["plan"] = torch.empty(2 * len(source) + 2 + 2 * start[-1], dtype=torch.int32, device=DEV)
        # (requests share other sources from step to step)
        named = torch.tensor(sorted({s for s in source if s >= 0}), device=DEV)
        state["source"] = torch.where(state["source"] >= 0, named[torch.randint(len(named), (len(source),), generator=gen, device=DEV)], -1).to(torch.int32)
        return state
    heads, group, block = case["heads"], case["group"], case["block"]
    if kind == "append":
        # the sources' own blocks are not looked at, only how many tokens they have
        n_blocks, table = _pool(block, [c + g if g else 0 for c, g in zip(cached, gain)], gen)
        width = (2 + group) * heads * D  # a fused projection holds the queries beside the keys and values
        x = torch.randn((start[-1], width), generator=gen, device=DEV)
        x *= torch.exp(0.5 * torch.randn((width,), generator=gen, device=DEV))
        x = x.to(torch.bfloat16)
        edge = [0, group * heads * D, (group + 1) * heads * D, width]
        state["q"], state["k"], state["v"] = (x[:, a:b].unflatten(1, ((b - a) // D, D)) for a, b in zip(edge, edge[1:]))
        far = max(lengths[s] for s in source if s >= 0) if max(source) >= 0 else 0
        half = case["rot"] // 2
        angle = torch.arange(far + case["ctx"] + max(gain), device=DEV, dtype=torch.float64)[:, None]
        angle = angle * torch.exp(torch.arange(half, device=DEV, dtype=torch.float64) * (-math.log(500000.0) / half))
        state["rope"] = torch.cat([torch.cos(angle), torch.sin(angle)], 1).float()
        state["data"] = torch.zeros((n_blocks, heads, block // TILE, TILE_BYTES), dtype=torch.uint8, device=DEV)
        state.update(table=table, first=_i32(cached), seq_len=_i32(lengths), most=max(gain))
        return state
    n_blocks, table = _pool(block, lengths, gen)
    state["q"] = torch.randn((start[-1], heads * group, D), generator=gen, device=DEV).to(torch.bfloat16)
    state.update(data=_filled(heads, block, n_blocks, gen), table=table, seq_len=_i32(lengths), max_query=max(gain), host=(source, start, lengths))
    # the queries sorted by source: a step does that once, and its layers read it
    state["plan"] = _sorted_queries(state["source"], state["query_start"], state["seq_len"] if kind == "shared" else None, len(lengths), start[-1])
    rows = [s for s, g in zip(source, gain) for _ in range(g)]
    state["max_shared"] = max([rows.count(s) for s in set(rows) if s >= 0] or [1])
    state["max_len"] = max([x for x, g in zip(lengths, gain) if g] if kind == "shared" else lengths)
    state["max_source"] = max([lengths[s] for s in set(rows) if s >= 0] or [1])
    return state


# ----------------------------------------------------------------------------------------------------------- plain forms
def _encode(x):
    """Codes [..., 64] and scale bytes [..., 4] of float32 rows x [..., 128]."""
    x = x.unflatten(-1, (4, 32))
    bits = x.abs().amax(-1).view(torch.int32)
    exponent = bits >> 23
    lost = ~torch.isfinite(x).all(-1)
    scale = (exponent - 2 + ((bits & 0x7FFFFF) > 0x600000)).clamp(27, 252)
    m = torch.ldexp(x.abs(), (127 - scale)[..., None])
    code = (m > 0.25).to(torch.uint8)
    code += m >= 0.75
    code += m > 1.25
    code += m >= 1.75
    code += m > 2.5
    code += m >= 3.5
    code += m > 5
    code += torch.signbit(x) * 8
    scale = torch.where(lost, 255, scale).to(torch.uint8)
    code = torch.where(lost[..., None], 0, code).flatten(-2).unflatten(-1, (64, 2))
    return code[..., 0] | code[..., 1] << 4, scale


def _decode(codes, scales):
    """Float32 rows [..., 128] of codes [..., 64] and scale bytes [..., 4]."""
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    m = (c & 7).to(torch.int32)
    e = m >> 1
    value = torch.where(e > 0, torch.ldexp(1.0 + 0.5 * (m & 1), e - 1), 0.5 * m)
    value = torch.where(c > 7, -value, value).unflatten(-1, (4, 32))
    s = scales.to(torch.int32)
    s = torch.where(s == 255, float("nan"), torch.ldexp(torch.ones_like(s, dtype=torch.float32), s - 127))
    return (value * s[..., None]).flatten(-2)


def _rows(data, block_id, place, head):
    """Keys and values, float32 [..., 128] each, at `place` of block `block_id` of KV head `head` (index tensors that broadcast)."""
    tile, t = place // TILE, place % TILE
    at = 16 * (t % 4) + t // 4
    four = torch.arange(4, device=data.device) * 4
    index = (block_id, head, tile)
    both = []
    for side in (0, 1):
        codes = data[..., 1024 * side: 1024 * side + 1024].unflatten(-1, (16, 64))[(*index, t)]
        scales = data[..., 2048 + 64 * side: 2112 + 64 * side][tuple(i[..., None] for i in index) + (at[..., None] + four,)]
        both.append(_decode(codes, scales))
    return both


def _owners(start, n_tokens):
    token = torch.arange(n_tokens, device=DEV)
    owner = torch.searchsorted(start[1:].contiguous(), token, right=True)
    return token, owner


def _sorted_queries(source, query_start, seq_len, n_rows, n_tokens):
    start = query_start.long()
    token, owner = _owners(start, n_tokens)
    n = source.numel()
    to = source.long()
    none = (to < 0) | (to >= n_rows)
    if seq_len is not None:
        none |= to == torch.arange(n, device=DEV)
    to = torch.where(none, n_rows, to)
    row, order = torch.sort(to[owner], stable=True)
    begin = torch.searchsorted(row, torch.arange(n_rows + 2, device=DEV))
    place = torch.zeros_like(token)
    least = torch.full((n_rows + 1,), NONE, dtype=torch.int64, device=DEV)
    many = start[1:] - start[:-1]
    if seq_len is not None:
        place = seq_len.long()[owner] - many[owner] + token - start[owner]
        at = seq_len.long() - many
    else:
        at = torch.zeros_like(many)
    least = least.scatter_reduce(0, to, torch.where(many > 0, at, NONE), "amin")
    return torch.cat([begin, least[:n_rows], order, place[order]]).int()


def _rotate(x, cos, sin, pairs):
    half = cos.shape[-1]
    turned = x[..., : 2 * half]
    a, b = (turned[..., :half], turned[..., half:]) if pairs == "halves" else (turned[..., 0::2], turned[..., 1::2])
    a, b = a * cos - b * sin, a * sin + b * cos
    both = torch.cat([a, b], -1) if pairs == "halves" else torch.stack([a, b], -1).flatten(-2)
    return torch.cat([both, x[..., 2 * half:]], -1)


def _plain_append(s):
    case = s["case"]
    block, heads, data = case["block"], case["heads"], s["data"]
    start, seq_len, source = s["query_start"].long(), s["seq_len"].long(), s["source"].long()
    token, owner = _owners(start, s["n_tokens"])
    place = seq_len[owner] - start[owner + 1] + token
    position = place + torch.where(source >= 0, seq_len[source.clamp(min=0)], 0)[owner]
    cos, sin = s["rope"][position].unsqueeze(1).chunk(2, -1)
    q, k = (_rotate(x.float(), cos, sin, case["pairs"]) for x in (s["q"], s["k"]))
    head = torch.arange(heads, device=DEV)
    b, t = s["table"].long()[owner, place // block][:, None], (place % block)[:, None]
    tile, t = t // TILE, t % TILE
    at = (16 * (t % 4) + t // 4)[..., None] + 4 * torch.arange(4, device=DEV)
    for side, x in ((0, k), (1, s["v"].float())):
        codes, scales = _encode(x)
        data[..., 1024 * side: 1024 * side + 1024].unflatten(-1, (16, 64))[b, head, tile, t] = codes
        data[..., 2048 + 64 * side: 2112 + 64 * side][b[..., None], head[:, None], tile[..., None], at] = scales
    # back, request by request from its first new token on; 0 behind the last one
    pos = s["first"].long()[:, None] + torch.arange(s["most"], device=DEV)
    there = (pos < seq_len[:, None])[:, None, :, None]
    b = torch.gather(s["table"].long(), 1, (pos // block).clamp(max=s["table"].shape[1] - 1)).clamp(min=0)[:, None]
    k, v = _rows(data, b, (pos % block)[:, None], head[None, :, None])
    return q.to(torch.bfloat16), torch.where(there, k, 0.0).to(torch.bfloat16), torch.where(there, v, 0.0).to(torch.bfloat16)


def _row_keys(s, row, length):
    case = s["case"]
    pos = torch.arange(length, device=DEV)
    return _rows(s["data"], s["table"].long()[row, pos // case["block"]][None], (pos % case["block"])[None], torch.arange(case["heads"], device=DEV)[:, None])


def _softmax_rows(q, k, v, seen):
    """Rows q [heads, rows, 128]: (softmax over the seen keys) @ values, and the logarithm of the softmax's sum."""
    scores = torch.where(seen, torch.matmul(q, k.transpose(-1, -2)) / math.sqrt(D), float("-inf"))
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - top)
    total = p.sum(-1, keepdim=True)
    return torch.matmul(p, v) / total, (top + torch.log(total)).squeeze(-1)


def _plain_attend(s):
    case = s["case"]
    heads, group, window = case["heads"], case["group"], case.get("window", 0)
    source, start, lengths = s["host"]
    out = torch.zeros(s["q"].shape, dtype=torch.float32, device=DEV)
    lse = torch.full(s["q"].shape[:2], float("-inf"), device=DEV)
    common = {r: _row_keys(s, r, lengths[r]) for r in set(source) if r >= 0}
    for i, r in enumerate(source):
        n = start[i + 1] - start[i]
        parts = [common[r]] if r >= 0 else []
        if case["kind"] == "shared":
            parts.append(_row_keys(s, i, lengths[i]))
        if n == 0 or not parts:
            continue
        k, v = (torch.cat([p[side] for p in parts], 1) for side in (0, 1))
        q = s["q"][start[i]: start[i + 1]].float().unflatten(1, (heads, group)).permute(1, 0, 2, 3).flatten(1, 2)
        seen = torch.ones((1, 1), dtype=torch.bool, device=DEV)
        if case["kind"] == "shared":
            at, key = (k.shape[1] - n + torch.arange(n, device=DEV))[:, None], torch.arange(k.shape[1], device=DEV)
            seen = key <= at
            if window:
                seen &= key > at - window
            seen = seen.repeat_interleave(group, 0)
        o, z = _softmax_rows(q, k, v, seen)
        out[start[i]: start[i + 1]] = o.unflatten(1, (n, group)).permute(1, 0, 2, 3).flatten(1, 2)
        lse[start[i]: start[i + 1]] = z.unflatten(1, (n, group)).permute(1, 0, 2).flatten(1, 2)
    return out.to(getattr(torch, case["out"])), lse


def _own_run(s):
    from paper_2604_10539_amd import IceCache, ice_plan_sources
    case = s["case"]
    if case["kind"] == "sources":
        ice_plan_sources(s["source"], s["query_start"], s["seq_len"], s["plan"], s["seq_len"].numel(), s["n_tokens"])
        return s["plan"]
    cache = s.get("cache")
    if cache is None:  # the handle that a program keeps: it holds the tensor and its sizes
        cache = s["cache"] = IceCache(s["data"].shape[0], case["heads"], case["block"], data=s["data"])
    if case["kind"] == "append":
        q = cache.append(s["k"], s["v"], s["query_start"], s["seq_len"], s["table"], q=s["q"], rope=s["rope"], neighbours=case["pairs"] == "neighbours",
                         source=s["source"] if case["sources"] else None)
        return q, *cache.read(s["table"], s["seq_len"], s["most"], first=s["first"])
    dtype = getattr(torch, case["out"])
    if case["kind"] == "cross":
        return cache.attend_cross(s["q"], s["plan"], s["seq_len"], s["table"], max_shared=s["max_shared"], max_len=s["max_len"], out_dtype=dtype, with_lse=True)
    return cache.attend_shared(s["q"], s["query_start"], s["source"], s["plan"], s["seq_len"], s["table"], max_query=s["max_query"], max_shared=s["max_shared"],
                               max_len=s["max_len"], max_source=s["max_source"], window=case["window"], out_dtype=dtype, with_lse=True)


def run(state):
    if own:
        return _own_run(state)
    kind = state["case"]["kind"]
    if kind == "sources":
        return _sorted_queries(state["source"], state["query_start"], state["seq_len"], state["seq_len"].numel(), state["n_tokens"])
    return _plain_append(state) if kind == "append" else _plain_attend(state)


def work(case):
    source, cached, gain, lengths = _batch(case)
    kind, total, rows = case["kind"], sum(gain), len(source)
    if kind == "sources":
        return {"bytes": 4.0 * (3 * rows + 1 + 2 * rows + 2 + 2 * total), "flops": 0.0}
    heads, group, window = case["heads"], case["group"], case.get("window", 0)
    if kind == "append":  # rows in, queries out, codes out and in again, values out; a row of cos and sin for each token
        read_back = len(gain) * max(gain) * heads * 512.0
        return {"bytes": total * heads * (256.0 * (2 + 2 * group) + 2 * ROW_BYTES) + total * 4.0 * case["rot"] + read_back, "flops": 0.0}
    io = total * heads * group * (D * (2.0 + (4 if case["out"] == "float32" else 2)) + 4)
    keys, pairs, reach = 0, 0, {}  # reach: how many of a source's last tokens are read
    for r, c, g, n in zip(source, cached, gain, lengths if kind == "shared" else [0] * rows):
        if g == 0:
            continue
        p = lengths[r] if r >= 0 else 0
        if r >= 0:
            reach[r] = max(reach.get(r, 0), min(p, max(0, window - 1 - c)) if window else p)
        if kind == "cross":
            pairs += g * p
            continue
        keys += min(n, window + g - 1) if window else n
        pairs += sum(min(p + c + j + 1, window) if window else p + c + j + 1 for j in range(g))
    keys += sum(reach.values())
    return {"bytes": keys * heads * float(ROW_BYTES) + io, "flops": 4.0 * D * pairs * heads * group}


# ------------------------------------------------------------------------------------------------- 64 bits, written apart
_LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_held(x):
    """Float64 values that rows x [..., 128] are held as: the nearest level by distance, the even code on ties."""
    levels = torch.tensor(_LEVELS, dtype=torch.float64, device=DEV)
    even = torch.tensor([0.0, 1e-9] * 4, dtype=torch.float64, device=DEV)  # (a tie's two distances are equal; any others differ by far more than this)
    parts = []
    for y in torch.split(x.double().reshape(-1, 32), PART // 256):
        top = y.abs().amax(1, keepdim=True)
        _, e = torch.frexp(top)  # top = f * 2^e, f in [0.5, 1)
        e = e - 1
        e = torch.where(top > 1.75 * torch.exp2(e.double()), e + 1, e) - 2
        scale = torch.exp2(torch.where(top > 0, e, -100).clamp(-100, 125).double())
        best = ((y.abs() / scale)[..., None] - levels).abs().add(even).argmin(-1)
        held = levels[best] * scale * torch.sign(y)
        parts.append(torch.where(torch.isfinite(y).all(1, keepdim=True), held, float("nan")))
    return torch.cat(parts).reshape(x.shape)


def _exact_keys(data, blocks, length, block, heads):
    """Float64 keys and values [heads, length, 128] of the first tokens of a row of the table, byte by byte through tables."""
    low = torch.tensor([(_LEVELS[c & 7] if c & 15 < 8 else -_LEVELS[c & 7]) for c in range(256)], dtype=torch.float64, device=DEV)
    high = torch.tensor([(_LEVELS[c >> 4 & 7] if c >> 4 < 8 else -_LEVELS[c >> 4 & 7]) for c in range(256)], dtype=torch.float64, device=DEV)
    power = torch.tensor([2.0 ** (b - 127) for b in range(255)] + [float("nan")], dtype=torch.float64, device=DEV)
    pos = torch.arange(length, device=DEV)
    base = (blocks.long()[pos // block] * heads * (block // TILE) + pos % block // TILE) * TILE_BYTES
    base = base[None, :] + torch.arange(heads, device=DEV)[:, None] * (block // TILE) * TILE_BYTES
    flat, t, dim = data.reshape(-1), pos % TILE, torch.arange(D, device=DEV)
    both = []
    for side in (0, 1):
        byte = flat[base[..., None] + 1024 * side + (64 * t)[:, None] + dim // 2].long()
        scale = flat[base[..., None] + 2048 + 64 * side + (16 * (t % 4) + t // 4)[:, None] + 4 * (dim // 32)].long()
        both.append(torch.where(dim % 2 == 0, low[byte], high[byte]) * power[scale])
    return both


def exact(case, seed):
    kind = case["kind"]
    if kind == "sources":
        return None
    s = prepare(case, seed)
    source, cached, gain, lengths = _batch(case)
    start = _starts(gain)
    heads, group, block = case["heads"], case["group"], case["block"]
    if kind == "append":
        # the held keys have no such value: one next to a border goes to the other side of it by the last bit of a rotation
        half, q = case["rot"] // 2, s["q"].double()
        values = torch.zeros((len(gain), heads, max(gain), D), dtype=torch.float64, device=DEV)
        for i, n in enumerate(gain):
            rows = slice(start[i], start[i + 1])
            base = cached[i] + (lengths[source[i]] if source[i] >= 0 else 0)
            turn = s["rope"][base: base + n].double()
            z = torch.complex(turn[:, :half], turn[:, half:])[:, None]
            x = q[rows, :, : 2 * half]
            if case["pairs"] == "halves":
                y = torch.complex(x[..., :half].contiguous(), x[..., half:].contiguous()) * z
                q[rows, :, : 2 * half] = torch.cat([y.real, y.imag], -1)
            else:
                q[rows, :, : 2 * half] = torch.view_as_real(torch.view_as_complex(x.unflatten(-1, (half, 2)).contiguous()) * z).flatten(-2)
            values[i, :, :n] = _exact_held(s["v"][rows]).transpose(0, 1)
        return q, None, values
    q, window = s["q"].double(), case.get("window", 0)
    out, lse = torch.zeros_like(q), torch.full(q.shape[:2], float("-inf"), dtype=torch.float64, device=DEV)
    held = {}
    for i, n in enumerate(gain):
        names = ([source[i]] if source[i] >= 0 else []) + ([i] if kind == "shared" else [])
        if n == 0 or not names:
            continue
        for r in names:
            if r not in held:
                held[r] = _exact_keys(s["data"], s["table"][r], lengths[r], block, heads)
        k, v = (torch.cat([held[r][side] for r in names], 1) for side in (0, 1))
        if kind == "shared":
            del held[i]
        step = max(1, PART * 8 // (heads * group * k.shape[1]))
        for j in range(0, n, step):
            m = min(step, n - j)
            rows = slice(start[i] + j, start[i] + j + m)
            x = q[rows].reshape(m, heads, group, D).permute(1, 0, 2, 3).reshape(heads, m * group, D)
            x = torch.bmm(x, k.transpose(1, 2).contiguous()) * (1.0 / math.sqrt(128.0))
            if kind == "shared":
                back = (k.shape[1] - n + j + torch.arange(m, device=DEV)).repeat_interleave(group)[:, None] - torch.arange(k.shape[1], device=DEV)
                x.masked_fill_((back < 0) | (back >= (window or NONE)), float("-inf"))
            z = torch.logsumexp(x, -1)
            x.sub_(z[..., None]).exp_()
            out[rows] = torch.bmm(x, v).reshape(heads, m, group, D).permute(1, 0, 2, 3).reshape(m, heads * group, D)
            lse[rows] = z.reshape(heads, m, group).permute(1, 0, 2).reshape(m, heads * group)
    return out, lse
