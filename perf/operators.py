"""A KV cache held in 4 bits and the attention that reads it, as callable cases.

Five operators, in the order in which a serving step uses them:

  plan     block tables, lengths and slots of a step, from how many tokens each request gains or gives back
  write    keys and values of the step's tokens go into the cache as 4-bit codes with a scale per 32 values
  read     rows of the cache as bf16, in the layout that an index is built from
  attend   causal attention of the step's queries over their requests' cached tokens: single tokens, drafts, prompts
  tokens   attention of one query per request over listed positions: a layer that reuses another layer's selection

Held values.  A row of 128 values is four blocks of 32.  A block has one scale 2^(b - 127), b a byte, and its values are
x = scale * c with c of +-{0, 0.5, 1, 1.5, 2, 3, 4, 6}.  With e = floor(log2(max |x|)) the scale is 2^(e - 2), twice
that where max |x| > 1.75 * 2^e (the largest value then rounds to 4 of the larger scale and not down to 6), and never below 2^-100
or above 2^125; c is the nearest of the sixteen to x / scale, to the even code on a tie.  A block with a value that
is not finite is held as NaN (b = 255).

Layout.  The cache is [block][KV head][tile of 16 tokens][2176 bytes]: 1024 bytes of key codes (64 per token, dimension 2i in
the low half of byte i), 1024 of value codes, 64 of key scales, 64 of value scales; the scale of token t's block j is
at byte 16 (t mod 4) + 4 j + t / 4.  Token p of request s sits in block table[s][p / block], at p mod block; a slot is
block id * block + place in the block.
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
PART = 1 << 26  # values that the input makers and exact() touch at a time


def listed():
    return [
        # one decode step of a small batch: every request gains a token, a new block now and then
        {"name": "plan_step_16", "kind": "plan", "requests": 16, "block": 64, "ctx": 32768, "new": 1, "mix": 0},
        # a busy server's step: most requests gain a token, some start with a prompt, some end, some drop rejected drafts
        {"name": "plan_mixed_1000", "kind": "plan", "requests": 1000, "block": 16, "ctx": 32768, "new": 4096, "mix": 1},
        # the keys and values of one decode step of a batch, out of the fused projection's output
        {"name": "store_step_16", "kind": "store", "requests": 16, "heads": 8, "block": 64, "ctx": 32768, "new": 1, "fused": 1},
        # a prompt of 32k tokens goes into the cache and comes back for the index that is built over it
        {"name": "store_prompt_32k", "kind": "store", "requests": 1, "heads": 8, "block": 64, "ctx": 32768, "new": 32768, "fused": 0},
        # the smallest attention: one token of a short chat, two KV heads on this GPU
        {"name": "attend_1x4k", "kind": "attend", "requests": 1, "heads": 2, "group": 4, "block": 16, "ctx": 4097, "query": 1, "mix": 0,
         "window": 0, "out": "float32"},
        # a batch's decode step over ragged contexts up to 32k
        {"name": "attend_16x32k", "kind": "attend", "requests": 16, "heads": 8, "group": 4, "block": 64, "ctx": 32768, "query": 1, "mix": 0,
         "window": 0, "out": "float32"},
        # one token of one long document
        {"name": "attend_1x131k", "kind": "attend", "requests": 1, "heads": 8, "group": 4, "block": 64, "ctx": 131072, "query": 1, "mix": 0,
         "window": 0, "out": "float32"},
        # five drafted tokens per request are checked, with a sliding window and 64 query heads
        {"name": "attend_draft_32x8k", "kind": "attend", "requests": 32, "heads": 8, "group": 8, "block": 32, "ctx": 8192, "query": 5, "mix": 0,
         "window": 4096, "out": "bfloat16"},
        # two prompts in chunks of up to 2048 tokens behind up to 30k cached ones
        {"name": "attend_chunk_2x32k", "kind": "attend", "requests": 2, "heads": 8, "group": 4, "block": 64, "ctx": 32768, "query": 2048,
         "mix": 0, "window": 0, "out": "bfloat16"},
        # a mixed step: chunks of prompts beside single tokens, float32 for a layer whose outputs are merged with an index's
        {"name": "attend_mixed_24x8k", "kind": "attend", "requests": 24, "heads": 4, "group": 4, "block": 16, "ctx": 8192, "query": 500,
         "mix": 1, "window": 0, "out": "float32"},
        # a batch's layer that reuses its anchor layer's selections of 1024 tokens
        {"name": "tokens_16x1024", "kind": "tokens", "requests": 16, "heads": 8, "group": 4, "block": 16, "ctx": 32768, "tokens": 1024},
        # the same at the benchmark's budget of 256 tokens, one request: latency
        {"name": "tokens_1x256", "kind": "tokens", "requests": 1, "heads": 8, "group": 4, "block": 64, "ctx": 32768, "tokens": 256},
    ]


def _near(rng, low, high):
    """A whole number between the two, spread over the logarithm."""
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    kind = rng.choice(["plan", "store", "attend", "attend", "attend", "tokens", "tokens"])
    block = rng.choice([16, 32, 64])
    heads = rng.choice([1, 2, 4, 5, 8])
    if kind == "plan":
        mix = rng.choice([0, 1])
        return {"kind": kind, "requests": _near(rng, 1, 2000), "block": block, "ctx": _near(rng, 16, 32768), "new": _near(rng, 1, 4096) if mix else 1,
                "mix": mix}
    if kind == "store":
        requests = _near(rng, 1, 64)
        new = _near(rng, 1, 32768 // requests)
        return {"kind": kind, "requests": requests, "heads": heads, "block": block, "ctx": new + _near(rng, 1, 8192), "new": new,
                "fused": rng.choice([0, 1])}
    requests = _near(rng, 1, 32)
    ctx = _near(rng, 1, min(131072, (1 << 22) // (requests * heads)))
    if kind == "tokens":
        return {"kind": kind, "requests": requests, "heads": heads, "group": rng.choice([1, 2, 4, 7, 8]), "block": block, "ctx": ctx,
                "tokens": _near(rng, 1, 2048)}
    group = rng.choice([1, 2, 4, 5, 8, 16])
    query = min(ctx, rng.choice([1, 1, 1, _near(rng, 2, 8), _near(rng, 16, 2048)]))
    # no more (query row, key) pairs than the largest case: they are what the plain form writes out
    query = max(1, min(query, int(1.5e9 / (requests * heads * group * ctx))))
    return {"kind": kind, "requests": requests, "heads": heads, "group": group, "block": block, "ctx": ctx, "query": query,
            "mix": int(query > 1 and rng.random() < 0.5), "window": rng.choice([0, 0, 0, max(1, ctx // 3)]), "out": rng.choice(["float32", "bfloat16"])}


# ---------------------------------------------------------------------------------------------------------------- inputs
def _lengths(case):
    """(cached tokens before the step, tokens the step brings) per request: fixed by the case."""
    r = random.Random(zlib.crc32(repr(sorted((k, v) for k, v in case.items() if k != "name")).encode()))
    n, kind = case["requests"], case["kind"]
    if kind == "plan":
        cached = [r.randint(0, case["ctx"]) for _ in range(n)]
        gain = [1] * n
        for i in range(n if case["mix"] else 0):
            x = r.random()
            if x < 0.05:  # a request that starts
                cached[i], gain[i] = 0, r.randint(1, case["new"])
            elif x < 0.10:  # one that ends
                gain[i] = -cached[i]
            elif x < 0.15:  # one whose last drafted tokens were rejected
                gain[i] = -min(cached[i], r.randint(1, 4))
        return cached, gain
    if kind == "store":
        gain = [case["new"]] * n
        return [r.randint(0, case["ctx"] - case["new"]) for _ in range(n)], gain
    total = [case["ctx"]] + [r.randint(max(1, case["ctx"] // 4), case["ctx"]) for _ in range(n - 1)]
    if kind == "tokens":
        return [t - 1 for t in total], [1] * n
    if case["mix"]:  # chunks of prompts beside single tokens, and a request that waits
        gain = [case["query"]] + [r.choice([1, 1, 1, r.randint(0, case["query"])]) for _ in range(n - 1)]
    else:
        gain = [case["query"]] * n if case["query"] <= 16 else [case["query"]] + [r.randint(case["query"] // 2, case["query"]) for _ in range(n - 1)]
    gain = [min(g, t) for g, t in zip(gain, total)]
    return [t - g for t, g in zip(total, gain)], gain


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _pool(case, lengths, gen):
    """A pool with room to spare and the requests' block tables, blocks in no order: (n_blocks, table, ids not in use)."""
    block = case["block"]
    need = [-(-x // block) for x in lengths]
    n_blocks = sum(need) + 8
    ids = torch.randperm(n_blocks, generator=gen, device=DEV, dtype=torch.int32)
    width = max(1, -(-max(case["ctx"], max(lengths)) // block))
    place = torch.full((len(need), width), -1, dtype=torch.int32)
    at = 0
    for s, k in enumerate(need):
        place[s, :k] = torch.arange(at, at + k, dtype=torch.int32)
        at += k
    place = place.to(DEV)
    table = torch.where(place >= 0, ids[place.clamp(min=0).long()], -1).to(torch.int32)
    return n_blocks, table, ids[at:].contiguous()


def _filled(case, n_blocks, gen):
    """A cache whose every slot holds a token: keys with a few strong channels, values N(0, 1)."""
    heads, tiles = case["heads"], case["block"] // TILE
    data = torch.empty((n_blocks, heads, tiles, TILE_BYTES), dtype=torch.uint8, device=DEV)
    channel = torch.exp(0.5 * torch.randn((heads, 1, 1, D), generator=gen, device=DEV))
    step = max(1, PART // (heads * case["block"] * D))
    for at in range(0, n_blocks, step):
        part = data[at: at + step]
        shape = (part.shape[0], heads, tiles, TILE, D)
        for side, scale in ((0, channel), (1, 1.0)):
            codes, scales = _encode((torch.randn(shape, generator=gen, device=DEV) * scale).to(torch.bfloat16))
            part[..., 1024 * side: 1024 * side + 1024] = codes.reshape(*shape[:3], 1024)
            # token t = 4 i + g: the scales lie as [g][block of 32][i]
            part[..., 2048 + 64 * side: 2112 + 64 * side] = scales.reshape(*shape[:3], 4, 4, 4).permute(0, 1, 2, 4, 5, 3).reshape(*shape[:3], 64)
    return data


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    kind, block = case["kind"], case["block"]
    cached, gain = _lengths(case)
    after = [c + g for c, g in zip(cached, gain)]
    if kind == "plan":
        n_blocks, table, spare = _pool(case, [max(c, a) for c, a in zip(cached, after)], gen)
        # the blocks that the step needs are still free: they lie on the stack, mixed with the spare ones
        held = [-(-c // block) for c in cached]
        new = [max(0, -(-a // block) - h) for a, h in zip(after, held)]
        column = torch.arange(table.shape[1], device=DEV, dtype=torch.int32)
        fresh = (column >= _i32(held)[:, None]) & (column < _i32([h + k for h, k in zip(held, new)])[:, None])
        free = torch.cat([spare, table[fresh]])
        free = free[torch.randperm(free.numel(), generator=gen, device=DEV)]
        table = torch.where(fresh, -1, table).to(torch.int32)
        free_ids = torch.full((n_blocks,), -1, dtype=torch.int32, device=DEV)
        free_ids[: free.numel()] = free
        n = case["requests"]
        slots = -(-max(1, sum(g for g in gain if g > 0)) // 256) * 256  # a step's arrays are padded to a multiple of 256 tokens
        e = lambda *shape: torch.empty(shape, dtype=torch.int32, device=DEV)  # noqa: E731
        return {"case": case, "n_blocks": n_blocks, "gain": _i32(gain), "cached": _i32(cached), "table": table, "free_ids": free_ids,
                "n_free": _i32([free.numel()]), "seq_len": e(n), "n_free_left": e(1), "query_start": e(n + 1), "slots": e(slots), "info": e(4)}
    if kind == "store":
        n, heads, new = case["requests"], case["heads"], case["new"]
        n_blocks, table, _ = _pool(case, after, gen)
        pos = _i32(cached)[:, None] + torch.arange(new, dtype=torch.int32, device=DEV)
        slots = torch.gather(table, 1, (pos // block).long()) * block + pos % block
        width = (2 + 4 * case["fused"]) * heads * D  # a fused projection holds the queries beside the keys and values
        x = torch.randn((n * new, width), generator=gen, device=DEV)
        x *= torch.exp(0.5 * torch.randn((width,), generator=gen, device=DEV))
        x = x.to(torch.bfloat16)
        k, v = (x[:, width - (2 - i) * heads * D: width - (1 - i) * heads * D].unflatten(1, (heads, D)) for i in (0, 1))
        data = torch.zeros((n_blocks, heads, block // TILE, TILE_BYTES), dtype=torch.uint8, device=DEV)
        return {"case": case, "data": data, "k": k, "v": v, "slots": slots.reshape(-1).contiguous(), "table": table, "first": _i32(cached),
                "seq_len": _i32(after)}
    n_blocks, table, _ = _pool(case, after, gen)
    total = sum(gain)
    q = torch.randn((total, case["heads"] * case["group"], D), generator=gen, device=DEV).to(torch.bfloat16)
    state = {"case": case, "data": _filled(case, n_blocks, gen), "table": table, "seq_len": _i32(after), "q": q}
    if kind == "tokens":
        # a selection: every KV head has positions of its own, some heads fewer than the others
        n, heads, most = case["requests"], case["heads"], case["tokens"]
        pos = torch.rand((n, heads, most), generator=gen, device=DEV)
        pos = (pos * state["seq_len"][:, None, None]).floor().to(torch.int32)
        state["pos"] = torch.minimum(pos, state["seq_len"][:, None, None] - 1)
        less = torch.rand((n, heads), generator=gen, device=DEV)
        state["n_tok"] = torch.where(less < 0.25, (less * 4 * most).floor(), float(most)).to(torch.int32)
    else:
        start = [0]
        for g in gain:
            start.append(start[-1] + g)
        state["query_start"], state["max_query"], state["max_len"] = _i32(start), max(gain), max(after)
    return state


# ----------------------------------------------------------------------------------------------------------- plain forms
def _encode(x):
    """Codes [..., 64] and scale bytes [..., 4] of rows x [..., 128]."""
    x = x.float().unflatten(-1, (4, 32))
    bits = x.abs().amax(-1).view(torch.int32)
    exponent = bits >> 23
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
    lost = exponent == 255
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


def _softmax_rows(scores, seen, values):
    """(softmax over the seen keys) @ values, and the logarithm of the softmax's sum; 0 and -inf where nothing is seen."""
    scores = torch.where(seen, scores, float("-inf"))
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(seen.any(-1, keepdim=True), top, 0.0))
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, values) / torch.where(seen.any(-1, keepdim=True), total, 1.0)
    return out, (top + torch.log(total)).squeeze(-1)


def _plain_plan(s):
    block, gain, cached, table = s["case"]["block"], s["gain"].long(), s["cached"].long(), s["table"].clone()
    n, width, free_ids = cached.numel(), table.shape[1], s["free_ids"].clone()
    after = (cached + gain).clamp(min=0)
    held, need = (cached + block - 1) // block, (after + block - 1) // block
    column = torch.arange(width, device=DEV)
    # blocks given back go on the stack, request by request
    back = (held - need).clamp(min=0)
    gone = (column >= need[:, None]) & (column < held[:, None])
    back_at = torch.where(gone, s["n_free"] + (torch.cumsum(back, 0) - back)[:, None] + column - need[:, None], s["n_blocks"])
    free_ids = torch.cat([free_ids, free_ids[:1]]).scatter(0, back_at.flatten(), table.flatten())[: s["n_blocks"]]
    n_free = s["n_free"].long() + back.sum()
    # blocks taken come off its end, in the same order
    take = (need - held).clamp(min=0)
    fresh = (column >= held[:, None]) & (column < need[:, None])
    order = (torch.cumsum(take, 0) - take)[:, None] + column - held[:, None]
    table = torch.where(fresh, free_ids[(n_free - 1 - order).clamp(0, s["n_blocks"] - 1)], table)
    left = n_free - take.sum()
    new = gain.clamp(min=0)
    start = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), torch.cumsum(new, 0)])
    token = torch.arange(s["slots"].numel(), device=DEV)
    owner = torch.searchsorted(start[1:], token, right=True).clamp(max=n - 1)
    pos = (cached[owner] + token - start[owner]).clamp(0, width * block - 1)
    slots = torch.where(token < start[-1], table[owner, pos // block].long() * block + pos % block, -1)
    info = torch.stack([start[-1], take.sum(), back.sum(), torch.zeros_like(start[-1])])
    return after.int(), table, free_ids, left.int(), start.int(), slots.int(), info.int()


def _plain_store(s):
    block, heads, data, slots = s["case"]["block"], s["case"]["heads"], s["data"], s["slots"].long()
    head = torch.arange(heads, device=DEV)
    b, t = (slots // block)[:, None], (slots % block)[:, None]
    tile, t = t // TILE, t % TILE
    at = (16 * (t % 4) + t // 4)[..., None] + 4 * torch.arange(4, device=DEV)
    for side, x in ((0, s["k"]), (1, s["v"])):
        codes, scales = _encode(x)
        data[..., 1024 * side: 1024 * side + 1024].unflatten(-1, (16, 64))[b, head, tile, t] = codes
        data[..., 2048 + 64 * side: 2112 + 64 * side][b[..., None], head[:, None], tile[..., None], at] = scales
    pos = s["first"].long()[:, None] + torch.arange(s["case"]["new"], device=DEV)
    b = torch.gather(s["table"].long(), 1, pos // block)[:, None]
    k, v = _rows(data, b, (pos % block)[:, None], head[None, :, None])
    return k.to(torch.bfloat16), v.to(torch.bfloat16)


def _plain_attend(s):
    case = s["case"]
    block, heads, group, length, most = case["block"], case["heads"], case["group"], s["max_len"], s["max_query"]
    n, total = case["requests"], s["q"].shape[0]
    pos = torch.arange(length, device=DEV)
    b = s["table"].long()[:, pos // block].clamp(min=0)[:, None]
    k, v = _rows(s["data"], b, (pos % block)[None, None], torch.arange(heads, device=DEV)[None, :, None])
    start, seq_len = s["query_start"].long(), s["seq_len"].long()
    j = torch.arange(most, device=DEV)
    row = (start[:-1, None] + j).clamp(max=max(total - 1, 0))  # [n, most]
    q = s["q"].float()[row].unflatten(2, (heads, group)).permute(0, 2, 1, 3, 4).flatten(2, 3)  # [n, heads, most * group, D]
    query_pos = seq_len[:, None] - (start[1:] - start[:-1])[:, None] + j
    seen = (pos <= query_pos[..., None]) & (pos < seq_len[:, None, None])
    if case["window"]:
        seen &= pos > query_pos[..., None] - case["window"]
    seen = seen[:, None].repeat_interleave(group, 2)
    out, lse = _softmax_rows(torch.matmul(q, k.transpose(-1, -2)) / math.sqrt(D), seen, v)
    out = out.unflatten(2, (most, group)).permute(0, 2, 1, 3, 4).flatten(2, 3)
    lse = lse.unflatten(2, (most, group)).permute(0, 2, 1, 3).flatten(2, 3)
    token = torch.arange(total, device=DEV)
    owner = torch.searchsorted(start[1:], token, right=True)
    at = (owner, token - start[owner])
    return out[at].to(getattr(torch, case["out"])), lse[at]


def _plain_tokens(s):
    case = s["case"]
    pos = s["pos"].long()
    b = torch.gather(s["table"].long()[:, None].expand(-1, case["heads"], -1), 2, pos // case["block"])
    k, v = _rows(s["data"], b, pos % case["block"], torch.arange(case["heads"], device=DEV)[None, :, None])
    seen = (torch.arange(case["tokens"], device=DEV) < s["n_tok"][..., None])[:, :, None]
    q = s["q"].float().unflatten(1, (case["heads"], case["group"]))
    out, lse = _softmax_rows(torch.matmul(q, k.transpose(-1, -2)) / math.sqrt(D), seen, v)
    return out.flatten(1, 2), lse.flatten(1, 2)


def _own_run(s):
    from paper_2604_10539_amd import IceCache, ice_plan_blocks
    case = s["case"]
    if case["kind"] == "plan":
        ice_plan_blocks(s["gain"], s["cached"], s["seq_len"], s["table"], s["free_ids"], s["n_free"], s["n_free_left"], s["query_start"],
                        s["slots"], s["info"], case["block"])
        return s["seq_len"], s["table"], s["free_ids"], s["n_free_left"], s["query_start"], s["slots"], s["info"]
    cache = s.get("cache")
    if cache is None:  # the handle that a program keeps: it holds the tensor and its sizes
        cache = s["cache"] = IceCache(s["data"].shape[0], case["heads"], case["block"], data=s["data"])
    if case["kind"] == "store":
        cache.write(s["k"], s["v"], s["slots"])
        return cache.read(s["table"], s["seq_len"], case["new"], first=s["first"])
    if case["kind"] == "attend":
        return cache.attend(s["q"], s["query_start"], s["seq_len"], s["table"], max_query=s["max_query"], max_len=s["max_len"],
                            window=case["window"], out_dtype=getattr(torch, case["out"]), with_lse=True)
    return cache.attend_tokens(s["q"], s["seq_len"], s["table"], s["pos"], s["n_tok"], with_lse=True)


def run(state):
    if own:
        return _own_run(state)
    return {"plan": _plain_plan, "store": _plain_store, "attend": _plain_attend, "tokens": _plain_tokens}[state["case"]["kind"]](state)


def work(case):
    cached, gain = _lengths(case)
    after, heads, kind = [c + g for c, g in zip(cached, gain)], case.get("heads", 0), case["kind"]
    if kind == "plan":
        new, n = sum(g for g in gain if g > 0), len(gain)
        blocks = sum(abs(-(-a // case["block"]) - -(-c // case["block"])) for a, c in zip(after, cached))
        return {"bytes": 4.0 * (4 * n + 2 * blocks + new + 6), "flops": 0.0}
    if kind == "store":  # values in, codes out and in again, values out
        rows = sum(gain) * heads
        return {"bytes": rows * (2.0 * 512 + 2 * ROW_BYTES) + 4 * sum(gain), "flops": 0.0}
    rows = sum(gain) * heads * case["group"]
    if kind == "tokens":
        keys = case["requests"] * heads * case["tokens"] * 0.875  # a quarter of the lists is half as long on average
        return {"bytes": keys * (ROW_BYTES + 4) + rows * D * 6.0, "flops": 4.0 * D * keys * case["group"]}
    window = case["window"] or max(after) + 1
    keys = sum(min(a, window + g - 1) for a, g in zip(after, gain) if g > 0) * heads
    pairs = sum(sum(min(c + j + 1, window) for j in range(g)) for c, g in zip(cached, gain)) * heads * case["group"]
    return {"bytes": keys * float(ROW_BYTES) + rows * D * (2.0 + (4 if case["out"] == "float32" else 2)), "flops": 4.0 * D * pairs}


# ------------------------------------------------------------------------------------------------- 64 bits, written apart
_LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_held(x):
    """Float64 values that rows x [n, 128] are held as: the nearest level by distance, the even code on ties."""
    levels = torch.tensor(_LEVELS, dtype=torch.float64, device=DEV)
    even = torch.tensor([0.0, 1e-9] * 4, dtype=torch.float64, device=DEV)  # (a tie's two distances are equal; any others differ by far more than this)
    parts = []
    for x in torch.split(x.double().reshape(-1, 32), PART // 256):
        top = x.abs().amax(1, keepdim=True)
        _, e = torch.frexp(top)  # top = f * 2^e, f in [0.5, 1)
        e = e - 1
        e = torch.where(top > 1.75 * torch.exp2(e.double()), e + 1, e) - 2
        scale = torch.exp2(torch.where(top > 0, e, -100).clamp(-100, 125).double())
        best = ((x.abs() / scale)[..., None] - levels).abs().add(even).argmin(-1)
        held = levels[best] * scale * torch.sign(x)
        parts.append(torch.where(torch.isfinite(x).all(1, keepdim=True), held, float("nan")))
    return torch.cat(parts).reshape(-1, D)


def _exact_rows(data, table, pos, block, heads):
    """Float64 keys and values [heads, len(pos), 128] of one request's positions, byte by byte through tables."""
    low = torch.tensor([(_LEVELS[c & 7] if c & 15 < 8 else -_LEVELS[c & 7]) for c in range(256)], dtype=torch.float64, device=DEV)
    high = torch.tensor([(_LEVELS[c >> 4 & 7] if c >> 4 < 8 else -_LEVELS[c >> 4 & 7]) for c in range(256)], dtype=torch.float64, device=DEV)
    power = torch.tensor([2.0 ** (b - 127) for b in range(255)] + [float("nan")], dtype=torch.float64, device=DEV)
    base = (table.long()[pos // block] * heads * (block // TILE) + pos % block // TILE) * TILE_BYTES
    base = base[None, :] + torch.arange(heads, device=DEV)[:, None] * (block // TILE) * TILE_BYTES
    flat, t = data.reshape(-1), pos % TILE
    dim = torch.arange(D, device=DEV)
    both = []
    for side in (0, 1):
        byte = flat[base[..., None] + 1024 * side + (64 * t)[:, None] + dim // 2].long()
        scale = flat[base[..., None] + 2048 + 64 * side + (16 * (t % 4) + t // 4)[:, None] + 4 * (dim // 32)].long()
        both.append(torch.where(dim % 2 == 0, low[byte], high[byte]) * power[scale])
    return both


def _exact_softmax(q, k, v, seen):
    """Rows q [h, r, 128] against k, v [h, n, 128]; seen [h or 1, r, n]."""
    x = torch.bmm(q, k.transpose(1, 2).contiguous()) * (1.0 / math.sqrt(128.0))
    x.masked_fill_(~seen, float("-inf"))
    lse = torch.logsumexp(x, -1)
    x.sub_(torch.where(torch.isinf(lse), 0.0, lse)[..., None]).exp_()
    return torch.bmm(x, v), lse


def exact(case, seed):
    if case["kind"] == "plan":
        return None
    s = prepare(case, seed)
    block, heads = case["block"], case["heads"]
    if case["kind"] == "store":
        got = []
        for x in (s["k"], s["v"]):
            held = _exact_held(x.reshape(-1, D)).reshape(case["requests"], case["new"], heads, D)
            got.append(held.transpose(1, 2))
        return tuple(got)
    group, q = case["group"], s["q"].double()
    out, lse = torch.zeros_like(q), torch.full(q.shape[:2], float("-inf"), dtype=torch.float64, device=DEV)
    cached, gain = _lengths(case)
    at = 0
    for r in range(case["requests"]):
        if case["kind"] == "tokens":
            for h in range(heads):
                pos = s["pos"][r, h, : int(s["n_tok"][r, h])].long()
                if not pos.numel():
                    continue
                k, v = _exact_rows(s["data"], s["table"][r], pos, block, heads)
                rows = slice(h * group, (h + 1) * group)
                o, z = _exact_softmax(q[r: r + 1, rows], k[h: h + 1], v[h: h + 1], torch.ones((1, 1, 1), dtype=torch.bool, device=DEV))
                out[r, rows], lse[r, rows] = o[0], z[0]
            continue
        pos = torch.arange(cached[r] + gain[r], device=DEV)
        k, v = _exact_rows(s["data"], s["table"][r], pos, block, heads)
        step = max(1, PART * 8 // max(1, heads * group * pos.numel()))
        for j in range(0, gain[r], step):
            m = min(step, gain[r] - j)
            here = q[at + j: at + j + m].reshape(m, heads, group, D).permute(1, 0, 2, 3).reshape(heads, m * group, D)
            p = (cached[r] + j + torch.arange(m, device=DEV))[:, None]
            seen = pos <= p
            if case["window"]:
                seen &= p - pos < case["window"]
            o, z = _exact_softmax(here.contiguous(), k, v, seen.repeat_interleave(group, 0)[None])
            out[at + j: at + j + m] = o.reshape(heads, m, group, D).permute(1, 0, 2, 3).reshape(m, heads * group, D)
            lse[at + j: at + j + m] = z.reshape(heads, m, group).permute(1, 0, 2).reshape(m, heads * group)
        at += gain[r]
    return out, lse
