"""Operators on a K/V cache that is held at 8 or 4 bits, with their plain forms, as cases to be measured.

write:  K and V rows of new tokens are quantised into the held pool, each group of channels of a token with a scale and a
        zero-point of its own; optionally the values that the pool then holds come back as rows.
read:   rows of tokens out of the held pool.
attend: one new token per sequence attends to its tokens in the held pool (one layer); optionally its own K/V row is quantised
        into the pool by the same call.

A held pool is bytes [layer][KV head][tile][K codes | V codes | K parameters | V parameters], a tile being 16 tokens of a chunk
slot; a sequence's table lists the slots of its chunks.  Inside a tile, with W = dim * bits / 128 and VW the largest of 4, 2, 1
that divides W: the K codes of a token are W * 4 little-endian words of 32 bits, word (w, j) (w < W, j < 4) of token (i, g)
(i < 2, g < 8) lying at place [i][w / VW][g][j][w % VW]; the V codes of a token are W * 8 units of 16 bits, unit (w, g) (g < 8) of
token (i, j, e) (j < 4, e < 2) lying at place [i][w / VW][g][j][w % VW][e].  Parameters: [token][group] of (scale, zero) in fp16.
The rule of quantisation fixes every rounding, so the pool's bytes are the same for every implementation: they come back as
they are, and so do the values that they stand for where an operator gives them.

Where `own` is true the calls go to the package's binding, otherwise plain torch operations compute the same.
"""
import math
import random

import torch

own = False

_TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
_package = None


def _binding():
    global _package
    if _package is None:
        from paper_2403_11805_b200 import binding
        _package = binding
    return _package


def _write(name, **kw):
    case = {"name": name, "op": "write", "type": "f16", "bits": 4, "span": 128, "seqs": 1, "heads": 32, "dim": 128, "tokens": 4096,
            "new": 4096, "chunk": 16, "ragged": False, "seen": True}
    case.update(kw)
    return case


def _read(name, **kw):
    return {**_write(name, op="read", **kw), "seen": False}


def _attend(name, **kw):
    case = {"name": name, "op": "attend", "type": "f16", "bits": 4, "span": 128, "seqs": 1, "heads": 32, "group": 1, "dim": 128,
            "tokens": 4096, "chunk": 16, "ragged": False, "append": True, "window": 0}
    case.update(kw)
    return case


def listed():
    return [
        # a few tokens behind a short context, the smallest call: latency
        _write("write tiny", heads=4, dim=64, span=64, tokens=256, new=5),
        # one token for each sequence of a batch, the multi-query shape at 8 bits
        _write("write gemma2b step", type="bf16", bits=8, seqs=32, heads=1, dim=256, tokens=2048, new=1, seen=False),
        # parts of several apps' prompts, ragged, with the values that their attention is to see
        _write("write multiapp prompts", seqs=8, tokens=1024, new=1024, chunk=32, ragged=True),
        # one long prompt
        _write("write mistral7b 32k", heads=8, tokens=32768, new=32768, chunk=64, seen=False),
        # the last tokens of a ragged batch, multi-query, 8 bits, odd counts
        _read("read gemma2b", type="bf16", bits=8, seqs=4, heads=1, dim=256, tokens=2047, new=1999, ragged=True),
        # a whole 7B context of a layer
        _read("read llama7b"),
        # a short single context, the smallest call: latency
        _attend("attend tiny", heads=4, dim=64, span=64, tokens=256, append=False),
        # one context of the multi-query shape: a single KV head shared by eight query heads, 8 bits
        _attend("attend gemma2b", type="bf16", bits=8, heads=1, group=8, dim=256, tokens=2048),
        # one 4096-token context of the 7B shape
        _attend("attend llama7b"),
        # one long grouped-query context
        _attend("attend mistral7b 32k", heads=8, group=4, tokens=32768, chunk=64),
        # a batch of ragged long contexts whose new token sees a sliding window, a padded row among them
        _attend("attend mistral7b window", type="bf16", seqs=32, heads=8, group=4, tokens=8191, chunk=64, ragged=True, window=4096),
        # a full batch of the 7B shape: throughput
        _attend("attend llama7b batch", seqs=16),
    ]


def _spread(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    case = {"type": rng.choice(["f16", "bf16"]), "bits": rng.choice([4, 4, 8]), "chunk": rng.choice([16, 32, 48, 64])}
    heads, group, dim = rng.choice([(4, 1, 64), (1, 8, 256), (32, 1, 128), (8, 4, 128), (4, 7, 64), (2, 16, 64), (8, 3, 128), (5, 2, 96)])
    case.update(heads=heads, dim=dim, span=rng.choice({64: [32, 64], 96: [32], 128: [32, 64, 128], 256: [64, 128, 256]}[dim]))
    if rng.random() < 0.5:
        tokens = _spread(rng, 1, 32768)
        room = 16 * 4096 * 32 * 128 // (heads * dim * tokens * (case["bits"] // 4))
        seqs = _spread(rng, 1, max(1, min(48, room)))
        case.update(op="attend", group=group, tokens=tokens, seqs=seqs, ragged=rng.random() < 0.6, append=rng.random() < 0.6,
                    window=_spread(rng, 1, 8192) if rng.random() < 0.25 else 0)
        return case
    new = _spread(rng, 1, 32768)
    tokens = min(32768, new + (_spread(rng, 1, 4096) if rng.random() < 0.5 else 0))
    seqs = _spread(rng, 1, max(1, min(64, 32768 * 8 * 128 // (heads * dim * tokens))))
    op = rng.choice(["write", "read"])
    case.update(op=op, tokens=tokens, new=new, seqs=seqs, ragged=rng.random() < 0.6, seen=op == "write" and rng.random() < 0.6)
    return case


def _lengths(case):
    """Tokens per sequence: all the same, or spread from 1 to the longest with one padded (empty) row in four or more."""
    n, longest = case["seqs"], case["tokens"]
    if not case["ragged"]:
        return [longest] * n
    rng = random.Random(n * 1000003 + longest)
    got = [longest] + [_spread(rng, 1, longest) for _ in range(n - 1)]
    if n >= 4:
        got[n // 2] = 0
    return got


def _new(case):
    """Tokens of each sequence, its last ones, that a write or read goes over."""
    return [min(x, case["new"]) for x in _lengths(case)]


def _seen(case, length):
    return min(length, case["window"]) if case["window"] else length


def _row_bytes(case):
    """Bytes of one token's K (or V) of one head in the pool."""
    return case["dim"] * case["bits"] // 8 + 4 * (case["dim"] // case["span"])


def work(case):
    row, held, lens = case["dim"] * 2, _row_bytes(case), _lengths(case)
    if case["op"] == "attend":
        seen = sum(_seen(case, n) for n in lens) * case["heads"]
        live = sum(n > 0 for n in lens) * case["heads"]
        moved = seen * 2 * held + live * (2 * case["group"] * row + case["group"] * 4)
        if case["append"]:
            moved += live * 2 * (row + held)
        return {"bytes": moved, "flops": seen * case["group"] * 4 * case["dim"]}
    rows = sum(_new(case)) * case["heads"] * 2
    return {"bytes": rows * (row + held + (row if case["seen"] else 0)), "flops": rows * case["dim"] * (6 if case["op"] == "write" else 2)}


# ----------------------------------------------------------------------------- the format, plainly

def _shape(case):
    words = case["dim"] * case["bits"] // 128
    vec = 4 if words % 4 == 0 else 2 if words % 2 == 0 else 1
    codes = 2 * case["dim"] * case["bits"]                    # bytes of 16 tokens' codes
    return words, vec, codes, 64 * (case["dim"] // case["span"])


def _quantise(case, x):
    """Rows [..., dim] -> codes [..., dim] (uint8), parameters [..., groups, 2] (fp16: scale, zero)."""
    top = (1 << case["bits"]) - 1
    x = x.float().clamp(-65504, 65504).half().float().unflatten(-1, (-1, case["span"]))
    low, high = x.amin(-1, keepdim=True) + 0.0, x.amax(-1, keepdim=True)
    scale = ((high - low) / top).half()
    inverse = torch.where(scale == 0, 0.0, 1.0 / scale.float())
    codes = torch.round((x - low) * inverse).clamp(max=top).to(torch.uint8)
    return codes.flatten(-2), torch.cat([scale, low.half()], -1)


def _values(codes, params):
    """What codes and parameters stand for, in 32 bits."""
    x = codes.float().unflatten(-1, (params.shape[-2], -1))
    return (params[..., 1:].float() + x * params[..., :1].float()).flatten(-2)


def _rows_of(values, kind):
    return (values.clamp(-65504, 65504) if kind == torch.float16 else values).to(kind)


def _packed(case, codes):
    """Codes [..., dim] as the row's little-endian bytes."""
    return codes if case["bits"] == 8 else codes[..., 0::2] | (codes[..., 1::2] << 4)


def _unpacked(case, rows):
    return rows if case["bits"] == 8 else torch.stack([rows & 15, rows >> 4], -1).flatten(-2)


def _tiles(case, k, v):
    """K and V rows [..., 16, dim] -> tiles [..., bytes]."""
    words, vec, codes, _ = _shape(case)
    lead = k.shape[:-2]
    (kc, kp), (vc, vp) = _quantise(case, k), _quantise(case, v)
    a = len(lead)

    def placed(x, split, order):
        return x.reshape(*lead, *split).permute(*range(a), *(a + i for i in order)).reshape(*lead, codes)

    kc = placed(_packed(case, kc), (2, 8, words // vec, vec, 4, 4), (0, 2, 1, 4, 3, 5))
    vc = placed(_packed(case, vc), (2, 4, 2, words // vec, vec, 8, 2), (0, 3, 5, 1, 4, 2, 6))
    return torch.cat([kc, vc, kp.contiguous().view(torch.uint8).reshape(*lead, -1), vp.contiguous().view(torch.uint8).reshape(*lead, -1)], -1)


def _opened(case, tiles):
    """Tiles [..., bytes] -> K values, V values [..., 16, dim] in 32 bits."""
    words, vec, codes, params = _shape(case)
    lead = tiles.shape[:-1]
    a = len(lead)

    def placed(x, split, order):
        return x.reshape(*lead, *split).permute(*range(a), *(a + i for i in order)).reshape(*lead, 16, -1)

    kc = placed(tiles[..., :codes], (2, words // vec, 8, 4, vec, 4), (0, 2, 1, 4, 3, 5))
    vc = placed(tiles[..., codes:2 * codes], (2, words // vec, 8, 4, vec, 2, 2), (0, 3, 5, 1, 4, 2, 6))
    kp, vp = (tiles[..., 2 * codes + i * params:2 * codes + (i + 1) * params].contiguous().view(torch.float16)
              .reshape(*lead, 16, -1, 2) for i in (0, 1))
    return _values(_unpacked(case, kc), kp), _values(_unpacked(case, vc), vp)


def _byte_places(case, device):
    """Offset inside a tile of every byte of a token's packed K row and V row [2, 16, bytes] and parameters [2, 16, bytes]."""
    words, vec, codes, params = _shape(case)
    token = torch.arange(16, device=device)[:, None]
    byte = torch.arange(case["dim"] * case["bits"] // 8, device=device)[None, :]
    w, j = byte // 16, byte // 4 % 4
    k = (((token // 8 * (words // vec) + w // vec) * 8 + token % 8) * 4 + j) * vec + w % vec
    k = k * 4 + byte % 4
    g, j, e = byte // 2 % 8, token // 2 % 4, token % 2
    v = ((((token // 8 * (words // vec) + w // vec) * 8 + g) * 4 + j) * vec + w % vec) * 2 + e
    v = codes + v * 2 + byte % 2
    p = token * (params // 16) + torch.arange(params // 16, device=device)[None, :]
    return torch.stack([k, v]), torch.stack([2 * codes + p, 2 * codes + params + p])


# ----------------------------------------------------------------------------- states

def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind = _TYPES[case["type"]]

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=gen)

    lens = _lengths(case)
    n, heads, dim, chunk = case["seqs"], case["heads"], case["dim"], case["chunk"]
    layers, layer = 2, 1
    width = -(-case["tokens"] // chunk)                       # chunks of the longest sequence
    need = torch.tensor([-(-x // chunk) for x in lens])
    slots = int(need.sum()) + 2                               # the last ones are nobody's
    order = torch.randperm(slots - 1, device="cuda", generator=gen).to(torch.int32)
    col = torch.arange(width)
    index = ((torch.cumsum(need, 0) - need)[:, None] + col[None, :]).clamp(max=slots - 2).cuda()
    table = torch.where((col[None, :] < need[:, None]).cuda(), order[index], -1).to(torch.int32).contiguous()
    words, _, codes, params = _shape(case)
    size, tiles = 2 * (codes + params), slots * chunk // 16
    state = {"case": case, "slots": slots, "table": table, "lens": torch.tensor(lens, dtype=torch.int32, device="cuda"), "layer": layer,
             "layers": layers}
    # K and V as caches hold them: a scale per channel, two K channels per head far above the others
    scale = torch.exp(0.5 * normal(2, heads, 1, dim))
    loud = torch.randint(0, dim, (heads, 1, 2), device="cuda", generator=gen)
    scale[0].scatter_(2, loud, 10.0)
    if case["op"] == "write":
        state["held"] = torch.randint(0, 256, (layers, heads, tiles, size), dtype=torch.uint8, device="cuda", generator=gen)
    else:
        held = torch.zeros(layers, heads, tiles, size, dtype=torch.uint8, device="cuda")
        for h in range(heads):
            rows = normal(2, tiles, 16, dim) * scale[:, h, :, None, :].reshape(2, 1, 1, dim)
            held[layer, h] = _tiles(case, rows[0].to(kind), rows[1].to(kind))
        state["held"] = held
    if case["op"] == "attend":
        q_heads = heads * case["group"]
        qkv = normal(n, q_heads + 2 * heads, dim)             # one projection's output: q, k and v side by side
        qkv[:, q_heads:q_heads + heads] *= scale[0, :, 0]
        qkv = qkv.to(kind)
        state["q"], state["k"], state["v"] = qkv[:, :q_heads], qkv[:, q_heads:q_heads + heads], qkv[:, q_heads + heads:]
        state["out"] = torch.empty(n, q_heads, dim, dtype=kind, device="cuda")
        state["lse"] = torch.empty(n, q_heads, dtype=torch.float32, device="cuda")
        return state
    new = _new(case)
    total = sum(new) + 3                                      # rows behind the last sequence are nobody's
    if case["new"] == 1 and not case["ragged"]:
        total, state["first_row"] = n, None                   # a row per sequence
    else:
        state["first_row"] = torch.tensor([0] + new, dtype=torch.int32).cumsum(0).to(torch.int32).cuda()
    state["rows"] = total
    if case["op"] == "read":
        state["k_out"], state["v_out"] = (torch.zeros(total, heads, dim, dtype=kind, device="cuda") for _ in range(2))
        return state
    rows = normal(total, 2, heads, dim)
    rows *= scale[:, :, 0]
    rows = rows.to(kind)                                      # one projection's output: k and v side by side
    state["k"], state["v"] = rows[:, 0], rows[:, 1]
    if case["seen"]:
        state["k_seen"], state["v_seen"] = (torch.zeros(total, heads, dim, dtype=kind, device="cuda") for _ in range(2))
    return state


def run(state):
    op = state["case"]["op"]
    if own:
        return _write_own(state) if op == "write" else _read_own(state) if op == "read" else _attend_own(state)
    return _write_plain(state) if op == "write" else _read_plain(state) if op == "read" else _attend_plain(state)


# ----------------------------------------------------------------------------- the framework's calls

def _desc(state):
    """The pool's descriptor and, for attend, a workspace: made once and kept, as a serving program does."""
    B, case = _binding(), state["case"]
    state["desc"] = B.make_desc(state["layers"], case["heads"], case["heads"] * case.get("group", 1), case["dim"],
                                state["slots"] * case["chunk"], case["chunk"], case["span"])
    if case["op"] == "attend":
        size = B.held_workspace_bytes(state["desc"], case["bits"], case["seqs"], case["tokens"])
        state["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    return state["desc"]


def _write_own(state):
    B, case = _binding(), state["case"]
    desc = state.get("desc") or _desc(state)
    B.held_write(desc, case["bits"], state["layer"], state["held"], state["k"], state["v"], state["table"], state["lens"], case["tokens"],
                 first_row=state["first_row"], k_seen=state.get("k_seen"), v_seen=state.get("v_seen"))
    return [state["held"], state["k_seen"], state["v_seen"]] if case["seen"] else [state["held"]]


def _read_own(state):
    B, case = _binding(), state["case"]
    desc = state.get("desc") or _desc(state)
    B.held_read(desc, case["bits"], state["layer"], state["held"], state["table"], state["lens"], case["tokens"], state["k_out"],
                state["v_out"], first_row=state["first_row"])
    return [state["k_out"], state["v_out"]]


def _attend_own(state):
    B, case = _binding(), state["case"]
    desc = state.get("desc") or _desc(state)
    new = case["append"]
    B.held_attention(desc, case["bits"], state["layer"], state["held"], state["q"], state["table"], state["lens"], case["tokens"],
                     state["out"], state["workspace"], k_new=state["k"] if new else None, v_new=state["v"] if new else None,
                     window=case["window"], lse=state["lse"])
    return [state["out"], state["lse"]] + ([state["held"]] if new else [])


# ----------------------------------------------------------------------------- the plain forms

def _places(state):
    """Of every row that is some token's: the row, its tile in the pool and its place in the tile."""
    lens, table, chunk = state["lens"].long(), state["table"].long(), state["case"]["chunk"]
    first = state["first_row"]
    if first is None:
        row = torch.arange(state["rows"], device="cuda")
        seq, position = row, lens - 1
    else:
        first = first.long()
        row = torch.arange(int(sum(_new(state["case"]))), device="cuda")
        seq = torch.searchsorted(first, row, right=True) - 1
        position = lens[seq] - first[seq + 1] + row
    pool_row = table[seq, position // chunk] * chunk + position % chunk
    return row, pool_row // 16, pool_row % 16


def _stored(state, k, v, tile, place):
    """Rows [rows, heads, dim] into the pool; the values that it then holds, in 32 bits."""
    case, held = state["case"], state["held"][state["layer"]]
    at_codes, at_params = _byte_places(case, "cuda")
    head = torch.arange(case["heads"], device="cuda")[None, :, None]
    seen = []
    for s, x in enumerate((k, v)):
        codes, params = _quantise(case, x)
        held[head, tile[:, None, None], at_codes[s, place][:, None, :]] = _packed(case, codes)
        held[head, tile[:, None, None], at_params[s, place][:, None, :]] = params.contiguous().view(torch.uint8).flatten(-2)
        seen.append(_values(codes, params))
    return seen


def _write_plain(state):
    case = state["case"]
    row, tile, place = _places(state)
    k, v = _stored(state, state["k"][row], state["v"][row], tile, place)
    if not case["seen"]:
        return [state["held"]]
    state["k_seen"][row], state["v_seen"][row] = _rows_of(k, state["k"].dtype), _rows_of(v, state["v"].dtype)
    return [state["held"], state["k_seen"], state["v_seen"]]


def _read_plain(state):
    case, held = state["case"], state["held"][state["layer"]]
    row, tile, place = _places(state)
    at_codes, at_params = _byte_places(case, "cuda")
    head = torch.arange(case["heads"], device="cuda")[None, :, None]
    for s, out in enumerate((state["k_out"], state["v_out"])):
        codes = _unpacked(case, held[head, tile[:, None, None], at_codes[s, place][:, None, :]])
        params = held[head, tile[:, None, None], at_params[s, place][:, None, :]].view(torch.float16).unflatten(-1, (-1, 2))
        out[row] = _rows_of(_values(codes, params), out.dtype)
    return [state["k_out"], state["v_out"]]


def _attend_plain(state):
    case, lens, table = state["case"], state["lens"], state["table"].long()
    n, heads, group, dim, tokens, chunk = case["seqs"], case["heads"], case["group"], case["dim"], case["tokens"], case["chunk"]
    if case["append"]:
        live = torch.tensor([i for i, x in enumerate(_lengths(case)) if x > 0], device="cuda")
        last = lens[live].long() - 1
        pool_row = table[live, last // chunk] * chunk + last % chunk
        _stored(state, state["k"][live], state["v"][live], pool_row // 16, pool_row % 16)
    whole = -(-tokens // 16)
    t = torch.arange(whole, device="cuda") * 16
    slot = table[:, t // chunk]
    tile = torch.where(slot < 0, state["slots"] - 1, slot) * (chunk // 16) + t % chunk // 16
    k, v = (x.flatten(2, 3)[:, :, :tokens] for x in _opened(case, state["held"][state["layer"]][:, tile]))     # [heads, n, tokens, dim]
    t = torch.arange(tokens, device="cuda")
    first = (lens - case["window"]).clamp(min=0) if case["window"] else torch.zeros_like(lens)
    seen = ((t[None, :] >= first[:, None]) & (t[None, :] < lens[:, None]))[None, :, :, None]
    k = torch.where(seen, k, 0.0)
    q = state["q"].float().reshape(n, heads, group, dim).permute(1, 0, 3, 2)
    s = torch.where(seen, torch.matmul(k, q) / math.sqrt(dim), -math.inf)                                     # [heads, n, tokens, group]
    del k
    top = s.amax(2, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(s - top)
    total = p.sum(2, keepdim=True)
    p = torch.where(total > 0, p / total, 0.0)
    v = torch.where(seen, v, 0.0)
    out = torch.matmul(p.transpose(2, 3), v).permute(1, 0, 2, 3).reshape(n, heads * group, dim).to(state["out"].dtype)
    lse = (top + torch.log(total)).permute(1, 0, 3, 2).reshape(n, heads * group)
    return [out, lse] + ([state["held"]] if case["append"] else [])


# ----------------------------------------------------------------------------- the definition in 64 bits

def _exact_values(case, rows):
    """Values that rows are held as: the rule's decisions are made in 32 bits by definition, everything else here in 64."""
    top = (1 << case["bits"]) - 1
    groups = rows.double().clamp(-65504, 65504).half().double().reshape(-1, case["span"])
    zero = groups.min(1, keepdim=True).values
    spread = (groups.max(1, keepdim=True).values - zero).float().double()
    scale = (spread / top).float().half().double()
    steps = ((groups - zero).float().double() * (1 / scale).float().double()).float().double()
    code = torch.where(scale > 0, torch.round(steps).clamp(max=top), 0.0)
    return (zero + code * scale).reshape(rows.shape)


def _exact_token_rows(state, h, seq, positions):
    """K and V values of tokens out of the pool: every code looked up at its place."""
    case, chunk, bits = state["case"], state["case"]["chunk"], state["case"]["bits"]
    words, vec, codes, params = _shape(case)
    pool_row = state["table"][seq].long()[positions // chunk] * chunk + positions % chunk
    tile = state["held"][state["layer"], h, pool_row // 16].long()
    t = (pool_row % 16)[:, None]
    c = torch.arange(case["dim"], device="cuda")[None, :]
    per_word = 32 // bits
    word, inside = c // per_word, c % per_word * bits
    w, j = word // 4, word % 4
    at_k = ((((t // 8 * (words // vec) + w // vec) * 8 + t % 8) * 4 + j) * vec + w % vec) * 4 + inside // 8
    unit, inside_unit = c // (per_word // 2), c % (per_word // 2) * bits
    w, g = unit // 8, unit % 8
    at_v = codes + (((((t // 8 * (words // vec) + w // vec) * 8 + g) * 4 + t % 8 // 2) * vec + w % vec) * 2 + t % 2) * 2 + inside_unit // 8
    got = []
    for s, (at, shift) in enumerate(((at_k, inside % 8), (at_v, inside_unit % 8))):
        code = (torch.gather(tile, 1, at) >> shift) & ((1 << bits) - 1)
        at_p = 2 * codes + s * params + (t * (case["dim"] // case["span"]) + c // case["span"]) * 4
        scale, zero = ((torch.gather(tile, 1, at_p + o) + (torch.gather(tile, 1, at_p + o + 1) << 8)).to(torch.int32).to(torch.int16)
                       .view(torch.float16).double() for o in (0, 2))
        got.append(zero + code * scale)
    return got


def exact(case, seed):
    state = prepare(case, seed)
    lens, heads = _lengths(case), case["heads"]
    if case["op"] == "write":
        if not case["seen"]:
            return None
        total = sum(_new(case)) if state["first_row"] is not None else case["seqs"]
        got = [None]
        for x in (state["k"], state["v"]):
            values = torch.zeros(x.shape, dtype=torch.float64, device="cuda")
            values[:total] = _exact_values(case, x[:total])
            got.append(values)
        return got
    if case["op"] == "read":
        got = [torch.zeros(state["rows"], heads, case["dim"], dtype=torch.float64, device="cuda") for _ in range(2)]
        row = 0
        for b, (length, new) in enumerate(zip(lens, _new(case))):
            positions = torch.arange(length - new, length, device="cuda")
            for h in range(heads):
                for out, x in zip(got, _exact_token_rows(state, h, b, positions)):
                    out[row:row + new, h] = x
            row += new
        return got
    group = case["group"]
    out = torch.zeros(case["seqs"], heads * group, case["dim"], dtype=torch.float64, device="cuda")
    lse = torch.full((case["seqs"], heads * group), -math.inf, dtype=torch.float64, device="cuda")
    for b, length in enumerate(lens):
        if length == 0:
            continue
        positions = torch.arange(length - _seen(case, length), length, device="cuda")
        for h in range(heads):
            k, v = _exact_token_rows(state, h, b, positions)
            if case["append"]:
                k[-1], v[-1] = _exact_values(case, state["k"][b, h]), _exact_values(case, state["v"][b, h])
            mine = slice(h * group, (h + 1) * group)
            s = state["q"][b, mine].double() @ k.T / case["dim"] ** 0.5
            lse[b, mine] = torch.logsumexp(s, 1)
            out[b, mine] = torch.softmax(s, 1) @ v
    return [out, lse] + ([None] if case["append"] else [])
