"""Operators on the paged K/V cache (the pool of chunk slots), with their plain forms, as cases to be measured.

attend: one new token per sequence attends to its cached tokens (one layer of the pool); optionally the new token's
        K/V row is stored by the same call, and every cached token's attention weight is added to an accumulator.
evict:  per layer and KV head the tokens with the largest accumulated weight stay (the most recent ones in any case);
        their K/V rows and weights are closed up, in place or into other slots of the pool.

A pool is kv[layer][K or V][KV head][slot * chunk + t][channel]; a sequence's table lists the slots of its chunks.
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


def _attend(name, **kw):
    case = {"name": name, "op": "attend", "type": "f16", "seqs": 1, "heads": 32, "group": 1, "dim": 128, "tokens": 4096, "chunk": 16,
            "ragged": False, "append": True, "mass": False, "window": 0}
    case.update(kw)
    return case


def _evict(name, **kw):
    case = {"name": name, "op": "evict", "type": "f16", "layers": 32, "seqs": 1, "heads": 32, "dim": 128, "tokens": 4096, "chunk": 16,
            "ragged": False, "budget": 2048, "recent": 256, "in_place": True}
    case.update(kw)
    return case


def listed():
    return [
        # a short single context, the smallest call: latency
        _attend("attend tiny", heads=4, dim=64, tokens=256, append=False),
        # one context of the multi-query shape: a single KV head shared by eight query heads
        _attend("attend gemma2b", type="bf16", heads=1, group=8, dim=256, tokens=2048),
        # one 4096-token context of the 7B shape, accumulating the weights that eviction ranks by
        _attend("attend llama7b", mass=True),
        # several apps' contexts of different lengths served in one batch, a padded row among them
        _attend("attend multiapp", seqs=8, tokens=1024, chunk=32, ragged=True),
        # one long grouped-query context
        _attend("attend mistral7b 32k", heads=8, group=4, tokens=32768, chunk=64, mass=True),
        # a batch of ragged long contexts whose new token sees a sliding window
        _attend("attend mistral7b window", type="bf16", seqs=32, heads=8, group=4, tokens=8191, chunk=64, ragged=True, window=4096),
        # a full batch of the 7B shape: throughput
        _attend("attend llama7b batch", seqs=16),
        # the smallest context shrunk to half
        _evict("evict tiny", layers=1, heads=4, dim=64, tokens=256, budget=128, recent=16),
        # the multi-query shape, odd length and budget
        _evict("evict gemma2b", type="bf16", layers=18, heads=1, dim=256, tokens=2047, budget=1001, recent=65),
        # several contexts shrunk at once, into slots of their own
        _evict("evict multiapp", layers=8, seqs=8, tokens=1024, chunk=32, ragged=True, budget=512, recent=64, in_place=False),
        # a whole 7B context shrunk to half where it lies
        _evict("evict llama7b"),
        # a long grouped-query context cut to a quarter, into other slots
        _evict("evict mistral7b 32k", heads=8, tokens=32768, chunk=64, budget=8192, recent=512, in_place=False),
    ]


def _spread(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["f16", "bf16"])
    chunk = rng.choice([16, 32, 64])
    if rng.random() < 0.6:
        heads, group, dim = rng.choice([(4, 1, 64), (1, 8, 256), (32, 1, 128), (8, 4, 128), (4, 7, 80), (2, 16, 64), (8, 3, 128), (5, 2, 96)])
        tokens = _spread(rng, 1, 32768)
        room = 16 * 4096 * 32 * 128 // (heads * dim * tokens)
        seqs = _spread(rng, 1, max(1, min(48, room)))
        return {"op": "attend", "type": kind, "seqs": seqs, "heads": heads, "group": group, "dim": dim, "tokens": tokens, "chunk": chunk,
                "ragged": rng.random() < 0.6, "append": rng.random() < 0.6, "mass": rng.random() < 0.4,
                "window": _spread(rng, 1, 8192) if rng.random() < 0.25 else 0}
    heads, dim = rng.choice([(4, 64), (1, 256), (32, 128), (8, 128), (4, 80), (5, 96)])
    tokens = _spread(rng, 2, 32768)
    room = 32 * 4096 * 32 * 128 // (heads * dim * tokens)
    layers = _spread(rng, 1, max(1, min(32, room)))
    seqs = _spread(rng, 1, max(1, min(16, room // layers)))
    budget = _spread(rng, 1, tokens)
    return {"op": "evict", "type": kind, "layers": layers, "seqs": seqs, "heads": heads, "dim": dim, "tokens": tokens, "chunk": chunk,
            "ragged": rng.random() < 0.5, "budget": budget, "recent": rng.randrange(0, budget + 1) // rng.choice([1, 2, 8]),
            "in_place": rng.random() < 0.5}


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


def _seen(case, length):
    return min(length, case["window"]) if case["window"] else length


def work(case):
    lens = _lengths(case)
    row = case["dim"] * 2
    if case["op"] == "attend":
        seen = sum(_seen(case, n) for n in lens) * case["heads"]
        live = sum(n > 0 for n in lens) * case["heads"]
        moved = seen * 2 * row + live * (2 * case["group"] * row + case["group"] * 4) + (live * 4 * row if case["append"] else 0)
        if case["mass"]:
            moved += sum(lens) * case["heads"] * 8
        return {"bytes": moved, "flops": seen * case["group"] * 4 * case["dim"]}
    slabs = case["layers"] * case["heads"]
    kept = sum(min(n, case["budget"]) for n in lens) * slabs
    return {"bytes": sum(lens) * slabs * 8 + kept * (4 * row + 4), "flops": sum(lens) * slabs}


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind = _TYPES[case["type"]]

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=gen)

    lens = _lengths(case)
    n, heads, dim, chunk = case["seqs"], case["heads"], case["dim"], case["chunk"]
    evict = case["op"] == "evict"
    layers = case["layers"] if evict else 2
    width = -(-case["tokens"] // chunk)                       # chunks of the longest sequence
    need = torch.tensor([-(-x // chunk) for x in lens])
    out_width = -(-min(case["budget"], case["tokens"]) // chunk) if evict and not case["in_place"] else 0
    out_need = torch.tensor([-(-min(x, case["budget"]) // chunk) if out_width else 0 for x in lens])
    slots = int(need.sum() + out_need.sum()) + 2              # the last slot is nobody's
    order = torch.randperm(slots - 1, device="cuda", generator=gen).to(torch.int32)
    at = torch.cumsum(need, 0) - need
    col = torch.arange(width)

    def table(first, count, cols):
        index = (first[:, None] + cols[None, :]).clamp(max=slots - 2).cuda()
        return torch.where((cols[None, :] < count[:, None]).cuda(), order[index], -1).to(torch.int32).contiguous()

    # K and V as caches hold them: a scale per channel, two K channels per head far above the others
    scale = torch.exp(0.5 * normal(layers, 2, heads, 1, dim))
    loud = torch.randint(0, dim, (layers, heads, 1, 2), device="cuda", generator=gen)
    scale[:, 0].scatter_(3, loud, 10.0)
    kv = torch.empty(layers, 2, heads, slots * chunk, dim, dtype=kind, device="cuda")
    for l in range(layers):
        kv[l] = normal(2, heads, slots * chunk, dim) * scale[l]
    state = {"case": case, "kv": kv, "slots": slots, "table": table(at, need, col), "lens": torch.tensor(lens, dtype=torch.int32, device="cuda")}
    if evict:
        # weights gathered over many steps: a few tokens carry most of it, some never got any
        weight = torch.rand(layers, n, heads, case["tokens"], device="cuda", generator=gen)
        state["mass"] = torch.where(weight < 0.02, torch.zeros_like(weight), weight ** 8 * 50)
        state["mass_out"] = torch.zeros_like(state["mass"])
        state["kept"] = torch.empty(layers, n, heads, case["budget"], dtype=torch.int32, device="cuda")
        state["new_lens"] = torch.empty(n, dtype=torch.int32, device="cuda")
        if out_width:
            state["dst"] = table(int(need.sum()) + torch.cumsum(out_need, 0) - out_need, out_need, torch.arange(out_width))
        else:
            state["dst"] = None
        return state
    q_heads = heads * case["group"]
    qkv = normal(n, q_heads + 2 * heads, dim).to(kind)        # one projection's output: q, k and v side by side
    state["q"], state["k_new"], state["v_new"] = qkv[:, :q_heads], qkv[:, q_heads:q_heads + heads], qkv[:, q_heads + heads:]
    state["out"] = torch.empty(n, q_heads, dim, dtype=kind, device="cuda")
    state["lse"] = torch.empty(n, q_heads, dtype=torch.float32, device="cuda")
    if case["mass"]:
        # zero behind a sequence's older tokens
        old = torch.arange(case["tokens"], device="cuda")[None, :] < state["lens"][:, None] - 1
        state["mass"] = (torch.rand(n, heads, case["tokens"], device="cuda", generator=gen) ** 8 * 50) * old[:, None, :]
        state["mass_out"] = torch.zeros_like(state["mass"])
    return state


def run(state):
    if state["case"]["op"] == "attend":
        return _attend_own(state) if own else _attend_plain(state)
    return _evict_own(state) if own else _evict_plain(state)


def _desc(state):
    """The pool's descriptor and, for attend, a workspace: made once and kept, as a serving program does."""
    B, case, kv = _binding(), state["case"], state["kv"]
    layers, _, heads, tokens, dim = kv.shape
    state["desc"] = B.make_desc(layers, heads, heads * case.get("group", 1), dim, tokens, case["chunk"], 16)
    if case["op"] == "attend":
        size = B.decode_workspace_bytes(state["desc"], case["seqs"], case["tokens"], case["mass"])
        state["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    return state["desc"]


def _attend_own(state):
    B, case = _binding(), state["case"]
    desc = state.get("desc") or _desc(state)
    new = case["append"]
    B.decode_attention(desc, 1, state["kv"], state["q"], state["table"], state["lens"], case["tokens"], state["out"], state["workspace"],
                       k_new=state["k_new"] if new else None, v_new=state["v_new"] if new else None, window=case["window"],
                       lse=state["lse"], mass_in=state.get("mass"), mass_out=state.get("mass_out"))
    got = [state["out"], state["lse"]]
    if case["mass"]:
        got.append(state["mass_out"])
    if new:
        got.append(state["kv"])
    return got


def _evict_own(state):
    B, case = _binding(), state["case"]
    desc = state.get("desc") or _desc(state)
    B.evict_tokens(desc, state["kv"], state["mass"], state["table"], state["lens"], case["tokens"], case["budget"], case["recent"],
                   state["kept"], state["new_lens"], mass_out=state["mass_out"], dst_table=state["dst"])
    return [state["kept"], state["new_lens"], state["mass_out"], state["kv"]]


def _rows(state, table, position):
    """Pool rows of token positions [n, ...] under a table; position -1 (or an unlisted chunk) is a row of the last slot."""
    chunk = state["case"]["chunk"]
    where = position.clamp(min=0).long()
    slot = torch.gather(table.long(), 1, (where // chunk).reshape(where.shape[0], -1).clamp(max=table.shape[1] - 1)).reshape(where.shape)
    slot = torch.where((position < 0) | (slot < 0), state["slots"] - 1, slot)
    return slot * chunk + torch.where(position < 0, 0, where % chunk)


def _attend_plain(state):
    case, lens = state["case"], state["lens"]
    n, heads, group, dim, tokens = case["seqs"], case["heads"], case["group"], case["dim"], case["tokens"]
    keys, values = state["kv"][1, 0], state["kv"][1, 1]       # [heads, pool rows, dim]
    if case["append"]:
        last = _rows(state, state["table"], (lens - 1)[:, None])[:, 0]
        there = (lens > 0)[None, :, None]
        keys[:, last] = torch.where(there, state["k_new"].transpose(0, 1), keys[:, last])
        values[:, last] = torch.where(there, state["v_new"].transpose(0, 1), values[:, last])
    t = torch.arange(tokens, device="cuda")
    rows = _rows(state, state["table"], t.expand(n, tokens))
    first = (lens - case["window"]).clamp(min=0) if case["window"] else torch.zeros_like(lens)
    seen = (t[None, :] >= first[:, None]) & (t[None, :] < lens[:, None])
    seen = seen[None, :, :, None]                             # [1, n, tokens, 1]
    k = torch.where(seen, keys[:, rows].float(), 0.0)         # [heads, n, tokens, dim]
    q = state["q"].float().reshape(n, heads, group, dim).permute(1, 0, 3, 2)
    s = torch.where(seen, torch.matmul(k, q) / math.sqrt(dim), -math.inf)     # [heads, n, tokens, group]
    del k
    top = s.amax(2, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(s - top)
    total = p.sum(2, keepdim=True)
    p = torch.where(total > 0, p / total, 0.0)
    v = torch.where(seen, values[:, rows].float(), 0.0)
    out = torch.matmul(p.transpose(2, 3), v).permute(1, 0, 2, 3).reshape(n, heads * group, dim).to(state["out"].dtype)
    lse = (top + torch.log(total)).permute(1, 0, 3, 2).reshape(n, heads * group)
    got = [out, lse]
    if case["mass"]:
        inside = (t[None, :] < lens[:, None])[:, None, :]
        got.append(torch.where(inside, state["mass"] + p.sum(3).transpose(0, 1), state["mass_out"]))
    if case["append"]:
        got.append(state["kv"])
    return got


def _evict_plain(state):
    case, kv, lens, mass = state["case"], state["kv"], state["lens"], state["mass"]
    layers, n, heads, tokens = mass.shape
    budget, dim = case["budget"], case["dim"]
    t = torch.arange(tokens, device="cuda")
    length = lens[None, :, None, None]
    kept_n = length.clamp(max=budget)
    # 64-bit keys: any weight lies between "not there" and "recent, stays"
    key = torch.nan_to_num(mass.double(), nan=-1e300, posinf=1e300, neginf=-1e300)
    key = torch.where(t >= length - case["recent"], math.inf, key)
    key = torch.where(t < length, key, -math.inf)
    best = torch.sort(key, dim=3, descending=True, stable=True).indices[..., :budget]
    j = torch.arange(best.shape[3], device="cuda")
    best = torch.sort(torch.where(j < kept_n, best, tokens), dim=3).values
    kept = torch.where(j < kept_n, best, -1)
    target = torch.where(j < kept_n, j, -1).expand(layers, n, heads, -1)
    order = (1, 0, 2, 3)                                      # rows() wants sequences first
    source = _rows(state, state["table"], kept.permute(order)).permute(order)
    table = state["table"] if state["dst"] is None else state["dst"]
    target = _rows(state, table, target.permute(order)).permute(order)

    def index(rows):                                          # [layers, n, heads, kept] -> [layers, 2, heads, n * kept, dim]
        rows = rows.permute(0, 2, 1, 3).reshape(layers, 1, heads, -1, 1)
        return rows.expand(layers, 2, heads, rows.shape[3], dim)

    kv.scatter_(3, index(target), torch.gather(kv, 3, index(source)))
    moved = torch.zeros_like(mass)
    moved[..., :best.shape[3]] = torch.where(j < kept_n, torch.gather(mass, 3, kept.clamp(min=0)), 0.0)
    mass_out = torch.where(t < length, moved, state["mass_out"])
    return [kept.to(torch.int32), lens.clamp(max=budget), mass_out, kv]


def exact(case, seed):
    state = prepare(case, seed)
    kv, lens = state["kv"], _lengths(case)
    chunk = case["chunk"]

    def places(table, b, positions):
        return table[b].long()[positions // chunk] * chunk + positions % chunk

    if case["op"] == "attend":
        heads, group, dim = case["heads"], case["group"], case["dim"]
        out = torch.zeros(case["seqs"], heads * group, dim, dtype=torch.float64, device="cuda")
        lse = torch.full((case["seqs"], heads * group), -math.inf, dtype=torch.float64, device="cuda")
        mass = state["mass_out"].double() if case["mass"] else None
        for b, length in enumerate(lens):
            if length == 0:
                continue
            rows = places(state["table"], b, torch.arange(length, device="cuda"))
            if case["append"]:
                kv[1, 0, :, rows[-1]] = state["k_new"][b]
                kv[1, 1, :, rows[-1]] = state["v_new"][b]
            if mass is not None:
                mass[b, :, :length] = state["mass"][b, :, :length].double()
            first = length - _seen(case, length)
            for h in range(heads):
                mine = slice(h * group, (h + 1) * group)
                s = state["q"][b, mine].double() @ kv[1, 0, h, rows[first:]].double().T / dim ** 0.5
                p = torch.softmax(s, 1)
                lse[b, mine] = torch.logsumexp(s, 1)
                out[b, mine] = p @ kv[1, 1, h, rows[first:]].double()
                if mass is not None:
                    mass[b, h, first:length] += p.sum(0)
        return [out, lse] + ([mass] if case["mass"] else []) + ([kv] if case["append"] else [])
    mass, mass_out = state["mass"].double(), state["mass_out"].double()
    layers, heads, budget = case["layers"], case["heads"], case["budget"]
    kept = torch.full(state["kept"].shape, -1, dtype=torch.int64, device="cuda")
    for b, length in enumerate(lens):
        if length == 0:
            continue
        count = min(length, budget)
        recent = min(case["recent"], count)
        older, quota = length - recent, count - recent
        value = mass[:, b, :, :older]
        stay = torch.ones(layers, heads, length, dtype=torch.bool, device="cuda")
        if quota == 0:
            stay[..., :older] = False
        elif quota < older:
            limit = torch.kthvalue(value, older - quota + 1, dim=2, keepdim=True).values
            above, level = value > limit, value == limit
            spare = quota - above.sum(2, keepdim=True)
            stay[..., :older] = above | (level & (torch.cumsum(level, 2) <= spare))
        ids = torch.nonzero(stay)[:, 2].reshape(layers, heads, count)
        kept[:, b, :, :count] = ids
        mass_out[:, b, :, :length] = 0
        mass_out[:, b, :, :count] = torch.gather(mass[:, b], 2, ids)
        source = places(state["table"], b, ids.reshape(-1)).reshape(ids.shape)
        target = places(state["table"] if state["dst"] is None else state["dst"], b, torch.arange(count, device="cuda"))
        for l in range(layers):
            for h in range(heads):
                kv[l, :, h, target] = kv[l, :, h, source[l, h]]
    return [kept, None, mass_out, kv]
