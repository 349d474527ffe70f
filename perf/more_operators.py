"""Serving attention over a cache held in 4 bits: measured cases of its append, of the attention that reads it (with, if
asked, the weight that each key has received), and of the eviction that keeps the heaviest keys, with their plain forms.

A long context is held in a quarter of the memory: every key and value row of a head is 4-bit codes, a least value and a
step.  `append` rotates new queries and keys and writes keys and values as codes; `attend` is a step or a part of a prompt
over the paged cache; `evict` moves, for each sequence and key head, the first keys, the last ones and the heaviest of
those between into pages of their own.

`run` is the plain form in elementary torch operations, in 32 bits, unless the module's `own` is true; then it makes
the library's calls.  `exact` states the same results from the definitions in 64 bits.

A row x of `d` channels is held as lo = bf16(min x), step = bf16((max x - lo) / 15) and codes rint((x - lo) / step) from 0 to
15; it stands for lo + step * code.  All in 32 bits, each operation rounded on its own, a division being a product with the
rounded reciprocal.
"""
import math

import numpy
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
MAX_POS = 32768


def listed():
    return [
        # ---- append: rotate, quantise, write; and what the cache then holds for these tokens
        # one sequence, one new token: the interactive decode step, where only latency counts
        dict(name="append4 1 token", op="append", kind="decode", tokens=1, hq=32, hkv=8, d=128, rot=128, page=64, dtype="bf16",
             packed=True, interleaved=False),
        # prompts of a batch of 8 x 2048 tokens
        dict(name="append4 prompt 8x2048", op="append", kind="prompt", tokens=16384, hq=32, hkv=8, d=128, rot=128, page=64, dtype="bf16",
             packed=True, interleaved=False),
        # an odd number of prompt tokens in 32 bits, 96-wide heads of which 64 channels rotate, pairs side by side
        dict(name="append4 fp32 odd", op="append", kind="prompt", tokens=3001, hq=16, hkv=4, d=96, rot=64, page=16, dtype="fp32",
             packed=False, interleaved=True),
        # ---- attend: each token over its sequence's keys up to itself
        # one sequence with a 4k context: latency
        dict(name="attend4 1x4096", op="attend", batch=1, qlen=1, hq=32, hkv=8, d=128, page=64, context=4096, dtype="bf16", weights=False),
        # the decode batch of 64 with ragged contexts up to 16k, four query heads for each key head: the largest step
        dict(name="attend4 64x16384", op="attend", batch=64, qlen=1, hq=32, hkv=8, d=128, page=64, context=16384, dtype="bf16", weights=False),
        # many short chats, every head its own keys
        dict(name="attend4 200x1000 d64", op="attend", batch=200, qlen=1, hq=16, hkv=16, d=64, page=16, context=1000, dtype="bf16", weights=False),
        # the decode batch of 32 that keeps the weight each key has received, to evict by
        dict(name="attend4 weights 32x8192", op="attend", batch=32, qlen=1, hq=32, hkv=8, d=128, page=128, context=8192, dtype="bf16", weights=True),
        # questions of up to 64 tokens behind contexts of up to 5000 keys, 96-wide heads
        dict(name="attend4 questions d96", op="attend", batch=8, qlen=64, hq=16, hkv=4, d=96, page=32, context=5001, dtype="bf16", weights=False),
        # a small batch in 32 bits, with weights
        dict(name="attend4 fp32", op="attend", batch=8, qlen=1, hq=12, hkv=12, d=64, page=16, context=1100, dtype="fp32", weights=True),
        # ---- evict: new pages for what stays; and what they then hold
        # one sequence that has passed its budget
        dict(name="evict4 1x4096", op="evict", batch=1, hkv=8, d=128, page=64, context=4096, budget=1024, first=4, last=128),
        # a batch of 32 with ragged contexts up to 16k, a quarter of it kept
        dict(name="evict4 32x16384", op="evict", batch=32, hkv=8, d=128, page=64, context=16384, budget=4096, first=64, last=512),
        # odd sizes: a budget that ends inside a page, some sequences below it
        dict(name="evict4 16x2500 d96", op="evict", batch=16, hkv=4, d=96, page=32, context=2500, budget=1501, first=1, last=77),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw(rng):
    op = rng.choice(["append", "attend", "attend", "evict"])
    while True:
        hkv, group, d = rng.choice([1, 2, 4, 8, 12, 16, 32]), rng.choice([1, 1, 2, 4, 4, 8, 16]), rng.choice([64, 96, 128, 128])
        if hkv * group <= 64:
            break
    c = dict(op=op, hkv=hkv, d=d, page=rng.choice([16, 32, 64, 64, 128]))
    if op == "evict":
        context = _log(rng, 64, 32768)
        budget = max(2, int(context * rng.uniform(0.1, 0.9)))
        first = min(budget, rng.choice([0, 1, 4, budget // 8]))
        c.update(batch=_log(rng, 1, 64), context=context, budget=budget, first=first, last=min(budget - first, rng.choice([0, 1, budget // 8, budget // 3])))
        return c
    c.update(hq=hkv * group, dtype=rng.choice(["bf16"] * 5 + ["fp32"]))
    if op == "append":
        kind = rng.choice(["decode", "prompt"])
        c.update(kind=kind, tokens=_log(rng, 1, 512) if kind == "decode" else _log(rng, 16, 16384), rot=rng.choice([d, d, d // 2]),
                 packed=rng.random() < 0.6, interleaved=rng.random() < 0.3)
    else:
        qlen = 1 if rng.random() < 0.7 else _log(rng, 2, 128)
        c.update(batch=_log(rng, 1, 256 if qlen == 1 else 16), qlen=qlen, context=qlen + _log(rng, 64, 32768), weights=rng.random() < 0.3)
    return c


def _cost(c):
    w = work(c)
    return max(w["bytes"] / 6.5e12, w["flops"] / (1.5e15 if c.get("dtype") == "bf16" else 5e13))


def draw(rng):
    most = {}
    for c in listed():
        most[c["op"]] = max(most.get(c["op"], 0.0), _cost(c))
    while True:
        c = _draw(rng)
        if _cost(c) > most[c["op"]]:
            continue
        if c["op"] == "attend" and 4 * c["batch"] * c["qlen"] * c["hq"] * c["context"] > 1.2e9:
            continue
        return c


def _mean_length(c):
    """Of a ragged batch: the first sequence has the whole context, the others between half of it and all."""
    rest = c.get("qlen", 0)
    return rest + (c["context"] - rest) * (1.0 if c["batch"] == 1 else 0.75)


def work(case):
    """Bytes and operations that the operator cannot do without: every input that it needs read once, every output
    written once.  Ragged lengths count with their mean.  A held row is d/2 bytes of codes and 4 of lo and step."""
    c = case
    row = c["d"] // 2 + 4.0
    if c["op"] == "append":
        e = 4 if c["dtype"] == "fp32" else 2
        live = c["tokens"] * (1.0 if c["kind"] == "decode" else 0.98)
        b = c["tokens"] * (2.0 * c["hq"] * c["d"] * e + 16) + live * (c["rot"] * 4 + 2 * c["hkv"] * (c["d"] * e + row))
        b += c["tokens"] * 2.0 * c["hkv"] * c["d"] * e                       # what the cache then holds
        return {"bytes": b, "flops": c["tokens"] * (3.0 * (c["hq"] + c["hkv"]) * c["rot"] + 10.0 * c["hkv"] * c["d"])}
    if c["op"] == "evict":
        n = c["batch"] * c["hkv"]
        kept = min(c["budget"], _mean_length(c))
        return {"bytes": n * (4.0 * _mean_length(c) + kept * (4 * row + 8) + 2.0 * c["budget"] * c["d"] * 2), "flops": n * 8.0 * _mean_length(c)}
    e = 4 if c["dtype"] == "fp32" else 2
    tokens = c["batch"] * (1 + c["qlen"]) / 2
    keys = c["batch"] * c["hkv"] * _mean_length(c)
    return {"bytes": 2.0 * tokens * c["hq"] * c["d"] * e + keys * (2 * row + (8 if c["weights"] else 0)),
            "flops": 4.0 * tokens * c["hq"] * c["d"] * (_mean_length(c) - (c["qlen"] - 1) / 4)}


# ---- how a row is held

def _hold(x):
    """x [..., d] in 32 bits -> codes uint8 [..., d], lo and step bf16 [...]."""
    lo = x.amin(-1).bfloat16()
    step = ((x.amax(-1) - lo.float()) * (1.0 / 15.0)).bfloat16()
    step = torch.where(step >= 2.0 ** -100, step, torch.zeros_like(step))
    inverse = torch.where(step > 0, step.float().reciprocal(), torch.zeros_like(step, dtype=torch.float32))
    codes = ((x - lo.float()[..., None]) * inverse[..., None]).round().clamp(0, 15)
    return codes.to(torch.uint8), lo, step


def _held(codes, lo, step):
    return lo.float()[..., None] + step.float()[..., None] * codes.float()


# ---- the library's layout: per page and head, for each 16 keys, the codes of the keys, those of the values, and lo and step

def _orders(d):
    """For 16 keys: at which place each half word of four codes lies, counted over (key, channel / 4), for keys and for values."""
    n = d // 32
    keys, values = [], []
    for j in range(16):
        at = ((j >> 1) & 3) | ((j & 1) << 2) | (j & 8)           # the place of value row j
        for quad in range(d // 4):                                # channels 4 quad .. 4 quad + 3
            g, u = quad // 8, quad % 8
            keys.append(j * 8 * n + (u >> 1) * 2 * n + 2 * g + (u & 1))
            if n == 4:
                values.append(at * 32 + (u ^ (4 * ((j >> 2) & 1))) * 4 + g)
            elif n == 2 or g < 2:
                values.append(at * 16 + u * 2 + g)
            else:
                values.append(16 * 16 + at * 8 + u)
    return [torch.argsort(torch.tensor(o, device="cuda")) for o in (keys, values)]


def _pack(held, page, d):
    """Keys and values as (codes, lo, step) of [pages, heads, page, ...] -> the cache [pages, heads, page / 16, 16 d + 128]."""
    parts = []
    for (codes, _, _), order in zip(held, _orders(d)):
        c = codes.view(*codes.shape[:2], page // 16, 16 * d // 4, 4).to(torch.int32)
        half = c[..., 0] | c[..., 1] << 4 | c[..., 2] << 8 | c[..., 3] << 12
        parts.append(half.to(torch.int16)[..., order])
    rows = torch.stack([held[0][2], held[0][1], held[1][2], held[1][1]], dim=-1).view(torch.int16)   # step, lo of the key, of the value
    parts.append(rows.reshape(*rows.shape[:2], page // 16, 64))
    return torch.cat(parts, dim=-1).view(torch.uint8)


# ---- inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 17)
    return g


def _ints(lo, hi, shape, g):  # lo <= value <= hi
    return torch.randint(lo, hi + 1, shape, generator=g, device="cuda", dtype=torch.int64)


def _normal(shape, dtype, g, scale=1.0):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, scale, generator=g)


def prepare(case, seed):
    return {"append": _prepare_append, "attend": _prepare_attend, "evict": _prepare_evict}[case["op"]](case, _gen(seed))


def _filled(pages, c, g):
    """A cache of `pages` pages full of earlier tokens: its plain parts and the library's form.  Channels of keys differ in their
    means, as a model's do."""
    plain = [[torch.empty(pages, c["hkv"], c["page"], *e, dtype=t, device="cuda")
              for e, t in (((c["d"],), torch.uint8), ((), torch.bfloat16), ((), torch.bfloat16))] for _ in range(2)]
    cache = torch.empty(pages, c["hkv"], c["page"] // 16, 16 * c["d"] + 128, dtype=torch.uint8, device="cuda")
    mean = _normal((c["hkv"], 1, c["d"]), torch.float32, g)
    n = max(1, (1 << 27) // (c["hkv"] * c["page"] * c["d"]))
    for p in range(0, pages, n):
        part = []
        for which in range(2):
            x = _normal((min(n, pages - p), c["hkv"], c["page"], c["d"]), torch.float32, g)
            held = _hold(x if which else x + mean)
            for whole, piece in zip(plain[which], held):
                whole[p:p + n] = piece
            part.append(held)
        cache[p:p + n] = _pack(part, c["page"], c["d"])
    return plain, cache


def _prepare_append(c, g):
    T, page, dt = c["tokens"], c["page"], DTYPES[c["dtype"]]
    i = torch.arange(T, device="cuda")
    if c["kind"] == "decode":
        # every sequence has one new token at a place of its own, on a page of its own
        positions = _ints(0, MAX_POS - 1, (T,), g)
        num_pages = T + 3
        slots = torch.randperm(num_pages, generator=g, device="cuda")[:T] * page + positions % page
    else:
        # prompts one after the other, some of them going on where an earlier part ended; the batch is padded at its end
        length = max(1, T // 8)
        start = _ints(0, 500, (T // length + 1,), g)
        start[0] = 0
        seq = i // length
        positions = start[seq] + i % length
        per = (length + 500) // page + 2
        num_pages = (T // length + 1) * per
        perm = torch.randperm(num_pages, generator=g, device="cuda")
        slots = perm[seq * per + positions // page - start[seq] // page] * page + positions % page
        slots[T - T // 50:] = -1
    inv = 10000.0 ** (-torch.arange(c["rot"] // 2, device="cuda", dtype=torch.float64) * 2 / c["rot"])
    angle = torch.arange(MAX_POS, device="cuda", dtype=torch.float64)[:, None] * inv
    if c["packed"]:
        q, k, v = _normal((T, c["hq"] + 2 * c["hkv"], c["d"]), dt, g).split([c["hq"], c["hkv"], c["hkv"]], dim=1)
    else:
        q, k, v = (_normal((T, h, c["d"]), dt, g) for h in (c["hq"], c["hkv"], c["hkv"]))
    plain, cache = _filled(num_pages, c, g)
    return dict(case=c, q=q, k=k, v=v, slots=slots, positions=positions.to(torch.int32), cos=angle.cos().float(), sin=angle.sin().float(),
                plain=plain, cache=cache)


def _lengths(c, g):
    n = c.get("qlen", 0)
    lens = _ints((c["context"] - n) // 2, c["context"] - n, (c["batch"],), g)
    lens[0] = c["context"] - n
    return lens


def _prepare_attend(c, g):
    B, page = c["batch"], c["page"]
    # the first sequence has the most tokens; the others lie between, the same for every seed, so that the batch has one size
    i = torch.arange(B, device="cuda")
    n = c["qlen"] - (c["qlen"] - 1) * (i * 5 % B) // B
    q_start = None if c["qlen"] == 1 else torch.cat([n.new_zeros(1), n.cumsum(0)]).to(torch.int32)
    lens = n + _lengths(c, g)
    width = -(-c["context"] // page)
    perm = torch.randperm(B * width + 1, generator=g, device="cuda").to(torch.int32)
    plain, cache = _filled(B * width + 1, c, g)
    weights = torch.rand(B, c["hkv"], width * page, generator=g, device="cuda") if c["weights"] else None
    return dict(case=c, q=_normal((int(n.sum()), c["hq"], c["d"]), DTYPES[c["dtype"]], g, 1.5), plain=plain, cache=cache,
                page_table=perm[:B * width].reshape(B, width).contiguous(), kv_lens=lens.to(torch.int32), q_start=q_start,
                scale=c["d"] ** -0.5, weights=weights)


def _prepare_evict(c, g):
    B, page = c["batch"], c["page"]
    lens = _lengths(c, g)
    width, width_out = -(-c["context"] // page), -(-c["budget"] // page)
    perm = torch.randperm(B * (width + width_out), generator=g, device="cuda").to(torch.int32)
    plain, cache = _filled(B * (width + width_out), c, g)
    # what keys have received falls off by orders of magnitude; some have received nothing
    weights = torch.exp(2.0 * _normal((B, c["hkv"], width * page), torch.float32, g))
    weights = torch.where(torch.rand(weights.shape, generator=g, device="cuda") < 0.1, torch.zeros_like(weights), weights)
    weights = torch.where(torch.arange(width * page, device="cuda") < lens[:, None, None], weights, torch.zeros_like(weights))
    out_table = perm[B * width:].reshape(B, width_out).contiguous()
    i = torch.arange(c["budget"], device="cuda")
    out_slots = out_table.long()[:, i // page] * page + i % page
    out_slots = torch.where(i < lens[:, None], out_slots, -1).flatten()       # sequences that have fewer keys than the budget
    return dict(case=c, plain=plain, cache=cache, page_table=perm[:B * width].reshape(B, width).contiguous(), kv_lens=lens.to(torch.int32),
                weights=weights, out_table=out_table, out_slots=out_slots)


# ---- one pass

def run(state):
    if own:
        from paper_2603_08343_b200 import attention as A
        s, c = state, state["case"]
        if c["op"] == "append":
            q = A.kv_append4(s["k"], s["v"], s["cache"], s["slots"], positions=s["positions"], cos=s["cos"], sin=s["sin"], q=s["q"],
                             interleaved=c["interleaved"])
            k, v = A.kv_read4(s["cache"], s["slots"], dtype=s["k"].dtype)
            return {"q": q, "keys": k, "values": v}
        if c["op"] == "attend":
            out = A.paged_attention4(s["q"], s["cache"], s["page_table"], s["kv_lens"], q_start=s["q_start"], max_q_len=c["qlen"],
                                     scale=s["scale"], weights=s["weights"])
            return {"out": out[0], "weights": out[1]} if c["weights"] else {"out": out}
        lens, kept, weights = A.kv_evict4(s["cache"], s["page_table"], s["kv_lens"], s["weights"], s["out_table"], c["budget"],
                                          keep_first=c["first"], keep_last=c["last"])
        k, v = A.kv_read4(s["cache"], s["out_slots"], dtype=torch.bfloat16)
        return {"lens": lens, "kept": kept, "weights": weights, "keys": k, "values": v}
    return {"append": _append, "attend": _attend, "evict": _evict}[state["case"]["op"]](state)


def _rotate(x, cos, sin, rot, interleaved):
    """x [T, H, D] in 32 bits; the first `rot` channels turn by the position's angles, in pairs (i, i + rot/2) or (2i, 2i + 1)."""
    h = rot // 2
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :h], x[..., h:rot])
    ra, rb = a * cos - b * sin, b * cos + a * sin
    r = torch.stack([ra, rb], dim=-1).flatten(-2) if interleaved else torch.cat([ra, rb], dim=-1)
    return torch.cat([r, x[..., rot:]], dim=-1)


def _rows_at(plain, slots, page, dtype):
    """What the cache holds at the slots: [n, heads, d]; zeros where a slot is negative."""
    at, off = slots.clamp(min=0) // page, slots.clamp(min=0) % page
    x = _held(*(p[at, :, off] for p in plain))
    return torch.where(slots[:, None, None] >= 0, x, torch.zeros_like(x)).to(dtype)


def _append(s):
    c = s["case"]
    cos, sin = s["cos"][s["positions"].long()][:, None], s["sin"][s["positions"].long()][:, None]
    q = _rotate(s["q"].float(), cos, sin, c["rot"], c["interleaved"]).to(s["q"].dtype)
    k = _rotate(s["k"].float(), cos, sin, c["rot"], c["interleaved"])
    live = s["slots"] >= 0
    at, off = s["slots"][live] // c["page"], s["slots"][live] % c["page"]
    for plain, x in zip(s["plain"], (k, s["v"].float())):
        for whole, part in zip(plain, _hold(x[live])):
            whole[at, :, off] = part
    keys, values = (_rows_at(plain, s["slots"], c["page"], s["k"].dtype) for plain in s["plain"])
    return {"q": q, "keys": keys, "values": values}


def _sequences(plain, table):
    """What a batch's pages hold, in 32 bits: [B, heads, width * page, d]."""
    codes, lo, step = (p[table.long()].transpose(1, 2).flatten(2, 3) for p in plain)
    return _held(codes, lo, step)


def _attend(s):
    c = s["case"]
    T, hq, d = s["q"].shape
    hkv, n, B = c["hkv"], c["qlen"], c["batch"]
    G = hq // hkv
    if s["q_start"] is None:
        at, live = torch.arange(B, device="cuda")[:, None], torch.ones(B, 1, dtype=torch.bool, device="cuda")
    else:
        start = s["q_start"].long()
        at = start[:-1, None] + torch.arange(n, device="cuda")
        live = at < start[1:, None]
    k = _sequences(s["plain"][0], s["page_table"])
    q = s["q"].float()[at.clamp(max=T - 1)].view(B, n, hkv, G, d).permute(0, 2, 1, 3, 4).reshape(B, hkv, n * G, d)
    w = (torch.matmul(q, k.transpose(2, 3)) * s["scale"]).view(B, hkv, n, G, -1)
    del k
    last = s["kv_lens"].long()[:, None] - live.sum(1, keepdim=True) + torch.arange(n, device="cuda")    # [B, n] the token's own place
    seen = (torch.arange(w.shape[-1], device="cuda") <= last[..., None]) & live[..., None]
    w = w.masked_fill(~seen[:, None, :, None], -math.inf)
    top = w.amax(-1, keepdim=True)
    w = torch.exp(w - top.masked_fill(top == -math.inf, 0.0))
    w = w / w.sum(-1, keepdim=True).clamp(min=1e-30)
    v = _sequences(s["plain"][1], s["page_table"])
    out = torch.matmul(w.view(B, hkv, n * G, -1), v).view(B, hkv, n, G, d)
    back = torch.arange(B, device="cuda")[:, None].expand(B, n)[live], torch.arange(n, device="cuda").expand(B, n)[live]
    out = {"out": out[back[0], :, back[1]].reshape(T, hq, d).to(s["q"].dtype)}
    if c["weights"]:
        there = torch.arange(w.shape[-1], device="cuda") < s["kv_lens"].long()[:, None, None]
        out["weights"] = torch.where(there, s["weights"] + w.sum((2, 3)), torch.zeros_like(s["weights"]))
    return out


def _evict(s):
    c = s["case"]
    lens = s["kv_lens"].long()[:, None, None]
    i = torch.arange(s["weights"].shape[-1], device="cuda")
    order = torch.where((i < c["first"]) | (i >= lens - c["last"]), torch.full_like(s["weights"], math.inf), s["weights"])
    order = torch.where(i < lens, order, torch.full_like(order, -math.inf))
    best = torch.sort(order, dim=-1, descending=True, stable=True).indices[..., :c["budget"]]           # ties: the lowest key first
    kept = torch.where(torch.gather(i < lens.expand_as(order), -1, best), best, i.numel()).sort(dim=-1).values
    there = kept < i.numel()
    kept = kept.clamp(max=i.numel() - 1)
    weights = torch.zeros(*kept.shape[:2], s["out_table"].shape[1] * c["page"], device="cuda")
    weights[..., :kept.shape[-1]] = torch.gather(s["weights"], -1, kept) * there
    # the rows, page by page, into pages of their own
    j = torch.arange(kept.shape[-1], device="cuda")
    B, H = kept.shape[:2]
    page_in = s["page_table"].long()[torch.arange(B, device="cuda")[:, None, None], kept // c["page"]]
    page_out = s["out_table"].long()[:, j // c["page"]][:, None].expand_as(kept)
    head = torch.arange(H, device="cuda")[None, :, None].expand_as(kept)
    to = page_out[there], head[there], (j % c["page"]).expand_as(kept)[there]
    for plain in s["plain"]:
        for x in plain:
            x[to] = x[page_in[there], head[there], (kept % c["page"])[there]]
    keys, values = (_rows_at(plain, s["out_slots"], c["page"], torch.bfloat16) for plain in s["plain"])
    return {"lens": s["kv_lens"].clamp(max=c["budget"]), "kept": torch.where(there, kept, -1).to(torch.int32), "weights": weights,
            "keys": keys, "values": values}


# ---- the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "evict": _exact_evict}[case["op"]](case, s)


def _exact_append(c, s):
    half = c["rot"] // 2
    i = torch.arange(half, device="cuda")
    first, second = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + half)
    at = s["positions"].long()
    q = s["q"].double()
    w = torch.complex(s["cos"].double(), s["sin"].double())[at].unsqueeze(1)
    z = torch.complex(q[..., first], q[..., second]) * w
    q[..., first], q[..., second] = z.real, z.imag

    def r32(x):  # held in 64 bits, rounded to 32 as the definition asks
        return x.float().double()

    k = s["k"].double()
    a, b = k[..., first].clone(), k[..., second].clone()
    cos, sin = s["cos"].double()[at].unsqueeze(1), s["sin"].double()[at].unsqueeze(1)
    k[..., first] = r32(r32(a * cos) - r32(b * sin))
    k[..., second] = r32(r32(b * cos) + r32(a * sin))
    out = {"q": q}
    for name, x in (("keys", k), ("values", s["v"].double())):
        lo = x.min(-1, keepdim=True).values.to(torch.bfloat16).double()
        step = r32(r32(x.max(-1, keepdim=True).values - lo) * r32(torch.tensor(1.0 / 15.0, dtype=torch.float64))).to(torch.bfloat16).double()
        code = torch.round(r32(r32(x - lo) * r32(1.0 / step))).clamp(0, 15)
        held = torch.where(step > 0, lo + step * code, lo)
        held[s["slots"] < 0] = 0.0
        out[name] = held
    return out


def _exact_rows(plain, pages, h, n):
    """What the pages of one sequence hold for head h: [n, d] in 64 bits."""
    codes, lo, step = (p[pages, h].flatten(0, 1)[:n] for p in plain)
    return torch.addcmul(lo.double()[:, None], step.double()[:, None], codes.double())


def _exact_attend(c, s):
    G = c["hq"] // c["hkv"]
    if c["batch"] * c["hkv"] > 6000:
        return None
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lens = s["kv_lens"].tolist()
    starts = list(range(c["batch"] + 1)) if s["q_start"] is None else s["q_start"].tolist()
    weights = torch.zeros(c["batch"], c["hkv"], s["page_table"].shape[1] * c["page"], dtype=torch.float64, device="cuda")
    for b in range(c["batch"]):
        t0, t1, n = starts[b], starts[b + 1], lens[b]
        place = n - (t1 - t0) + torch.arange(t1 - t0, device="cuda")
        hidden = torch.arange(n, device="cuda") > place[:, None]
        for h in range(c["hkv"]):
            pages = s["page_table"][b].long()
            k, v = (_exact_rows(x, pages, h, n) for x in s["plain"])
            w = torch.einsum("tgd,nd->tgn", s["q"][t0:t1, h * G:(h + 1) * G].double(), k) * s["scale"]
            w = torch.softmax(w.masked_fill(hidden[:, None], -math.inf), -1)
            out[t0:t1, h * G:(h + 1) * G] = w @ v
            if c["weights"]:
                weights[b, h, :n] = s["weights"][b, h, :n].double() + w.sum((0, 1))
    return {"out": out, "weights": weights} if c["weights"] else {"out": out}


def _exact_evict(c, s):
    lens = s["kv_lens"].tolist()
    received = s["weights"].double().cpu().numpy()
    B, H = c["batch"], c["hkv"]
    weights = numpy.zeros((B, H, s["out_table"].shape[1] * c["page"]))
    rows = [torch.zeros(B, c["budget"], H, c["d"], dtype=torch.float64, device="cuda") for _ in range(2)]
    for b in range(B):
        n = lens[b]
        middle = numpy.arange(min(c["first"], n), max(min(c["first"], n), n - c["last"]))
        spare = min(c["budget"], n) - (n - len(middle))
        for h in range(H):
            # by falling weight, then by place
            ranked = middle[numpy.lexsort((middle, -received[b, h, middle]))]
            kept = numpy.setdiff1d(numpy.arange(n), ranked[spare:])
            weights[b, h, :len(kept)] = received[b, h, kept]
            at = torch.from_numpy(kept).cuda()
            for which in range(2):
                rows[which][b, :len(kept), h] = _exact_rows(s["plain"][which], s["page_table"][b].long(), h, n)[at]
    return {"lens": None, "kept": None, "weights": torch.from_numpy(weights), "keys": rows[0].flatten(0, 1), "values": rows[1].flatten(0, 1)}
