"""Serving attention next to the head mixing: measured cases of the paged cache's append, of attention over a shared
prefix, and of attention over selected pages, with their plain forms.

A decoder layer that ends in the Walsh-Hadamard head mixing starts with these: the projection's new queries, keys and
values are rotated and the keys and values written into a paged cache (`append`); the queries then attend to a prefix
that all sequences of the batch have in common and to each sequence's own pages (`prefix`), or, for long contexts, to
the few pages that a whole-number score picks for each query (`select`).

`run` is the plain form in elementary torch operations, in 32 bits, unless the module's `own` is true; then it makes
the library's calls.  `exact` states the same results from the definitions in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
MAX_POS = 32768


def listed():
    return [
        # ---- append: rotate and write the new keys and values
        # one sequence, one new token: the interactive decode step, where only latency counts
        dict(name="append 1 token", op="append", kind="decode", tokens=1, hq=32, hkv=8, d=128, rot=128, page=64, dtype="bf16",
             summary=True, packed=True, interleaved=False),
        # the decode batch of 256 sequences at 32 x 128 heads, every head with keys and values of its own
        dict(name="append 256 decode", op="append", kind="decode", tokens=256, hq=32, hkv=32, d=128, rot=128, page=64, dtype="bf16",
             summary=False, packed=True, interleaved=False),
        # prompts of a batch of 8 x 2048 tokens at 16 x 64 heads, page summaries kept
        dict(name="append prompt 8x2048", op="append", kind="prompt", tokens=16384, hq=16, hkv=16, d=64, rot=64, page=64, dtype="bf16",
             summary=True, packed=False, interleaved=False),
        # an odd number of prompt tokens in 32 bits, 96-wide heads of which 64 channels rotate, pairs side by side
        dict(name="append fp32 odd", op="append", kind="prompt", tokens=3001, hq=16, hkv=4, d=96, rot=64, page=16, dtype="fp32",
             summary=True, packed=True, interleaved=True),
        # ---- prefix: one copy of the prefix's keys and values serves the whole batch
        # two short chats behind a short system prompt
        dict(name="prefix 2x512", op="prefix", batch=2, qlen=1, hq=16, hkv=16, d=64, page=16, prefix=512, suffix=48, dtype="bf16"),
        # the decode batch of 64 behind an 8k document, four query heads for each key head, ragged answers
        dict(name="prefix 64x8192 grouped", op="prefix", batch=64, qlen=1, hq=32, hkv=8, d=128, page=64, prefix=8192, suffix=500, dtype="bf16"),
        # 256 sequences behind a 32k document, every head its own keys: the largest decode step
        dict(name="prefix 256x32768", op="prefix", batch=256, qlen=1, hq=32, hkv=32, d=128, page=128, prefix=32768, suffix=256, dtype="bf16"),
        # questions of up to 64 tokens put to one text at once, 96-wide heads, a prefix that ends inside a page
        dict(name="prefix questions d96", op="prefix", batch=16, qlen=64, hq=16, hkv=16, d=96, page=32, prefix=5001, suffix=200, dtype="bf16"),
        # a small batch in 32 bits
        dict(name="prefix fp32", op="prefix", batch=8, qlen=1, hq=12, hkv=12, d=64, page=16, prefix=1000, suffix=100, dtype="fp32"),
        # ---- select: each query reads the pages whose score is highest
        # one sequence with a 4k context, 16 pages of it read
        dict(name="select 1x4096", op="select", batch=1, qlen=1, hq=32, hkv=8, d=128, page=64, context=4096, select=16, dtype="bf16"),
        # the decode batch of 64 with ragged contexts up to 32k, 32 pages read
        dict(name="select 64x32768", op="select", batch=64, qlen=1, hq=32, hkv=8, d=128, page=64, context=32768, select=32, dtype="bf16"),
        # a 2048-token part of one prompt, with 10k tokens before it
        dict(name="select prompt 2048", op="select", batch=1, qlen=2048, hq=32, hkv=4, d=128, page=64, context=12300, select=16, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _shape(rng, heads):
    while True:
        hkv, group, d = rng.choice(heads), rng.choice([1, 1, 2, 4, 8]), rng.choice([64, 96, 128, 128])
        if hkv * group <= 64 and 3 * 1024 not in (hkv * group * d, hkv * (group + 2) * d):
            return dict(hq=hkv * group, hkv=hkv, d=d, page=rng.choice([16, 32, 64, 64, 128]), dtype=rng.choice(["bf16"] * 5 + ["fp32"]))


def _draw(rng):
    op = rng.choice(["append", "prefix", "select"])
    c = dict(op=op, **_shape(rng, [1, 2, 4, 8, 12, 16, 32]))
    if op == "append":
        kind = rng.choice(["decode", "prompt"])
        c.update(kind=kind, tokens=_log(rng, 1, 512) if kind == "decode" else _log(rng, 16, 16384),
                 rot=rng.choice([c["d"], c["d"], c["d"] // 2]), summary=rng.random() < 0.6, packed=rng.random() < 0.6,
                 interleaved=rng.random() < 0.3)
    elif op == "prefix":
        qlen = 1 if rng.random() < 0.6 else _log(rng, 2, 128)
        c.update(batch=_log(rng, 1, 256 if qlen == 1 else 32), qlen=qlen, prefix=_log(rng, 64, 32768), suffix=qlen + _log(rng, 1, 1024))
    else:
        qlen = 1 if rng.random() < 0.6 else _log(rng, 2, 2048)
        c.update(batch=_log(rng, 1, 128) if qlen == 1 else max(1, min(8, 2048 // qlen)), qlen=qlen,
                 context=qlen + _log(rng, 256, 32768), select=rng.choice([4, 8, 16, 32, 64]))
    return c


def _cost(c):
    w = work(c)
    return max(w["bytes"] / 6.5e12, w["flops"] / (1.5e15 if c["dtype"] == "bf16" else 5e13))


def draw(rng):
    most = {}
    for c in listed():
        most[c["op"]] = max(most.get(c["op"], 0.0), _cost(c))
    while True:
        c = _draw(rng)
        if 3 * 1024 in c.values() or _cost(c) > most[c["op"]]:
            continue
        if c["op"] == "prefix" and 4 * c["batch"] * c["qlen"] * c["hq"] * (c["prefix"] + c["suffix"]) > 1.2e9:
            continue
        if c["op"] == "select" and 4 * c["batch"] * c["qlen"] * c["hkv"] * min(c["select"] * c["page"], c["context"]) * c["d"] > 4.5e9:
            continue
        if c["op"] == "select" and 4 * c["batch"] * c["context"] * c["hkv"] * c["d"] > 1.8e10:
            continue
        return c


def work(case):
    """Bytes and operations that the operator cannot do without: every input that it needs read once, every output
    written once.  Ragged lengths count with their mean."""
    c, e = case, 4 if case["dtype"] == "fp32" else 2
    if c["op"] == "append":
        rows = c["tokens"] * (c["hq"] + 2 * c["hkv"])
        b = 2.0 * rows * c["d"] * e + c["tokens"] * (c["rot"] * 4 + 12)
        pages = c["tokens"] if c["kind"] == "decode" else c["tokens"] / c["page"]
        if c["summary"]:
            b += pages * c["hkv"] * 2 * c["d"] * (2 if c["kind"] == "decode" else 1)
        return {"bytes": b, "flops": 3.0 * c["tokens"] * (c["hq"] + c["hkv"]) * c["rot"]}
    tokens = c["batch"] * (c["qlen"] if c["op"] == "select" else (1 + c["qlen"]) / 2)
    io = 2.0 * tokens * c["hq"] * c["d"] * e
    kv = 2.0 * c["hkv"] * c["d"] * e
    if c["op"] == "prefix":
        own_len = (c["qlen"] + c["suffix"]) / 2
        return {"bytes": io + kv * (c["prefix"] + c["batch"] * own_len),
                "flops": 4.0 * tokens * c["hq"] * c["d"] * (c["prefix"] + own_len - (c["qlen"] - 1) / 4)}
    mean = 0.75 * (c["context"] - c["qlen"]) + c["qlen"]
    keys = min(c["select"] * c["page"], mean)
    pages = mean / c["page"]
    return {"bytes": io + kv * min(tokens * keys, c["batch"] * mean) + c["batch"] * pages * c["hkv"] * 2 * c["d"] + tokens * c["hkv"] * c["select"] * 4,
            "flops": 4.0 * tokens * c["hq"] * c["d"] * keys + 4.0 * tokens * c["hkv"] * c["d"] * pages}


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
    return {"append": _prepare_append, "prefix": _prepare_prefix, "select": _prepare_select}[case["op"]](case, _gen(seed))


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
        qkv = _normal((T, c["hq"] + 2 * c["hkv"], c["d"]), dt, g)
        q, k, v = qkv.split([c["hq"], c["hkv"], c["hkv"]], dim=1)
    else:
        q, k, v = (_normal((T, h, c["d"]), dt, g) for h in (c["hq"], c["hkv"], c["hkv"]))
    shape = (num_pages, c["hkv"], page, c["d"])
    s = dict(case=c, q=q, k=k, v=v, slots=slots, positions=positions.to(torch.int32), cos=angle.cos().float(), sin=angle.sin().float(),
             k_cache=_normal(shape, dt, g), v_cache=_normal(shape, dt, g), summary=None, summary_scale=None)
    if c["summary"]:
        s["summary"] = torch.stack([_ints(-70, 0, (num_pages, c["hkv"], c["d"]), g), _ints(0, 70, (num_pages, c["hkv"], c["d"]), g)], dim=2).to(torch.int8)
        s["summary_scale"] = 20.0 + 10.0 * torch.rand(c["hkv"], generator=g, device="cuda")
    return s


def _ragged(lo, hi, n, g):
    """n lengths between lo and hi, the first of them hi."""
    v = _ints(lo, hi, (n,), g)
    v[0] = hi
    return v


def _queries(c, g):
    if c["qlen"] == 1:
        return torch.ones(c["batch"], dtype=torch.int64, device="cuda"), None
    # the first has the most; the others lie between, the same for every seed, so that the batch has one size
    i = torch.arange(c["batch"], device="cuda")
    n = c["qlen"] - (c["qlen"] - 1) * (i * 5 % c["batch"]) // c["batch"]
    return n, torch.cat([n.new_zeros(1), n.cumsum(0)]).to(torch.int32)


def _prepare_prefix(c, g):
    B, page, dt = c["batch"], c["page"], DTYPES[c["dtype"]]
    n, q_start = _queries(c, g)
    tokens = int(n.sum())
    lens = n + (_ints(0, 1 << 20, (B,), g) * (c["suffix"] - n)) // (1 << 20)
    n_pre, n_own = -(-c["prefix"] // page), -(-c["suffix"] // page)
    num_pages = n_pre + B * n_own + 1
    perm = torch.randperm(num_pages, generator=g, device="cuda").to(torch.int32)
    shape = (num_pages, c["hkv"], page, c["d"])
    return dict(case=c, q=_normal((tokens, c["hq"], c["d"]), dt, g, 1.5), k_cache=_normal(shape, dt, g), v_cache=_normal(shape, dt, g),
                prefix_pages=perm[:n_pre].contiguous(), page_table=perm[n_pre:n_pre + B * n_own].reshape(B, n_own).contiguous(),
                kv_lens=lens.to(torch.int32), q_start=q_start, scale=c["d"] ** -0.5)


def _prepare_select(c, g):
    B, page, dt = c["batch"], c["page"], DTYPES[c["dtype"]]
    n = torch.full((B,), c["qlen"], dtype=torch.int64, device="cuda")
    q_start = None if c["qlen"] == 1 else torch.arange(B + 1, device="cuda", dtype=torch.int32) * c["qlen"]
    lens = n + _ragged((c["context"] - c["qlen"]) // 2, c["context"] - c["qlen"], B, g)
    width = -(-c["context"] // page)
    num_pages = B * width + 1
    perm = torch.randperm(num_pages, generator=g, device="cuda").to(torch.int32)
    shape = (num_pages, c["hkv"], page, c["d"])
    k_cache, v_cache = _normal(shape, dt, g), _normal(shape, dt, g)
    k_cache += _normal((num_pages, c["hkv"], 1, c["d"]), dt, g, 0.5)  # the tokens of a page have something in common
    scale = torch.full((c["hkv"],), 28.0, device="cuda")
    summary = torch.empty(num_pages, c["hkv"], 2, c["d"], dtype=torch.int8, device="cuda")
    step = max(1, (1 << 28) // (c["hkv"] * page * c["d"]))
    for p in range(0, num_pages, step):
        k8 = (k_cache[p:p + step].float() * scale[:, None, None]).round().clamp(-127, 127)
        summary[p:p + step, :, 0] = k8.amin(2).to(torch.int8)
        summary[p:p + step, :, 1] = k8.amax(2).to(torch.int8)
    return dict(case=c, q=_normal((B * c["qlen"], c["hq"], c["d"]), dt, g, 1.5), k_cache=k_cache, v_cache=v_cache, summary=summary,
                page_table=perm[:B * width].reshape(B, width).contiguous(), kv_lens=lens.to(torch.int32), q_start=q_start,
                scale=c["d"] ** -0.5)


# ---- one pass

def run(state):
    if own:
        from paper_2603_08343_b200 import attention as A
        s, c = state, state["case"]
        if c["op"] == "append":
            q = A.kv_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["slots"], positions=s["positions"], cos=s["cos"], sin=s["sin"],
                            q=s["q"], summary=s["summary"], summary_scale=s["summary_scale"], interleaved=c["interleaved"])
            return _append_outputs(s, q)
        if c["op"] == "prefix":
            return A.shared_prefix_attention(s["q"], s["k_cache"], s["v_cache"], s["prefix_pages"], c["prefix"], s["page_table"], s["kv_lens"],
                                             q_start=s["q_start"], max_q_len=c["qlen"], scale=s["scale"])
        return A.selected_page_attention(s["q"], s["k_cache"], s["v_cache"], s["summary"], s["page_table"], s["kv_lens"], c["select"],
                                         q_start=s["q_start"], max_q_len=c["qlen"], scale=s["scale"])
    return {"append": _append, "prefix": _prefix, "select": _select}[state["case"]["op"]](state)


def _append_outputs(s, q):
    out = {"q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    if s["summary"] is not None:
        out["summary"] = s["summary"]
    return out


def _rotate(x, cos, sin, rot, interleaved):
    """x [T, H, D] in 32 bits; the first `rot` channels turn by the position's angles, in pairs (i, i + rot/2) or (2i, 2i + 1)."""
    h = rot // 2
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :h], x[..., h:rot])
    ra, rb = a * cos - b * sin, b * cos + a * sin
    r = torch.stack([ra, rb], dim=-1).flatten(-2) if interleaved else torch.cat([ra, rb], dim=-1)
    return torch.cat([r, x[..., rot:]], dim=-1)


def _append(s):
    c = s["case"]
    dt, page = s["k"].dtype, c["page"]
    cos, sin = s["cos"][s["positions"].long()][:, None], s["sin"][s["positions"].long()][:, None]
    q = _rotate(s["q"].float(), cos, sin, c["rot"], c["interleaved"]).to(dt)
    k = _rotate(s["k"].float(), cos, sin, c["rot"], c["interleaved"]).to(dt)
    live = s["slots"] >= 0
    slots, k, v = s["slots"][live], k[live], s["v"][live]
    at, off = slots // page, slots % page
    s["k_cache"][at, :, off] = k
    s["v_cache"][at, :, off] = v
    if s["summary"] is not None:
        k8 = (k.float() * s["summary_scale"][:, None]).round().clamp(-127, 127).to(torch.int32)
        old = s["summary"].to(torch.int32)
        fresh = at[off == 0]  # a page begins anew with its first token
        old[fresh, :, 0] = 127
        old[fresh, :, 1] = -127
        where = at[:, None, None].expand_as(k8)
        s["summary"][:, :, 0] = old[:, :, 0].scatter_reduce(0, where, k8, "amin").to(torch.int8)
        s["summary"][:, :, 1] = old[:, :, 1].scatter_reduce(0, where, k8, "amax").to(torch.int8)
    return _append_outputs(s, q)


def _rows(pages, cache):
    """cache rows of the pages [..., n] of one table: [..., Hkv, n * page, D] in 32 bits."""
    x = cache[pages.long()].float()  # [..., n, Hkv, page, D]
    return x.movedim(-3, -4).flatten(-3, -2)


def _places(s):
    """Each sequence's tokens side by side: token numbers [B, n] and which of them there are."""
    B = s["page_table"].shape[0]
    n = s["case"]["qlen"]
    if s["q_start"] is None:
        return torch.arange(B, device="cuda")[:, None], torch.ones(B, 1, dtype=torch.bool, device="cuda")
    start = s["q_start"].long()
    at = start[:-1, None] + torch.arange(n, device="cuda")
    return at, at < start[1:, None]


def _prefix(s):
    c = s["case"]
    T, hq, d = s["q"].shape
    hkv = c["hkv"]
    G = hq // hkv
    q = s["q"].float() * s["scale"]
    # the prefix: all tokens against the same keys
    kp, vp = (_rows(s["prefix_pages"], x)[:, :c["prefix"]] for x in (s["k_cache"], s["v_cache"]))  # [Hkv, L, D]
    qp = q.view(T, hkv, G, d).transpose(0, 1).reshape(hkv, T * G, d)
    sp = torch.matmul(qp, kp.transpose(1, 2))                                                       # [Hkv, T*G, L]
    # each sequence's own keys, a token seeing those up to itself
    ko, vo = (_rows(s["page_table"], x) for x in (s["k_cache"], s["v_cache"]))                      # [B, Hkv, N, D]
    at, live = _places(s)
    B, n = at.shape
    qo = q[at.clamp(max=T - 1)].view(B, n, hkv, G, d).permute(0, 2, 1, 3, 4).reshape(B, hkv, n * G, d)
    so = torch.matmul(qo, ko.transpose(2, 3)).view(B, hkv, n, G, -1)
    last = s["kv_lens"].long()[:, None] - live.sum(1, keepdim=True) + torch.arange(n, device="cuda")  # [B, n]
    seen = torch.arange(so.shape[-1], device="cuda") <= last[..., None]                             # [B, n, N]
    so = so.masked_fill(~seen[:, None, :, None], -math.inf)
    # one softmax over both
    back = torch.arange(B, device="cuda")[:, None].expand(B, n)[live], torch.arange(n, device="cuda").expand(B, n)[live]
    mo = so.amax(-1)[back[0], :, back[1]]                                                           # [T, Hkv, G]
    mp = sp.amax(-1).view(hkv, T, G).transpose(0, 1)
    m = torch.maximum(mo, mp)
    pp = torch.exp(sp - m.transpose(0, 1).reshape(hkv, T * G, 1))
    mo_pad = torch.zeros(B, n, hkv, G, device="cuda")
    mo_pad[back] = m
    po = torch.exp(so - mo_pad.permute(0, 2, 1, 3)[..., None])
    lp = pp.sum(-1).view(hkv, T, G).transpose(0, 1)
    lo = po.sum(-1)[back[0], :, back[1]]
    op = torch.matmul(pp, vp).view(hkv, T, G, d).transpose(0, 1)
    vo = vo.masked_fill(torch.arange(vo.shape[2], device="cuda")[:, None] >= s["kv_lens"].long()[:, None, None, None], 0.0)
    oo = torch.matmul(po.view(B, hkv, n * G, -1), vo).view(B, hkv, n, G, d)[back[0], :, back[1]]
    return ((op + oo) / (lp + lo)[..., None]).reshape(T, hq, d).to(s["q"].dtype)


def _select(s):
    c = s["case"]
    T, hq, d = s["q"].shape
    hkv, page = c["hkv"], c["page"]
    G, B = hq // hkv, s["page_table"].shape[0]
    n = T // B
    q = s["q"].float().view(T, hkv, G, d)
    # whole-number queries, and the score of each page: the largest product that its summary allows
    top = q.abs().amax((2, 3), keepdim=True)
    q8 = (q * torch.where(top > 1e-30, 127.0 / top, torch.zeros_like(top))).round()
    up, down = (q8.clamp(min=0).sum(2), q8.clamp(max=0).sum(2))                       # [T, Hkv, D]
    box = s["summary"][s["page_table"].long()].float()                                # [B, P, Hkv, 2, D]
    up, down = (x.view(B, n, hkv, d).transpose(1, 2) for x in (up, down))             # [B, Hkv, n, D]
    score = torch.matmul(up, box[:, :, :, 1].permute(0, 2, 3, 1)) + torch.matmul(down, box[:, :, :, 0].permute(0, 2, 3, 1))
    last = s["kv_lens"].long()[:, None] - n + torch.arange(n, device="cuda")          # [B, n] the token's own place
    mine = (last // page)[:, None, :, None]
    P = score.shape[-1]
    index = torch.arange(P, device="cuda")
    score = score.masked_fill(index >= mine, -math.inf)
    best, order = torch.sort(score, dim=-1, descending=True, stable=True)             # ties: the lowest page first
    order = order.masked_fill(best == -math.inf, P)[..., :c["select"] - 1]
    chosen = torch.cat([order, mine.expand(B, hkv, n, 1)], dim=-1).sort(dim=-1).values
    if chosen.shape[-1] < c["select"]:
        chosen = torch.nn.functional.pad(chosen, (0, c["select"] - chosen.shape[-1]), value=P)
    chosen = chosen.transpose(1, 2).reshape(T, hkv, c["select"])                      # P stands for none
    # attention over what was chosen
    seq = torch.arange(T, device="cuda") // n
    physical = s["page_table"].long()[seq[:, None, None], chosen.clamp(max=P - 1)]
    head = torch.arange(hkv, device="cuda")[None, :, None]
    k, v = (x[physical, head].float().flatten(2, 3) for x in (s["k_cache"], s["v_cache"]))  # [T, Hkv, S*page, D]
    where = (chosen[..., None] * page + torch.arange(page, device="cuda")).flatten(2)
    seen = where <= last.reshape(T)[:, None, None]
    w = torch.matmul(q, k.transpose(2, 3)) * s["scale"]
    w = w.masked_fill(~seen[:, :, None], -math.inf)
    w = torch.exp(w - w.amax(-1, keepdim=True))
    v = v.masked_fill(~seen[..., None], 0.0)
    out = torch.matmul(w, v) / w.sum(-1, keepdim=True)
    return out.reshape(T, hq, d).to(s["q"].dtype), chosen.masked_fill(chosen == P, -1).to(torch.int32)


# ---- the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "prefix": _exact_prefix, "select": _exact_select}[case["op"]](case, s)


def _exact_append(c, s):
    half = c["rot"] // 2
    i = torch.arange(half, device="cuda")
    first, second = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + half)
    w = torch.complex(s["cos"].double(), s["sin"].double())[s["positions"].long()].unsqueeze(1)
    turned = []
    for x in (s["q"], s["k"]):
        y = x.double().clone()
        z = torch.complex(y[..., first], y[..., second]) * w
        y[..., first], y[..., second] = z.real, z.imag
        turned.append(y)
    kc, vc = s["k_cache"].double(), s["v_cache"].double()
    for h in range(c["hkv"]):
        for new, cache in ((turned[1], kc), (s["v"].double(), vc)):
            flat = cache[:, h].reshape(-1, c["d"])
            t = (s["slots"] >= 0).nonzero()[:, 0]
            flat[s["slots"][t]] = new[t, h]
            cache[:, h] = flat.view(-1, c["page"], c["d"])
    out = {"q": turned[0], "k_cache": kc, "v_cache": vc}
    if c["summary"]:
        out["summary"] = None  # whole numbers
    return out


def _exact_prefix(c, s):
    G = c["hq"] // c["hkv"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    lens = s["kv_lens"].tolist()
    starts = list(range(c["batch"] + 1)) if s["q_start"] is None else s["q_start"].tolist()
    for h in range(c["hkv"]):
        kp = s["k_cache"][s["prefix_pages"].long(), h].reshape(-1, c["d"])[:c["prefix"]].double()
        vp = s["v_cache"][s["prefix_pages"].long(), h].reshape(-1, c["d"])[:c["prefix"]].double()
        for b in range(c["batch"]):
            t0, t1 = starts[b], starts[b + 1]
            pages = s["page_table"][b].long()
            k = torch.cat([kp, s["k_cache"][pages, h].reshape(-1, c["d"])[:lens[b]].double()])
            v = torch.cat([vp, s["v_cache"][pages, h].reshape(-1, c["d"])[:lens[b]].double()])
            w = torch.einsum("tgd,nd->tgn", s["q"][t0:t1, h * G:(h + 1) * G].double(), k) * s["scale"]
            for t in range(t1 - t0):
                w[t, :, c["prefix"] + lens[b] - (t1 - t0) + t + 1:] = -math.inf
            out[t0:t1, h * G:(h + 1) * G] = torch.softmax(w, -1) @ v
    return out


def _exact_select(c, s):
    G, page = c["hq"] // c["hkv"], c["page"]
    step = max(1, min(128, (1 << 27) // (s["page_table"].shape[1] ** 2)))
    if c["batch"] * c["hkv"] * -(-c["qlen"] // step) > 3000:
        return None
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    lens = s["kv_lens"].tolist()
    for b in range(c["batch"]):
        for h in range(c["hkv"]):
            pages = s["page_table"][b].long()
            k = s["k_cache"][pages, h].reshape(-1, c["d"])[:lens[b]].double()
            v = s["v_cache"][pages, h].reshape(-1, c["d"])[:lens[b]].double()
            low, high = s["summary"][pages, h, 0].double(), s["summary"][pages, h, 1].double()
            for t0 in range(0, c["qlen"], step):
                t1 = min(c["qlen"], t0 + step)
                q = s["q"][b * c["qlen"] + t0:b * c["qlen"] + t1, h * G:(h + 1) * G].double()
                # the quantisation is a definition in 32 bits
                top = q.float().abs().flatten(1).amax(1)
                q8 = (q.float() * (127.0 / top)[:, None, None]).round().double()
                score = sum(torch.maximum(q8[:, g, None] * low, q8[:, g, None] * high).sum(-1) for g in range(G))  # [t, P]
                place = lens[b] - c["qlen"] + torch.arange(t0, t1, device="cuda")
                index = torch.arange(len(pages), device="cuda")
                # rank of a page = how many pages go before it
                before = (score[:, None, :] > score[:, :, None]) | ((score[:, None, :] == score[:, :, None]) & (index < index[:, None]))
                before &= (index < (place // page)[:, None])[:, None, :]
                taken = (before.sum(-1) < c["select"] - 1) & (index < (place // page)[:, None]) | (index == (place // page)[:, None])
                key = torch.arange(lens[b], device="cuda")
                seen = taken[:, key // page] & (key <= place[:, None])
                w = torch.einsum("tgd,nd->tgn", q, k) * s["scale"]
                w = w.masked_fill(~seen[:, None], -math.inf)
                out[b * c["qlen"] + t0:b * c["qlen"] + t1, h * G:(h + 1) * G] = torch.softmax(w, -1) @ v
    return out, None
