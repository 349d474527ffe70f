"""Plain 64-bit statements of the serving-attention operators, one loop per definition, for the tests."""
import math

import torch


def rotate(x, positions, cos, sin, interleaved):
    """x [T, H, D] fp64 copy with its first 2 * cos.shape[1] channels turned."""
    x = x.double().clone()
    half = cos.shape[1]
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        c, s = cos[positions.long(), i].double()[:, None], sin[positions.long(), i].double()[:, None]
        xa, xb = x[..., a].clone(), x[..., b].clone()
        x[..., a], x[..., b] = xa * c - xb * s, xb * c + xa * s
    return x


def rotate32(x, positions, cos, sin, interleaved):
    """The same in fp32 with every product and sum rounded on its own, rounded to x's type: the stored value, bit for bit."""
    y = x.float().clone()
    half = cos.shape[1]
    i = torch.arange(half)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    c, s = cos[positions.long()][:, None], sin[positions.long()][:, None]
    xa, xb = y[..., a].clone(), y[..., b].clone()
    y[..., a] = xa * c - xb * s
    y[..., b] = xb * c + xa * s
    return y.to(x.dtype)


def attend(q, k, v, scale):
    """q [G, D], k and v [n, D] -> [G, D]; zeros without keys."""
    if k.shape[0] == 0:
        return torch.zeros(q.shape, dtype=torch.float64)
    w = (q.double() @ k.double().T) * scale
    w = torch.exp(w - w.max(dim=-1, keepdim=True).values)
    return (w @ v.double()) / w.sum(dim=-1, keepdim=True)


def keys_of(cache, pages, head, n):
    """The first n rows of a sequence's pages for one key head."""
    page = cache.shape[2]
    need = -(-n // page) if n > 0 else 0
    if need == 0:
        return cache.new_zeros(0, cache.shape[3])
    return torch.cat([cache[int(p), head] for p in pages[:need]])[:n]


def spans(q_start, tokens, batch):
    return [(b, b + 1) for b in range(batch)] if q_start is None else [(int(q_start[b]), int(q_start[b + 1])) for b in range(batch)]


def prefix_attention(q, k_cache, v_cache, prefix_pages, prefix_len, page_table, kv_lens, q_start, scale):
    T, hq, d = q.shape
    hkv = k_cache.shape[1]
    G = hq // hkv
    out = torch.zeros(T, hq, d, dtype=torch.float64)
    for b, (t0, t1) in enumerate(spans(q_start, T, page_table.shape[0])):
        for t in range(t0, t1):
            seen = int(kv_lens[b]) - (t1 - t0) + (t - t0) + 1
            for h in range(hkv):
                k = torch.cat([keys_of(k_cache, prefix_pages, h, prefix_len), keys_of(k_cache, page_table[b], h, max(0, seen))])
                v = torch.cat([keys_of(v_cache, prefix_pages, h, prefix_len), keys_of(v_cache, page_table[b], h, max(0, seen))])
                out[t, h * G:(h + 1) * G] = attend(q[t, h * G:(h + 1) * G], k, v, scale)
    return out


def whole_queries(q):
    """q [G, D] -> the whole-number queries of the score (a definition in 32 bits)."""
    top = q.float().abs().max()
    if not top > 1e-30:
        return torch.zeros(q.shape, dtype=torch.int64)
    return (q.float() * (torch.reciprocal(top) * 127.0)).round().to(torch.int64)


def choose(q, summary, pages, head, own, select):
    """The pages that a query reads: `own` and the best select - 1 before it."""
    q8 = whole_queries(q)
    score = []
    for i in range(own):
        low, high = summary[int(pages[i]), head].to(torch.int64)
        score.append(int(torch.maximum(q8 * low, q8 * high).sum()))
    best = sorted(range(own), key=lambda i: (-score[i], i))[:select - 1]
    return sorted(best) + [own]


def select_attention(q, k_cache, v_cache, summary, page_table, kv_lens, select, q_start, scale):
    T, hq, d = q.shape
    hkv, page = k_cache.shape[1], k_cache.shape[2]
    G = hq // hkv
    out = torch.zeros(T, hq, d, dtype=torch.float64)
    read = torch.full((T, hkv, select), -1, dtype=torch.int32)
    for b, (t0, t1) in enumerate(spans(q_start, T, page_table.shape[0])):
        for t in range(t0, t1):
            place = int(kv_lens[b]) - (t1 - t0) + (t - t0)
            if place < 0:
                continue
            for h in range(hkv):
                own = place // page
                taken = choose(q[t, h * G:(h + 1) * G], summary, page_table[b], h, own, select)
                read[t, h, :len(taken)] = torch.tensor(taken, dtype=torch.int32)
                n = (len(taken) - 1) * page + place % page + 1
                rows = [int(page_table[b, i]) for i in taken]
                out[t, h * G:(h + 1) * G] = attend(q[t, h * G:(h + 1) * G], keys_of(k_cache, rows, h, n), keys_of(v_cache, rows, h, n), scale)
    return out, read


def page_summary(k_cache, scale, lens=None):
    """Least and largest whole values of each page; lens[p]: how many places of page p count (default all)."""
    k8 = (k_cache.float() * scale[:, None, None]).round().clamp(-127, 127)
    out = torch.zeros(k_cache.shape[0], k_cache.shape[1], 2, k_cache.shape[3], dtype=torch.int8)
    for p in range(k_cache.shape[0]):
        n = k_cache.shape[2] if lens is None else int(lens[p])
        if n:
            out[p, :, 0] = k8[p, :, :n].amin(1).to(torch.int8)
            out[p, :, 1] = k8[p, :, :n].amax(1).to(torch.int8)
    return out


def tolerance(dtype, values):
    """Bound on |out - exact| given the largest |value| of the row's keys' values V (every output is a weighted mean of
    values, so its terms are at most V).  bf16: the weights are rounded to bf16 (relative 2^-8 at most, and their sum is
    not, so at most 2^-8 V) and the result is rounded once (2^-8 V); scores and sums in fp32 add less than
    2^-12 V.  fp32: scores to about 2^-20 relative of |q||k| (at most a few tens), so weights to 2^-15; 2^-14 V covers it."""
    return values * (2 * 2 ** -8 + 2 ** -12 if dtype == torch.bfloat16 else 2 ** -14)


def inverse_frequencies(rot, max_pos):
    inv = 10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64) * 2 / rot)
    angle = torch.arange(max_pos, dtype=torch.float64)[:, None] * inv
    return angle.cos().float(), angle.sin().float()


__all__ = [n for n in dir() if not n.startswith("_")] + ["math"]
