"""Plain statements of the 4-bit cache for the tests: how a row is held (in 32 bits, as its definition has it), and attention,
received weight and eviction in 64 bits, one loop per definition."""
import math

import torch

import attention_ref as R


def hold(x):
    """x [..., D] fp32 -> the values that the cache stands for, fp32."""
    x = x.float()
    lo = x.amin(-1).bfloat16().float()
    spread = x.amax(-1) - lo
    step = (spread * torch.tensor(1.0 / 15.0)).bfloat16().float()
    step = torch.where(step >= 2.0 ** -100, step, torch.zeros_like(step))
    bad = ~torch.isfinite(x).all(-1) | ~torch.isfinite(spread)
    inverse = torch.where(step > 0, 1.0 / step, torch.zeros_like(step))
    codes = ((x - lo[..., None]) * inverse[..., None]).round().clamp(0, 15)
    held = lo[..., None] + step[..., None] * codes
    return torch.where(bad[..., None], torch.full_like(held, math.nan), held)


def rotated(x, positions, cos, sin, interleaved):
    """fp32, every product and sum rounded on its own."""
    return R.rotate32(x.float(), positions, cos, sin, interleaved)


def attention(q, keys, values, kv_lens, q_start, scale, weights=None):
    """keys, values: per sequence [n, Hkv, D] of held values.  Returns out [T, Hq, D] and received [B][Hkv][n], fp64."""
    T, hq, d = q.shape
    hkv = keys[0].shape[1]
    G = hq // hkv
    out = torch.zeros(T, hq, d, dtype=torch.float64)
    received = []
    for b, (t0, t1) in enumerate(R.spans(q_start, T, len(keys))):
        n = int(kv_lens[b])
        got = torch.zeros(hkv, n, dtype=torch.float64)
        for t in range(t0, t1):
            seen = n - (t1 - t0) + (t - t0) + 1
            if seen <= 0:
                continue
            for h in range(hkv):
                k, v = keys[b][:seen, h].double(), values[b][:seen, h].double()
                w = torch.softmax(q[t, h * G:(h + 1) * G].double() @ k.T * scale, -1)
                out[t, h * G:(h + 1) * G] = w @ v
                got[h, :seen] += w.sum(0)
        received.append(got)
    return out, received


def keep(weights, n, budget, first, last):
    """weights: list of n floats.  The keys that stay, ascending."""
    if n <= budget:
        return list(range(n))
    always = set(range(min(first, n))) | set(range(max(0, n - last), n))
    rank = sorted((i for i in range(n) if i not in always),
                  key=lambda i: (-(weights[i] if weights[i] == weights[i] else -math.inf), weights[i] != weights[i], i))
    return sorted(always | set(rank[:budget - len(always)]))


def tolerance(q, spread, vmax, scale):
    """Bound on |out - exact|; spread: the largest (max - lo) of a held key row, vmax: the largest |held value|.
    Scores: queries lose at most 2^-22 of the row's largest per channel (fp32: two fp16 terms; bf16: 2^-35), and eight
    or so accumulations of the tensor core truncate to 24 bits, each 2^-23 of a sum of at most sum|q| * spread; the two fp32 operations
    on top add 2^-23 each: below 2^-19 of scale * sum|q| * spread in all, which moves each weight by that factor and the result by
    twice that of vmax.  bf16: the weights times the values' steps (together at most 2 vmax of spread) are rounded to 11 bits (2^-11 relative), and
    the result once (2^-8 of vmax).  fp32: 22 bits, and rounding of the sums: 2^-20 covers both."""
    score = scale * q.double().abs().sum(-1).max().item() * spread * 2 ** -19
    rounding = 2 ** -8 + 2 * 2 ** -11 if q.dtype == torch.bfloat16 else 2 ** -20
    return vmax * (rounding + 2 * score + 2 ** -20) + 1e-37
