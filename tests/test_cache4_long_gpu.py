"""Attention over long 4-bit caches, relative to the result: over n keys of even weight it shrinks with the root of n, and whatever
is lost in sums of products shows beside it.

Bounds are of the norm of the difference over the norm of the result.  bf16: 2^-8, the most that rounding the result to bf16 can
come to (about 2^-9.2 where numbers lie evenly).  The other errors are added to it in squares, being independent of it: the weights' 11
bits, up to 2^-11 of products with codes up to 15 of which some 2.3 are left about the mean, 2^-10.7 at most; sums of 64 or 256 truncating
additions, each below 2^-22 of a sum that does not grow but by chance, 2^-14; scores, 2^-19 of scale * sum|q| * spread of the keys, below 2^-11 here.
fp32: 2^-15; weights of 22 bits and the same sums with rounding, below 2^-17; scores 2^-19 of scale * sum|q| * spread < 12 for the queries
taken here, independent from key to key, so that the half of it is ample."""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
BOUND = {BF16: 2.0 ** -8, F32: 2.0 ** -15}


@pytest.fixture(scope="module")
def A():
    from paper_2603_08343_b200 import build
    build.build()
    from paper_2603_08343_b200 import attention
    yield attention
    attention.device_status()


def off(A, q, cache, table, lens, tokens, sample):
    """|out - exact| / |exact| over the sampled sequences, whose tables are all the same; exact by 64 bits from what the cache holds."""
    batch, hkv, d = lens.shape[0], cache.shape[1], q.shape[2]
    group, page = q.shape[1] // hkv, cache.shape[2] * 16
    starts = None if tokens == 1 else (torch.arange(batch + 1, device="cuda") * tokens).int()
    out = A.paged_attention4(q, cache, table, lens, q_start=starts, max_q_len=tokens)
    n = int(lens[0])
    slots = (table[0].long()[:, None] * page + torch.arange(page, device="cuda")).flatten()[:n]
    keys, values = A.kv_read4(cache, slots)
    error = norm = 0.0
    for h in range(hkv):
        k, v = keys[:, h].double(), values[:, h].double()
        for b in sample:
            for t in sorted({0, tokens // 2, tokens - 1}):
                seen = n - tokens + t + 1
                rows = slice(h * group, (h + 1) * group)
                want = torch.softmax(q[b * tokens + t, rows].double() @ k[:seen].T * d ** -0.5, -1) @ v[:seen]
                error += (out[b * tokens + t, rows].double() - want).square().sum().item()
                norm += want.square().sum().item()
    return (error / norm) ** 0.5


def long_cache(A, n, hkv, d, page, seed, keys=None):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    pages = -(-n // page)
    order = torch.randperm(pages, device="cuda", generator=g)
    cache = A.cache4(pages, hkv, page, d)
    for i in range(0, n, 1 << 16):
        at = torch.arange(i, min(n, i + (1 << 16)), device="cuda")
        k, v = (torch.randn(len(at), hkv, d, device="cuda", generator=g) for _ in range(2))
        if keys is not None:
            k = keys(at, k)
        A.kv_append4(k, v, cache, order[at // page] * page + at % page)
    return cache, order.int(), g


# batch, key heads, heads of each, channels, page, tokens of a sequence.  The batch is large, so that a warp (a block) has a long run.
SHAPES = [(128, 4, 4, 128, 64, 1), (256, 2, 8, 64, 128, 1), (128, 4, 2, 96, 16, 1), (32, 2, 4, 96, 64, 4), (32, 4, 3, 128, 32, 5), (32, 4, 8, 64, 64, 2),
          (4, 2, 4, 128, 64, 150), (8, 2, 8, 64, 128, 70), (4, 2, 3, 96, 16, 200), (8, 2, 4, 128, 64, 27), (8, 2, 4, 64, 64, 26)]


@pytest.mark.parametrize("size", [0.0, 0.5, 1.5])
@pytest.mark.parametrize("batch,hkv,group,d,page,tokens", SHAPES)
def test_even_and_uneven_weights_over_131071_keys(A, batch, hkv, group, d, page, tokens, size):
    n = (1 << 17) - 1
    cache, order, g = long_cache(A, n, hkv, d, page, batch + d)
    table, lens = order[None].repeat(batch, 1), torch.full((batch,), n, dtype=torch.int32, device="cuda")
    q = (torch.randn(batch * tokens, hkv * group, d, device="cuda", generator=g) * size).bfloat16()
    assert off(A, q, cache, table, lens, tokens, (0, batch // 2, batch - 1)) <= BOUND[BF16]


@pytest.mark.parametrize("size", [0.0, 0.5])
@pytest.mark.parametrize("batch,hkv,group,d,page,tokens", SHAPES[:6])
def test_fp32_over_131071_keys(A, batch, hkv, group, d, page, tokens, size):
    n = (1 << 17) - 1
    cache, order, g = long_cache(A, n, hkv, d, page, batch + d)
    table, lens = order[None].repeat(batch, 1), torch.full((batch,), n, dtype=torch.int32, device="cuda")
    q = torch.randn(batch * tokens, hkv * group, d, device="cuda", generator=g) * size
    assert off(A, q, cache, table, lens, tokens, (0, batch // 2, batch - 1)) <= BOUND[F32]


@pytest.mark.parametrize("d", [64, 128])
def test_fp32_prompts_of_even_weights(A, d):
    """600 tokens over 262143 keys of one weight: a warp adds up tens of thousands of equal numbers, whose roundings are alike; values about 3, so that
    nothing but the sums' own errors shows."""
    n, batch, hkv, group, page = (1 << 18) - 1, 4, 2, 8, 128
    g = torch.Generator(device="cuda")
    g.manual_seed(d)
    cache = A.cache4(-(-n // page), hkv, page, d)
    for i in range(0, n, 1 << 16):
        k, v = (torch.randn(min(n - i, 1 << 16), hkv, d, device="cuda", generator=g) for _ in range(2))
        A.kv_append4(k, v + 3, cache, torch.arange(i, i + k.shape[0], device="cuda"))
    table, lens = torch.arange(-(-n // page), dtype=torch.int32, device="cuda")[None].repeat(batch, 1), torch.full((batch,), n, dtype=torch.int32, device="cuda")
    q = torch.zeros(batch * 600, hkv * group, d, device="cuda")
    assert off(A, q, cache, table, lens, 600, (0, batch - 1)) <= BOUND[F32]


@pytest.mark.parametrize("batch,hkv,group,d,page,tokens", [(64, 8, 4, 128, 64, 1), (64, 8, 8, 64, 64, 1), (64, 4, 2, 96, 32, 6), (8, 4, 4, 128, 64, 100), (8, 4, 4, 64, 64, 100)])
@pytest.mark.parametrize("course", ["rising", "falling", "a leap"])
def test_scores_that_change_along_the_keys(A, batch, hkv, group, d, page, tokens, course):
    """Scores rise or fall by some 60 (in log2) along 20000 keys, evenly or at once: rows' references move between the times at which sums are put
    aside, and far more than one time."""
    n, rise = 20000, 45.0
    towards = torch.ones(d, device="cuda") / d ** 0.5

    def keys(at, k):
        x = at / n if course == "rising" else 1 - at / n if course == "falling" else (at > 0.6 * n).float()
        return 0.1 * k + (rise * x)[:, None, None] * towards

    cache, order, g = long_cache(A, n, hkv, d, page, batch + d, keys)
    table, lens = order[None].repeat(batch, 1), torch.full((batch,), n, dtype=torch.int32, device="cuda")
    q = (torch.randn(batch * tokens, hkv * group, d, device="cuda", generator=g) * 0.1 + towards * d ** 0.5).bfloat16()
    assert off(A, q, cache, table, lens, tokens, (0, batch // 2, batch - 1)) <= BOUND[BF16]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tokens,d", [(1, 64), (1, 128), (5, 96), (100, 64), (100, 128)])
@pytest.mark.parametrize("kind", ["equal channels", "tiny beside them", "both signs"])
def test_large_values_without_a_step_behind_a_leap_of_the_scores(A, dtype, tokens, d, kind):
    """Rows of equal channels have no step and bring no products that would move a row's reference; their weights, times values of 2^60, stay in range all
    the same, however the scores rise."""
    n, page, batch, hkv, group = 6000, 64, 2, 2, 4
    g = torch.Generator(device="cuda")
    g.manual_seed(tokens + d)
    at = torch.arange(n, device="cuda")
    towards = torch.ones(d, device="cuda") / d ** 0.5
    k = ((at > 64).float() * 60.0)[:, None, None] * towards + 0.05 * torch.randn(n, hkv, d, device="cuda", generator=g)   # 86 in log2, behind the first step
    v = (torch.rand(n, hkv, 1, device="cuda", generator=g) + 0.5).bfloat16().float().mul(2.0 ** 60).expand(n, hkv, d).contiguous()
    if kind == "tiny beside them":
        v[::2] = torch.randn(n // 2, hkv, d, device="cuda", generator=g) * 2.0 ** -80
    elif kind == "both signs":
        v[::3] *= -0.5
    cache = A.cache4(-(-n // page), hkv, page, d)
    A.kv_append4(k, v, cache, at)
    table, lens = torch.arange(-(-n // page), dtype=torch.int32, device="cuda")[None].repeat(batch, 1), torch.full((batch,), n, dtype=torch.int32, device="cuda")
    q = (0.05 * torch.randn(batch * tokens, hkv * group, d, device="cuda", generator=g) + towards * d ** 0.5).to(dtype)
    assert off(A, q, cache, table, lens, tokens, (0, batch - 1)) <= (2.0 ** -8 if dtype == BF16 else 2.0 ** -13)
