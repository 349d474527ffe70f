"""The 4-bit cache on a GPU against plain statements: what is held bit for bit, attention and received weight within bounds from the
kernels' arithmetic, eviction exactly."""
import math

import pytest
import torch

import attention_ref as R
import cache4_ref as C

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    from paper_2603_08343_b200 import build
    build.build()
    from paper_2603_08343_b200 import attention
    return attention


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def poisoned(A, pages, hkv, page, d):
    """Fresh memory may hold anything: all ones are NaN steps and least values."""
    cache = A.cache4(pages, hkv, page, d)
    return cache.fill_(255)


# ---- append and read

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d,rot,interleaved", [(64, 64, False), (64, 0, False), (96, 64, True), (96, 96, False), (128, 128, False), (128, 48, True)])
@pytest.mark.parametrize("page,tokens,hq,hkv", [(16, 1, 4, 4), (64, 77, 15, 5), (128, 300, 8, 1), (32, 18, 64, 1)])
def test_append_holds_what_the_definition_says(A, dtype, d, rot, interleaved, page, tokens, hq, hkv):
    g = gen(tokens * d + rot)
    qkv = torch.randn(tokens, hq + 2 * hkv, d, generator=g)
    qkv[:, :, 3] *= 8.0                                   # a channel of its own size
    qkv = qkv.to(dtype)
    pages = -(-tokens // page) + 3
    slots = torch.randperm(pages * page, generator=g)[:tokens]
    slots[::7] = -1
    if tokens == 1:
        slots[0] = 2 * page + 5
    positions = torch.randint(0, 500, (tokens,), generator=g).int()
    cos, sin = R.inverse_frequencies(rot, 500) if rot else (None, None)
    before = torch.randint(0, 120, (pages, hkv, page // 16, 16 * d + 128), generator=g, dtype=torch.uint8)
    cache = before.cuda()
    old_k, old_v = A.kv_read4(cache, torch.arange(pages * page).cuda())
    dq, dk, dv = qkv.cuda().split([hq, hkv, hkv], 1)
    turn = dict(positions=positions.cuda(), cos=cos.cuda(), sin=sin.cuda()) if rot else {}
    got_q = A.kv_append4(dk, dv, cache, slots.cuda(), q=dq, interleaved=interleaved, **turn)
    new_k, new_v = A.kv_read4(cache, torch.arange(pages * page).cuda())
    A.device_status()
    q, k, v = qkv.split([hq, hkv, hkv], 1)
    if rot:
        want_q = C.rotated(q, positions, cos, sin, interleaved).to(dtype)
        k = C.rotated(k, positions, cos, sin, interleaved)
    else:
        want_q, k = q, k.float()
    assert torch.equal(got_q.cpu(), want_q)
    want_k, want_v = old_k.cpu(), old_v.cpu()
    live = slots >= 0
    want_k[slots[live]], want_v[slots[live]] = C.hold(k[live]), C.hold(v[live].float())
    assert torch.equal(new_k.cpu(), want_k) and torch.equal(new_v.cpu(), want_v)   # the others are left as they were
    # at slots, negative ones as zeros, rounded once to bf16
    rows_k, rows_v = A.kv_read4(cache, slots.cuda(), dtype=torch.bfloat16)
    assert torch.equal(rows_k.cpu(), torch.where(live[:, None, None], want_k[slots], torch.zeros(1)).bfloat16())
    assert torch.equal(rows_v.cpu(), torch.where(live[:, None, None], want_v[slots], torch.zeros(1)).bfloat16())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_of_any_size_and_kind(A, dtype):
    """Rows of equal channels, of one channel that stands out, huge, tiny and subnormal ones, zeros; NaN and infinities."""
    d, rows = 96, []
    g = gen(5)
    base = torch.randn(d, generator=g)
    for scale in (1.0, 1e30, 3e37, 1e-20, 1e-29, 1e-31, 1e-38, 1e-41, 0.0):
        rows += [base * scale, base.abs() * scale, -base.abs() * scale, torch.full((d,), 3.0 * scale), torch.eye(d)[5] * scale, base * scale * 1e-3 + scale]
    x = torch.stack(rows).to(dtype)
    bad = x.clone()[:6]
    bad[0, 3], bad[1, 95], bad[2, 0] = math.nan, math.inf, -math.inf
    bad[3:6] = 3e38
    bad[3:6, 7] = -3e38                                   # a spread beyond fp32
    x = torch.cat([x, bad])[:, None]
    n = x.shape[0]
    cache = poisoned(A, n // 16 + 1, 1, 16, d)
    slots = torch.arange(n)
    A.kv_append4(x.cuda(), x.flip(0).contiguous().cuda(), cache, slots.cuda())
    k, v = A.kv_read4(cache, slots.cuda())
    want = C.hold(x.float())
    assert torch.equal(torch.nan_to_num(k.cpu(), nan=7e7), torch.nan_to_num(want, nan=7e7))
    assert torch.equal(torch.nan_to_num(v.cpu(), nan=7e7), torch.nan_to_num(want.flip(0), nan=7e7))
    # half a step, and what rounding lo and step to bf16 moves a row's end by
    finite = torch.isfinite(want).all(-1)[:, 0]
    x, want = x[finite].double()[:, 0], want[finite].double()[:, 0]
    spread = x.amax(-1) - x.amin(-1)
    bound = spread / 30 + 2 ** -8 * (x.abs().amax(-1) + spread) + 15 * 2 ** -100
    assert ((x - want).abs().amax(-1) <= bound).all()


# ---- attention

def batch(A, d, page, lens, hkv, seed, spread=1.0, extra_pages=2):
    """A poisoned cache with sequences of these lengths, appended through the public call; held rows per sequence."""
    g = gen(seed)
    width = max(1, max(-(-n // page) for n in lens)) + 1
    pages = len(lens) * width + extra_pages
    perm = torch.randperm(pages, generator=g).int()
    table = perm[:len(lens) * width].reshape(len(lens), width).contiguous()
    cache = poisoned(A, pages, hkv, page, d)
    keys, values = [], []
    for b, n in enumerate(lens):
        k = (torch.randn(n, hkv, d, generator=g) + torch.randn(hkv, d, generator=g)) * spread
        v = torch.randn(n, hkv, d, generator=g)
        i = torch.arange(n)
        slots = table[b].long()[i // page] * page + i % page
        if n:
            A.kv_append4(k.cuda(), v.cuda(), cache, slots.cuda())
        keys.append(C.hold(k) if n else k)
        values.append(C.hold(v) if n else v)
    return cache, table, keys, values


def spread_of(rows):
    return max([(r.amax(-1) - r.amin(-1)).max().item() for r in rows if r.numel()] + [0.0])


def vmax_of(rows):
    return max([r.abs().max().item() for r in rows if r.numel()] + [0.0])


def check(A, q, cache, table, lens, counts, keys, values, scale=None, weighed=True):
    d, hkv = q.shape[2], keys[0].shape[1]
    s = d ** -0.5 if scale is None else scale
    q_start = None if counts is None else torch.tensor([0] + counts).cumsum(0).int()
    max_q = 1 if counts is None else max([1] + counts)
    kv = torch.tensor(lens).int()
    args = dict(q_start=None if q_start is None else q_start.cuda(), max_q_len=max_q, scale=scale)
    got = A.paged_attention4(q.cuda(), cache, table.cuda(), kv.cuda(), **args)
    page = cache.shape[2] * 16
    received = torch.rand(len(lens), hkv, table.shape[1] * page, generator=gen(3))
    out, weights = A.paged_attention4(q.cuda(), cache, table.cuda(), kv.cuda(), weights=received.cuda(), **args)
    A.device_status()
    assert torch.equal(got, out)
    want, extra = C.attention(q, keys, values, lens, q_start, s)
    tol = C.tolerance(q, spread_of(keys), vmax_of(values), s)
    assert (got.cpu().double() - want).abs().max().item() <= tol
    group = q.shape[1] // hkv
    for b, n in enumerate(lens):
        assert torch.equal(weights[b, :, n:].cpu(), torch.zeros_like(received[b, :, n:]))
        if n == 0:
            continue
        rows = group * (1 if counts is None else counts[b])
        # each weight is off by the factor of its score's error (2^-19 of scale * sum|q| * spread) and of the row's sum, at most twice that; sums in fp32
        factor = s * q.double().abs().sum(-1).max().item() * spread_of(keys) * 2 ** -18 + 2 ** -20
        bound = extra[b] * factor + (received[b, :, :n] + extra[b]) * 2 ** -22 * max(1, rows) + 1e-30
        assert ((weights[b, :, :n].cpu().double() - received[b, :, :n].double() - extra[b]).abs() <= bound).all()
    return got


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("group,hkv", [(1, 3), (4, 2), (7, 1), (12, 1), (16, 2), (33, 1), (64, 1)])
def test_single_tokens(A, dtype, d, group, hkv):
    lens = [1, 0, 15, 16, 17, 33, 250, 600]
    cache, table, keys, values = batch(A, d, 16 if d == 96 else 64, lens, hkv, d + group)
    q = (torch.randn(len(lens), group * hkv, d, generator=gen(group)) * 1.5).to(dtype)
    check(A, q, cache, table, lens, None, keys, values)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d,page", [(64, 16), (96, 32), (128, 128)])
@pytest.mark.parametrize("group,hkv,counts,lens", [
    (1, 2, [5, 1, 0, 40], [5, 77, 30, 40]),               # a prompt from its start, one token, none, a prompt
    (4, 1, [3, 2, 17], [130, 2, 300]),
    (8, 2, [9, 1], [9, 1]),
    (5, 1, [70], [333]),
    (2, 1, [4, 4], [2, 0]),                               # fewer keys than tokens: the first see nothing
])
def test_several_tokens_a_sequence(A, dtype, d, page, group, hkv, counts, lens):
    cache, table, keys, values = batch(A, d, page, lens, hkv, d + group + 1)
    q = (torch.randn(sum(counts), group * hkv, d, generator=gen(group)) * 1.5).to(dtype)
    got = check(A, q, cache, table, lens, counts, keys, values)
    if lens == [2, 0]:
        assert (got[:2] == 0).all() and (got[4:] == 0).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_long_and_many(A, dtype):
    """Units cut into several runs, runs of several units."""
    lens = [5000, 1, 3, 2047, 0, 4100]
    cache, table, keys, values = batch(A, 128, 64, lens, 2, 1)
    check(A, torch.randn(6, 8, 128, generator=gen(2)).to(dtype), cache, table, lens, None, keys, values)
    lens = [int(n) for n in torch.randint(0, 40, (300,), generator=gen(4))]
    cache, table, keys, values = batch(A, 64, 16, lens, 1, 5)
    check(A, torch.randn(300, 2, 64, generator=gen(6)).to(dtype), cache, table, lens, None, keys, values)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("size", [1e-30, 1e-6, 1.0, 1e6, 1e25])
def test_values_of_any_size(A, dtype, size):
    """Steps of any size, alone and side by side: the weights' range follows the keys that count."""
    d, n = 64, 200
    g = gen(11)
    k = torch.randn(n, 1, d, generator=g)
    for mixed in (False, True):
        v = torch.randn(n, 1, d, generator=g) * size
        if mixed:                                         # a tenth of the keys a thousand times as large, most of them hardly seen
            v[::10] *= 1000.0
            k[::10] *= 0.1
        cache = poisoned(A, 4, 1, 64, d)
        i = torch.arange(n)
        A.kv_append4(k.cuda(), v.cuda(), cache, i.cuda())
        q = torch.randn(3, 4, d, generator=g).to(dtype)
        table = torch.arange(4).int()[None]
        out = A.paged_attention4(q.cuda(), cache, table.cuda(), torch.tensor([n]).int().cuda(), q_start=torch.tensor([0, 3]).int().cuda(), max_q_len=3)
        keys, values = [C.hold(k)], [C.hold(v)]
        want, _ = C.attention(q, keys, values, [n], torch.tensor([0, 3]), d ** -0.5)
        tol = C.tolerance(q, spread_of(keys), vmax_of(values), d ** -0.5)
        assert (out.cpu().double() - want).abs().max().item() <= tol


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_weights_of_a_far_smaller_reference(A, dtype):
    """The first key has a huge value and almost no weight; the others still come out to the last bit that counts."""
    d, n = 128, 64
    g = gen(12)
    q = torch.ones(1, 1, d) * 4.0
    k = torch.randn(n, 1, d, generator=g) * 0.1
    k[0] = -8.0                                           # score -8 * 4 * 128 / sqrt(128) = -362
    k[0, 0, 0] = -7.9
    v = torch.randn(n, 1, d, generator=g)
    v[0] *= 1e20
    cache = poisoned(A, 1, 1, 64, d)
    A.kv_append4(k.cuda(), v.cuda(), cache, torch.arange(n).cuda())
    out = A.paged_attention4(q.to(dtype).cuda(), cache, torch.zeros(1, 1).int().cuda(), torch.tensor([n]).int().cuda())
    want, _ = C.attention(q, [C.hold(k)], [C.hold(v)], [n], None, d ** -0.5)
    tol = C.tolerance(q.to(dtype), spread_of([C.hold(k)[1:]]), vmax_of([C.hold(v)[1:]]), d ** -0.5)
    assert (out.cpu().double() - want).abs().max().item() <= tol


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("factor", [1e-4, 1.0, 40.0, 1e4])
def test_scores_of_any_size(A, dtype, factor):
    """From all weights alike to one key that takes everything.  (The bound grows with the scores: rows whose two best keys lie
    within it are not compared.)"""
    d, lens = 64, [300]
    cache, table, keys, values = batch(A, d, 16, lens, 1, 21)
    q = (torch.randn(1, 4, d, generator=gen(22)) * factor).to(dtype)
    out = A.paged_attention4(q.cuda(), cache, table.cuda(), torch.tensor(lens).int().cuda()).cpu().double()
    want, _ = C.attention(q, keys, values, lens, None, d ** -0.5)
    tol = C.tolerance(q, spread_of(keys), vmax_of(values), d ** -0.5)
    if tol < 0.1 * vmax_of(values):
        assert (out - want).abs().max().item() <= tol
    else:
        score = (q[0].double() @ keys[0][:, 0].double().T * d ** -0.5).sort(-1).values
        clear = score[:, -1] - score[:, -2] > d ** -0.5 * q.double().abs().sum(-1)[0] * spread_of(keys) * 2 ** -18 + 30.0
        assert clear.any()
        assert (out - want)[0, clear].abs().max().item() <= vmax_of(values) * (2 ** -8 + 2 ** -10)


def test_negative_and_zero_scale(A):
    lens = [100, 40]
    cache, table, keys, values = batch(A, 96, 32, lens, 1, 31)
    q = torch.randn(2, 3, 96, generator=gen(32)).bfloat16()
    for scale in (-0.1, 0.0, 0.3):
        got = A.paged_attention4(q.cuda(), cache, table.cuda(), torch.tensor(lens).int().cuda(), scale=scale)
        want, _ = C.attention(q, keys, values, lens, None, scale)
        assert (got.cpu().double() - want).abs().max().item() <= C.tolerance(q, spread_of(keys), vmax_of(values), abs(scale))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("group", [4, 12])
def test_bad_rows_reach_only_who_sees_them(A, dtype, group):
    """A NaN among the keys or values of a later token, in another sequence, or among the queries of another row."""
    d, n, m = 64, 40, 5
    g = gen(41)
    k, v = torch.randn(n, 1, d, generator=g), torch.randn(n, 1, d, generator=g)
    q = torch.randn(m, group, d, generator=g).to(dtype)
    start = torch.tensor([0, m]).int()
    table, lens = torch.arange(3).int()[None], torch.tensor([n]).int()

    def run(k, v, q):
        cache = poisoned(A, 3, 1, 16, d)
        A.kv_append4(k.cuda(), v.cuda(), cache, torch.arange(n).cuda())
        out, w = A.paged_attention4(q.cuda(), cache, table.cuda(), lens.cuda(), q_start=start.cuda(), max_q_len=m,
                                    weights_out=torch.empty(1, 1, 48).cuda())
        return out.cpu(), w.cpu()

    clean, weights = run(k, v, q)
    at = n - 2                                            # the place of the last token but one
    for which in range(2):
        k2, v2 = k.clone(), v.clone()
        (v2 if which else k2)[at, 0, 9] = math.nan
        out, _ = run(k2, v2, q)
        assert torch.equal(out[:m - 2], clean[:m - 2]) and torch.isnan(out[m - 2:]).all()
    q2 = q.clone()
    q2[1, 2, 5] = math.inf
    out, _ = run(k, v, q2)
    assert torch.isnan(out[1, 2]).any()
    out[1, 2] = clean[1, 2]
    assert torch.equal(out, clean)
    assert torch.isfinite(weights).all()


def test_results_repeat(A):
    lens = [3000, 17, 900]
    cache, table, _, _ = batch(A, 128, 64, lens, 2, 51)
    q = torch.randn(3, 8, 128, generator=gen(52)).bfloat16().cuda()
    kv = torch.tensor(lens).int().cuda()
    w = torch.zeros(3, 2, table.shape[1] * 64).cuda()
    first = [x.clone() for x in A.paged_attention4(q, cache, table.cuda(), kv, weights=w)]
    for _ in range(5):
        again = A.paged_attention4(q, cache, table.cuda(), kv, weights=w)
        assert all(torch.equal(x, y) for x, y in zip(first, again))
    # in place, and from nothing
    ws = w.clone()
    out, same = A.paged_attention4(q, cache, table.cuda(), kv, weights=ws, weights_out=ws)
    assert same is ws and torch.equal(ws, first[1])
    fresh = torch.full_like(w, math.nan)
    A.paged_attention4(q, cache, table.cuda(), kv, weights_out=fresh)
    assert torch.equal(fresh, first[1])


def test_strides_and_given_outputs(A):
    lens = [50, 20]
    cache, table, keys, values = batch(A, 64, 16, lens, 2, 61)
    fused = torch.randn(2, 12, 64, generator=gen(62)).bfloat16().cuda()
    q = fused[:, 2:10]
    out = torch.empty(2, 8, 64, dtype=torch.bfloat16, device="cuda")
    got = A.paged_attention4(q, cache, table.cuda(), torch.tensor(lens).int().cuda(), out=out)
    assert got is out
    assert torch.equal(out, A.paged_attention4(q.contiguous(), cache, table.cuda(), torch.tensor(lens).int().cuda()))


def test_tables_wider_than_the_sequences_and_bad_entries_beyond(A):
    lens = [70, 5]
    cache, table, keys, values = batch(A, 64, 16, lens, 1, 71)
    q = torch.randn(2, 4, 64, generator=gen(72)).bfloat16().cuda()
    kv = torch.tensor(lens).int().cuda()
    want = A.paged_attention4(q, cache, table.cuda(), kv)
    wide = torch.full((2, 4000), -5, dtype=torch.int32)
    for b, n in enumerate(lens):
        wide[b, :-(-n // 16)] = table[b, :-(-n // 16)]
    assert torch.equal(A.paged_attention4(q, cache, wide.cuda(), kv), want)
    A.device_status()


# ---- eviction

@pytest.mark.parametrize("d,page", [(64, 16), (96, 32), (128, 64), (128, 128)])
@pytest.mark.parametrize("lens,budget,first,last", [
    ([100, 40, 0, 41, 1], 40, 0, 0), ([100, 40, 0, 41, 1], 40, 4, 16), ([300, 33], 17, 10, 7), ([64], 1, 0, 1), ([500, 20], 499, 3, 3)])
def test_eviction(A, d, page, lens, budget, first, last):
    hkv = 3
    cache, table, keys, values = batch(A, d, page, lens, hkv, budget, extra_pages=len(lens) * (-(-budget // page)) + 1)
    g = gen(7)
    width, width_out = table.shape[1], -(-budget // page)
    free = torch.tensor([p for p in range(cache.shape[0]) if p not in set(table.flatten().tolist())]).int()
    out_table = free[torch.randperm(len(free), generator=g)][:len(lens) * width_out].reshape(len(lens), width_out).contiguous()
    weights = torch.randint(0, 6, (len(lens), hkv, width * page), generator=g).float() / 4    # many ties
    before = cache.clone()
    new, kept, received = A.kv_evict4(cache, table.cuda(), torch.tensor(lens).int().cuda(), weights.cuda(), out_table.cuda(), budget,
                                      keep_first=first, keep_last=last)
    A.device_status()
    assert new.tolist() == [min(n, budget) for n in lens]
    moved = torch.zeros(cache.shape[0], hkv, page, dtype=torch.bool)
    for b, n in enumerate(lens):
        m = min(n, budget)
        i = torch.arange(m)
        slots = out_table[b].long()[i // page] * page + i % page
        k, v = (x.cpu() for x in A.kv_read4(cache, slots.cuda()))
        for h in range(hkv):
            stay = C.keep(weights[b, h, :n].tolist(), n, budget, first, last)
            assert kept[b, h].tolist() == stay + [-1] * (budget - m)
            assert torch.equal(received[b, h].cpu(), torch.cat([weights[b, h, stay], torch.zeros(width_out * page - m)]))
            assert torch.equal(k[:, h], keys[b][stay, h]) and torch.equal(v[:, h], values[b][stay, h])
            moved[slots // page, h, slots % page] = True
    # everything else in the cache is as it was
    rest = (~moved).any(1).flatten().nonzero()[:, 0]
    old, now = A.kv_read4(before, rest.cuda()), A.kv_read4(cache, rest.cuda())
    still = ~moved.transpose(1, 2).reshape(-1, hkv)[rest]
    for x, y in zip(old, now):
        assert torch.equal(torch.nan_to_num(x.cpu()[still], nan=5e5), torch.nan_to_num(y.cpu()[still], nan=5e5))


@pytest.mark.parametrize("n,budget", [(60000, 20000), (5000, 4999), (70001, 3)])
def test_eviction_of_long_sequences(A, n, budget):
    """Longer than shared memory holds; weights of all sizes, zeros of both signs, infinities, NaN (the least of all)."""
    d, page, hkv = 64, 128, 1
    g = gen(n)
    width, width_out = -(-n // page), -(-budget // page)
    cache = torch.randint(0, 100, (width + width_out, hkv, page // 16, 16 * d + 128), generator=g, dtype=torch.uint8).cuda()
    w = torch.exp(6 * torch.randn(n, generator=g))
    w[torch.randperm(n, generator=g)[:n // 3]] = 0.0
    w[::17] = -0.0
    w[5::1001], w[6::1001], w[7::1001] = math.nan, math.inf, -1.0
    weights = torch.zeros(1, 1, width * page)
    weights[0, 0, :n] = w
    table = torch.arange(width).int()[None]
    out_table = torch.arange(width, width + width_out).int()[None]
    new, kept, received = A.kv_evict4(cache, table.cuda(), torch.tensor([n]).int().cuda(), weights.cuda(), out_table.cuda(), budget, keep_first=1, keep_last=1)
    stay = C.keep((w + 0.0).tolist(), n, budget, 1, 1)
    assert new.item() == budget and kept[0, 0].tolist() == stay
    assert torch.equal(received[0, 0, :budget].cpu().nan_to_num(nan=-3.0), w[stay].nan_to_num(nan=-3.0))
    src, dst = torch.tensor(stay), torch.arange(budget) + width * page
    for x, y in zip(A.kv_read4(cache, src.cuda()), A.kv_read4(cache, dst.cuda())):
        assert torch.equal(x, y)


def test_a_run_of_them_together(A):
    """Append, attend with weights, evict into new pages, go on: every step against the statement in 64 bits."""
    d, page, hkv, group, budget, steps = 64, 16, 2, 2, 24, 40
    g = gen(91)
    B, width = 3, 4                                       # room for 64 keys; eviction at 40
    pages = torch.randperm(2 * B * width, generator=g).int().reshape(2, B, width)
    cache = poisoned(A, 2 * B * width, hkv, page, d)
    cos, sin = R.inverse_frequencies(d, 200)
    lens = torch.zeros(B, dtype=torch.int32)
    now = 0
    keys, values = [torch.zeros(0, hkv, d) for _ in range(B)], [torch.zeros(0, hkv, d) for _ in range(B)]
    weights = torch.zeros(B, hkv, width * page).cuda()
    evictions = 0
    for step in range(steps):
        if int(lens.max()) == 30:
            # the statement follows the library's weights: which keys stay is exact for those
            host = weights.cpu()
            new, kept, weights = A.kv_evict4(cache, pages[now].cuda().contiguous(), lens.cuda(), weights, pages[1 - now].cuda().contiguous(), budget,
                                             keep_first=2, keep_last=8)
            for b in range(B):
                stays = [C.keep(host[b, h, :int(lens[b])].tolist(), int(lens[b]), budget, 2, 8) for h in range(hkv)]
                assert kept[b].tolist() == stays
                keys[b] = torch.stack([keys[b][stays[h], h] for h in range(hkv)], 1)
                values[b] = torch.stack([values[b][stays[h], h] for h in range(hkv)], 1)
            lens, now, evictions = new.cpu(), 1 - now, evictions + 1
        qkv = torch.randn(B, (group + 2) * hkv, d, generator=g).bfloat16()
        q, k, v = qkv.split([group * hkv, hkv, hkv], 1)
        at = pages[now].gather(1, (lens // page).long()[:, None])[:, 0].long() * page + lens % page
        position = torch.full((B,), step).int()
        dq, dk, dv = qkv.cuda().split([group * hkv, hkv, hkv], 1)
        q2 = A.kv_append4(dk, dv, cache, at.cuda(), positions=position.cuda(), cos=cos.cuda(), sin=sin.cuda(), q=dq)
        lens = lens + 1
        k, v = C.hold(C.rotated(k, position, cos, sin, False)), C.hold(v.float())
        for b in range(B):
            keys[b], values[b] = torch.cat([keys[b], k[b:b + 1]]), torch.cat([values[b], v[b:b + 1]])
        before = weights.cpu()
        out, weights = A.paged_attention4(q2, cache, pages[now].cuda().contiguous(), lens.cuda(), weights=weights, weights_out=weights)
        want, extra = C.attention(q2.cpu(), keys, values, lens, None, d ** -0.5)
        tol = C.tolerance(q2.cpu(), spread_of(keys), vmax_of(values), d ** -0.5)
        assert (out.cpu().double() - want).abs().max().item() <= tol
        for b in range(B):
            n = int(lens[b])
            got = weights[b, :, :n].cpu().double() - before[b, :, :n].double()
            assert (got - extra[b]).abs().max().item() <= 1e-4
    A.device_status()
    assert evictions == 2
