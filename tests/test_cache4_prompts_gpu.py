"""Long prompts over the 4-bit cache (the tcgen05 kernel) against the statement in 64 bits, on the GPU; the sizes are those from which a call
takes that kernel (test_cache4_plan.py)."""
import math

import pytest
import torch

import cache4_ref as C

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    from paper_2603_08343_b200 import build
    build.build()
    from paper_2603_08343_b200 import attention
    yield attention
    attention.device_status()


def made(A, lens, counts, hq, hkv, d, page, seed=0, spread=1.0, values=1.0):
    """Sequences appended through the public call on poisoned pages; what they hold, on the GPU."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    width = max(1, max(-(-n // page) for n in lens))
    perm = torch.randperm(len(lens) * width, device="cuda", generator=g).int()
    table = perm.reshape(len(lens), width).contiguous()
    cache = A.cache4(len(lens) * width, hkv, page, d).fill_(255)
    held = []
    for b, n in enumerate(lens):
        i = torch.arange(n, device="cuda")
        slots = table[b].long()[i // page] * page + i % page
        k = (torch.randn(n, hkv, d, device="cuda", generator=g) + torch.randn(hkv, d, device="cuda", generator=g)) * spread
        v = torch.randn(n, hkv, d, device="cuda", generator=g) * values
        if n:
            A.kv_append4(k, v, cache, slots)
        held.append(A.kv_read4(cache, slots))               # (bit for bit what the definition says: test_cache4_gpu.py)
    q = torch.randn(sum(counts), hq, d, device="cuda", generator=g).bfloat16()
    start = torch.tensor([0] + counts).cumsum(0).int().cuda()
    return q, cache, table, torch.tensor(lens).int().cuda(), start, held


def statement(q, held, lens, counts, scale):
    """[T, Hq, D] and the received weight of each sequence [Hkv, n], in 64 bits."""
    T, hq, d = q.shape
    out, received, t0 = torch.zeros(T, hq, d, dtype=torch.float64, device="cuda"), [], 0
    for (k, v), n, c in zip(held, lens, counts):
        hkv = k.shape[1]
        place = n - c + torch.arange(c, device="cuda")
        got = torch.zeros(hkv, n, dtype=torch.float64, device="cuda")
        if n and c:
            for h in range(hkv):
                G = hq // hkv
                w = torch.einsum("tgd,nd->tgn", q[t0:t0 + c, h * G:(h + 1) * G].double(), k[:, h].double()) * scale
                w = w.masked_fill((torch.arange(n, device="cuda") > place[:, None])[:, None], -math.inf)
                w = torch.softmax(w, -1).nan_to_num(0.0)   # (rows that see nothing)
                out[t0:t0 + c, h * G:(h + 1) * G] = w @ v[:, h].double()
                got[h] = w.sum((0, 1))
        received.append(got)
        t0 += c
    return out, received


def bound(q, held, scale):
    ks, vs = [k for k, _ in held if k.numel()], [v for _, v in held if v.numel()]
    return C.tolerance(q.cpu(), max((k.amax(-1) - k.amin(-1)).max().item() for k in ks), max(v.abs().max().item() for v in vs), scale)


@pytest.mark.parametrize("d,hq,hkv,page,lens,counts", [
    (128, 32, 8, 64, [5000], [600]),                       # one prompt; the last unit has rows of one tile alone
    (128, 8, 2, 128, [16001, 9000, 700], [513, 1, 700]),   # a prompt from its start, a single token, odd lengths
    (96, 12, 4, 32, [7000, 0, 40, 4000], [800, 3, 64, 1]), # none, fewer keys than tokens
    (64, 16, 16, 16, [3000, 2999], [900, 411]),            # a row a head
    (64, 64, 1, 64, [12000], [77]),                        # 64 rows a token
])
def test_prompts(A, d, hq, hkv, page, lens, counts):
    q, cache, table, kv, start, held = made(A, lens, counts, hq, hkv, d, page, seed=d + hq)
    scale = d ** -0.5
    got = A.paged_attention4(q, cache, table, kv, q_start=start, max_q_len=max(counts))
    want, received = statement(q, held, lens, counts, scale)
    assert (got.double() - want).abs().max().item() <= bound(q, held, scale)
    out, weights = A.paged_attention4(q, cache, table, kv, q_start=start, max_q_len=max(counts),
                                      weights_out=torch.empty(len(lens), hkv, table.shape[1] * page, device="cuda"))
    assert torch.equal(out, got)
    for b, n in enumerate(lens):
        # (weights within 1e-4 of themselves, sums of many of them in fp32)
        assert ((weights[b, :, :n].double() - received[b]).abs() <= 1e-4 * received[b] + 1e-30).all()
        assert (weights[b, :, n:] == 0).all()
    for _ in range(3):
        assert torch.equal(A.paged_attention4(q, cache, table, kv, q_start=start, max_q_len=max(counts)), got)
    A.device_status()


@pytest.mark.parametrize("spread,values", [(0.01, 1e-25), (4.0, 1e20), (1.0, 1e-3)])
def test_keys_and_values_of_any_size(A, spread, values):
    """From all weights alike to few that count; values far from the range of fp16."""
    q, cache, table, kv, start, held = made(A, [6000], [500], 16, 4, 128, 64, seed=3, spread=spread, values=values)
    got = A.paged_attention4(q, cache, table, kv, q_start=start, max_q_len=500)
    want, _ = statement(q, held, [6000], [500], 128 ** -0.5)
    assert (got.double() - want).abs().max().item() <= bound(q, held, 128 ** -0.5)


@pytest.mark.parametrize("scale", [-0.05, 0.0, 0.2])
def test_any_scale(A, scale):
    q, cache, table, kv, start, held = made(A, [5000], [500], 16, 4, 96, 64, seed=4)
    got = A.paged_attention4(q, cache, table, kv, q_start=start, max_q_len=500, scale=scale)
    want, _ = statement(q, held, [5000], [500], scale)
    assert (got.double() - want).abs().max().item() <= bound(q, held, abs(scale))


def test_bad_rows_reach_only_who_sees_them(A):
    n, c = 5000, 600
    q, cache, table, kv, start, held = made(A, [n], [c], 8, 2, 128, 64, seed=5)
    args = dict(q_start=start, max_q_len=c)
    clean = A.paged_attention4(q, cache, table, kv, **args)
    at = n - 250                                           # the place of token 350
    slot = table[0, at // 64].long()[None] * 64 + at % 64
    for which in range(2):
        k, v = (x[at:at + 1].clone() for x in held[0])
        (v if which else k)[0, 0, 9] = math.nan            # of the first key head
        touched = cache.clone()
        A.kv_append4(k, v, touched, slot)
        out = A.paged_attention4(q, touched, table, kv, **args)
        token = c - 250
        assert torch.equal(out[:token, :4], clean[:token, :4]) and torch.equal(out[:, 4:], clean[:, 4:])
        assert torch.isnan(out[token:, :4]).all()
    q2 = q.clone()
    q2[123, 5, 7] = math.inf
    out = A.paged_attention4(q2, cache, table, kv, **args)
    assert torch.isnan(out[123, 5]).any()
    out[123, 5] = clean[123, 5]
    assert torch.equal(out, clean)


def test_captured_and_beside_another_stream(A):
    q, cache, table, kv, start, held = made(A, [5000], [600], 32, 8, 128, 64, seed=6)
    args = dict(q_start=start, max_q_len=600)
    alone = A.paged_attention4(q, cache, table, kv, **args)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = A.paged_attention4(q, cache, table, kv, **args)
    other = torch.cuda.Stream()
    beside = []
    for _ in range(5):
        graph.replay()
        beside.append(A.paged_attention4(q, cache, table, kv, stream=other, **args))
    torch.cuda.synchronize()
    assert torch.equal(out, alone) and all(torch.equal(x, alone) for x in beside)
    kv.fill_(4321)                                         # the graph follows its inputs
    graph.replay()
    want, _ = statement(q, [(held[0][0][:4321], held[0][1][:4321])], [4321], [600], 128 ** -0.5)
    assert (out.double() - want).abs().max().item() <= bound(q, held, 128 ** -0.5)
    A.device_status()


def test_what_is_out_of_range_is_reported(A):
    from paper_2603_08343_b200.binding import WhtError
    q, cache, table, kv, start, _ = made(A, [5000], [600], 32, 8, 128, 64, seed=7)
    bad = table.clone()
    bad[0, 3], bad[0, 40] = -1, 1 << 20
    out = A.paged_attention4(q, cache, bad, kv, q_start=start, max_q_len=600)
    assert torch.isfinite(out).all()
    with pytest.raises(WhtError):
        A.device_status()
    out = A.paged_attention4(q, cache, table, kv, q_start=torch.tensor([5, 590]).int().cuda(), max_q_len=600)
    assert (out[:5] == 0).all() and (out[590:] == 0).all() and (out[5:590] != 0).any(-1).all()
    with pytest.raises(WhtError):
        A.device_status()


def test_offsets_that_make_no_sense_stay_in_bounds(A):
    from paper_2603_08343_b200.binding import WhtError
    q, cache, table, kv, _, _ = made(A, [5000, 4000], [600, 500], 32, 8, 128, 64, seed=8)
    for starts in ((0, 1100, 300), (-7, 600, 1100), (1100, 500, 0), (0, 600, 1 << 30)):
        A.paged_attention4(q, cache, table, kv, q_start=torch.tensor(starts).int().cuda(), max_q_len=600)
        with pytest.raises(WhtError):
            A.device_status()
