"""The 4-bit cache at the edges of its calls: empty ones, tokens of no sequence, what is out of range, other streams, graphs, caches past
4 GiB, wide tables, refusals."""
import math

import pytest
import torch

import attention_ref as R
import cache4_ref as C

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def A():
    from paper_2603_08343_b200 import build
    build.build()
    from paper_2603_08343_b200 import attention
    yield attention
    attention.device_status()


@pytest.fixture(scope="module")
def Error():
    from paper_2603_08343_b200.binding import WhtError
    return WhtError


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def ints(*values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def filled(A, pages, hkv, page, d, seed=0):
    """A cache full of keys and values, and what it holds as [pages * page, hkv, d]."""
    g = gen(seed)
    n = pages * page
    k, v = torch.randn(n, hkv, d, generator=g), torch.randn(n, hkv, d, generator=g)
    cache = A.cache4(pages, hkv, page, d)
    A.kv_append4(k.cuda(), v.cuda(), cache, torch.arange(n).cuda())
    return cache, C.hold(k), C.hold(v)


def expected(q, keys, values, table, lens, page, q_start=None):
    rows = [torch.cat([torch.arange(int(p) * page, (int(p) + 1) * page) for p in t])[:n] if n else torch.zeros(0, dtype=torch.int64) for t, n in zip(table, lens)]
    return C.attention(q, [keys[r] for r in rows], [values[r] for r in rows], lens, q_start, q.shape[2] ** -0.5)


def close(got, want, q, spread=8.0, vmax=6.0):
    return (got.cpu().double() - want).abs().max().item() <= C.tolerance(q, spread, vmax, q.shape[2] ** -0.5)


# ---- nothing to do

def test_calls_of_no_tokens(A):
    cache, _, _ = filled(A, 3, 2, 16, 64)
    for dtype in (BF16, F32):
        none = torch.empty(0, 2, 64, dtype=dtype, device="cuda")
        before = cache.clone()
        assert A.kv_append4(none, none, cache, torch.empty(0, dtype=torch.int64, device="cuda"), q=none).shape == none.shape
        assert torch.equal(cache, before)
        k, v = A.kv_read4(cache, torch.empty(0, dtype=torch.int64, device="cuda"), dtype=dtype)
        assert k.shape == (0, 2, 64) and k.dtype == dtype and v.shape == k.shape
        for batch, starts in ((0, None), (0, ints(0)), (3, ints(0, 0, 0, 0))):
            table, lens = torch.zeros(batch, 2, dtype=torch.int32, device="cuda"), torch.full((batch,), 20, dtype=torch.int32, device="cuda")
            w = torch.rand(batch, 2, 32, device="cuda")
            out, received = A.paged_attention4(none, cache, table, lens, q_start=starts, weights=w)
            assert out.shape == none.shape
            want = w.clone()
            want[:, :, 20:] = 0
            assert torch.equal(received, want)           # nobody adds anything; beyond the length there is nothing
    lens, kept, w = A.kv_evict4(cache, torch.zeros(0, 2, dtype=torch.int32, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda"),
                                torch.zeros(0, 2, 32, device="cuda"), torch.zeros(0, 1, dtype=torch.int32, device="cuda"), 5)
    assert lens.shape == (0,) and kept.shape == (0, 2, 5) and w.shape == (0, 2, 16)
    # tables without pages: sequences without keys
    q = torch.randn(2, 4, 64, device="cuda")
    out, received = A.paged_attention4(q, cache, torch.zeros(2, 0, dtype=torch.int32, device="cuda"), ints(0, 0), weights_out=torch.empty(2, 2, 0, device="cuda"))
    assert torch.equal(out, torch.zeros_like(q)) and received.shape == (2, 2, 0)
    lens, kept, w = A.kv_evict4(cache, torch.zeros(1, 0, dtype=torch.int32, device="cuda"), ints(0), torch.zeros(1, 2, 0, device="cuda"), ints(2)[None], 3)
    assert lens.tolist() == [0] and (kept == -1).all() and (w == 0).all()
    A.device_status()


# ---- what is out of range

def test_slots_and_positions_out_of_range(A, Error):
    cache, keys, values = filled(A, 2, 1, 16, 64)
    before = cache.clone()
    x = torch.randn(3, 1, 64, device="cuda")
    A.kv_append4(x, x, cache, torch.tensor([32, 1 << 40, -7]).cuda())
    assert torch.equal(cache, before)
    with pytest.raises(Error):
        A.device_status()
    k, v = A.kv_read4(cache, torch.tensor([32, 5]).cuda())
    assert (k[0] == 0).all() and (v[0] == 0).all() and torch.equal(k[1].cpu(), keys[5])
    with pytest.raises(Error):
        A.device_status()
    cos, sin = R.inverse_frequencies(64, 10)
    A.kv_append4(x, x, cache, torch.tensor([0, 1, -1]).cuda(), positions=ints(10, 3, 99), cos=cos.cuda(), sin=sin.cuda())
    with pytest.raises(Error):
        A.device_status()
    A.kv_append4(x, x, cache, torch.tensor([0, 1, -1]).cuda(), positions=ints(9, 3, 99), cos=cos.cuda(), sin=sin.cuda())   # (a dropped token's is not used)
    A.device_status()


def test_pages_and_lengths_out_of_range(A, Error):
    cache, _, _ = filled(A, 4, 2, 16, 64)
    q = torch.randn(2, 4, 64, device="cuda")
    for table, lens in (([[0, 9], [1, 2]], [20, 20]), ([[0, -1], [1, 2]], [20, 20]), ([[0, 1], [1, 2]], [33, 5]), ([[0, 1], [1, 2]], [20, -1])):
        out, w = A.paged_attention4(q, cache, torch.tensor(table).int().cuda(), ints(*lens), weights_out=torch.empty(2, 2, 32, device="cuda"))
        assert torch.isfinite(out).all() and torch.isfinite(w).all()
        with pytest.raises(Error):
            A.device_status()
    weights = torch.rand(1, 2, 32, device="cuda")
    for table, lens, out_table in (([[0, 9]], [32], [[2]]), ([[0, 1]], [40], [[2]]), ([[0, 1]], [32], [[4]]), ([[0, 1]], [32], [[-1]])):
        lens2, kept, w = A.kv_evict4(cache, torch.tensor(table).int().cuda(), ints(*lens), weights, torch.tensor(out_table).int().cuda(), 7)
        assert lens2.tolist() == [7]
        with pytest.raises(Error):
            A.device_status()
    # entries that no key lies in are not looked at
    A.paged_attention4(q, cache, torch.tensor([[0, 9], [1, -4]]).int().cuda(), ints(16, 3))
    A.device_status()


def test_tokens_of_no_sequence_get_zeros(A, Error):
    cache, keys, values = filled(A, 4, 2, 16, 64)
    q = torch.randn(7, 4, 64, generator=gen(1))
    table, lens = torch.tensor([[0, 1], [2, 3]]).int(), [20, 32]
    for dtype in (BF16, F32):
        x = q.to(dtype)
        out = torch.full((7, 4, 64), 7.0, dtype=dtype, device="cuda")
        A.paged_attention4(x.cuda(), cache, table.cuda(), ints(*lens), q_start=ints(1, 3, 5), max_q_len=2, out=out)
        want, _ = expected(x[1:5], keys, values, table, lens, 16, torch.tensor([0, 2, 4]))
        assert close(out[1:5], want, x) and (out[0] == 0).all() and (out[5:] == 0).all()
        with pytest.raises(Error):
            A.device_status()


def test_offsets_that_make_no_sense_stay_in_bounds(A, Error):
    cache, _, _ = filled(A, 4, 2, 16, 64)
    q = torch.randn(6, 16, 64, device="cuda")
    table, lens = torch.tensor([[0, 1], [2, 3], [1, 0]]).int().cuda(), ints(32, 30, 31)
    for starts in ((0, 6, 2, 6), (-4, 2, 4, 6), (0, 2, 4, 99), (6, 4, 2, 0), (0, 0, 0, 1 << 30)):
        A.paged_attention4(q, cache, table, lens, q_start=ints(*starts), max_q_len=3, weights_out=torch.empty(3, 2, 32, device="cuda"))
        with pytest.raises(Error):
            A.device_status()


# ---- sizes

def test_a_cache_past_four_gibibytes(A):
    """Pages at both ends of a cache of 6 GB."""
    page, hkv, d = 128, 8, 128
    pages = 44000
    cache = torch.empty(pages, hkv, page // 16, 16 * d + 128, dtype=torch.uint8, device="cuda")
    assert cache.numel() > 1 << 32
    n, g = 300, gen(2)
    k, v = torch.randn(n, hkv, d, generator=g), torch.randn(n, hkv, d, generator=g)
    table = torch.tensor([[pages - 1, 0, pages - 2]]).int()
    i = torch.arange(n)
    slots = table[0].long()[i // page] * page + i % page
    A.kv_append4(k.cuda(), v.cuda(), cache, slots.cuda())
    got_k, got_v = A.kv_read4(cache, slots.cuda())
    keys, values = C.hold(k), C.hold(v)
    assert torch.equal(got_k.cpu(), keys) and torch.equal(got_v.cpu(), values)
    q = torch.randn(1, 32, d, generator=g).bfloat16()
    out, weights = A.paged_attention4(q.cuda(), cache, table.cuda(), ints(n), weights_out=torch.empty(1, hkv, 3 * page, device="cuda"))
    want, received = C.attention(q, [keys], [values], [n], None, d ** -0.5)
    assert close(out, want, q) and (weights[0, :, :n].cpu().double() - received[0]).abs().max() < 1e-5
    new = torch.tensor([[pages - 3]]).int()
    _, kept, _ = A.kv_evict4(cache, table.cuda(), ints(n), weights, new.cuda(), 100, keep_last=10)
    moved_k, moved_v = A.kv_read4(cache, (torch.arange(100) + (pages - 3) * page).cuda())
    for h in range(hkv):
        stay = kept[0, h].cpu().long()
        assert torch.equal(moved_k[:, h].cpu(), keys[stay, h]) and torch.equal(moved_v[:, h].cpu(), values[stay, h])
    A.device_status()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("group,tokens", [(4, 1), (2, 3), (8, 5)])
def test_scores_that_would_pass_a_gigabyte_are_taken_anew(A, dtype, group, tokens):
    """A very wide table: the received weight from the codes instead of kept scores."""
    page, width, n = 128, 300000, 700
    cache, keys, values = filled(A, 6, 1, page, 64, seed=3)
    table = torch.full((1, width), -1, dtype=torch.int32)
    table[0, :6] = torch.tensor([3, 1, 5, 0, 2, 4])
    q = torch.randn(tokens, group, 64, generator=gen(4)).to(dtype)
    start = torch.tensor([0, tokens])
    out, weights = A.paged_attention4(q.cuda(), cache, table.cuda(), ints(n), q_start=start.int().cuda(), max_q_len=tokens,
                                      weights_out=torch.empty(1, 1, width * page, device="cuda"))
    rows = torch.cat([torch.arange(int(p) * page, (int(p) + 1) * page) for p in table[0, :6]])[:n]
    want, received = C.attention(q, [keys[rows]], [values[rows]], [n], start, 64 ** -0.5)
    assert close(out, want, q)
    factor = 64 ** -0.5 * q.double().abs().sum(-1).max().item() * 8.0 * 2 ** -18 + 2 ** -20
    assert ((weights[0, 0, :n].cpu().double() - received[0][0]).abs() <= received[0][0] * (factor + 2 ** -20) + 1e-30).all()
    assert (weights[0, 0, n:] == 0).all()
    A.device_status()


def test_many_sequences(A):
    """1500 sequences of none to three tokens and none to forty keys, in one call."""
    page, hkv, d, B = 16, 2, 64, 1500
    cache, keys, values = filled(A, 50, hkv, page, d, seed=5)
    g = gen(6)
    table = torch.randint(0, 50, (B, 3), generator=g).int()                     # (sequences may share pages)
    counts = torch.randint(0, 4, (B,), generator=g)
    lens = (counts + torch.randint(0, 38, (B,), generator=g)).tolist()
    start = torch.cat([torch.zeros(1, dtype=torch.int64), counts.cumsum(0)])
    q = torch.randn(int(start[-1]), 6, d, generator=g)
    for dtype in (BF16, F32):
        x = q.to(dtype)
        out = A.paged_attention4(x.cuda(), cache, table.cuda(), torch.tensor(lens).int().cuda(), q_start=start.int().cuda(), max_q_len=3)
        want, _ = expected(x, keys, values, table, lens, page, start)
        assert close(out, want, x)
    A.device_status()


def test_rows_behind_the_last_key_moved_are_left_alone(A):
    page, d = 64, 128
    cache, keys, values = filled(A, 4, 1, page, d, seed=7)
    A.kv_evict4(cache, ints(0, 1)[None], ints(100), torch.rand(1, 1, 128, device="cuda"), ints(2)[None], 37)
    k, v = A.kv_read4(cache, torch.arange(2 * page + 37, 4 * page).cuda())
    assert torch.equal(k.cpu(), keys[2 * page + 37:]) and torch.equal(v.cpu(), values[2 * page + 37:])
    k, _ = A.kv_read4(cache, torch.arange(2 * page).cuda())
    assert torch.equal(k.cpu(), keys[:2 * page])                                # and so are the old pages


# ---- streams and graphs

def test_queries_in_place(A):
    g = gen(8)
    x = torch.randn(5, 3, 96, generator=g).bfloat16()
    cos, sin = R.inverse_frequencies(96, 20)
    pos = torch.arange(5).int()
    cache = A.cache4(1, 3, 16, 96)
    q = x.cuda()
    same = A.kv_append4(x.cuda(), x.cuda(), cache, torch.arange(5).cuda(), positions=pos.cuda(), cos=cos.cuda(), sin=sin.cuda(), q=q, q_out=q)
    assert same is q and torch.equal(q.cpu(), R.rotate32(x, pos, cos, sin, False))


def test_two_streams_at_once(A):
    """Calls of different sizes side by side, each with its own tensors, over and over: results as when alone."""
    jobs = []
    for i, (B, n, hkv, group) in enumerate(((1, 3000, 4, 2), (40, 200, 2, 4))):
        page = 64
        width = -(-n // page)
        cache, _, _ = filled(A, B * width, hkv, page, 128, seed=i)
        table = torch.arange(B * width).int().reshape(B, width).cuda()
        q = torch.randn(B, hkv * group, 128, generator=gen(i)).bfloat16().cuda()
        jobs.append((q, cache, table, torch.full((B,), n, dtype=torch.int32, device="cuda"), torch.rand(B, hkv, width * page, device="cuda")))
    alone = [[t.clone() for t in A.paged_attention4(q, c, t, n, weights=w)] for q, c, t, n, w in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    got = [[], []]
    for _ in range(20):
        for i, (q, c, t, n, w) in enumerate(jobs):
            got[i].append(A.paged_attention4(q, c, t, n, weights=w, stream=streams[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for out, w in got[i]:
            assert torch.equal(out, alone[i][0]) and torch.equal(w, alone[i][1])
    A.device_status()


def test_a_stream_context(A):
    cache, keys, values = filled(A, 4, 2, 16, 64, seed=9)
    q = torch.randn(1, 4, 64, generator=gen(10))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        out = A.paged_attention4(q.cuda(), cache, ints(1, 3)[None], ints(30))
    s.synchronize()
    want, _ = expected(q, keys, values, torch.tensor([[1, 3]]), [30], 16)
    assert close(out, want, q)


def test_a_captured_run_of_calls_follows_its_inputs(A):
    """Append, attend with weights, evict and read in one graph, replayed with other lengths, pages and values."""
    page, hkv, d, B, width, budget = 16, 2, 64, 3, 6, 20
    pages = B * (width + 2)
    cache = A.cache4(pages, hkv, page, d)
    state = dict(x=torch.zeros(B, 3 * hkv, d, device="cuda"), slots=torch.zeros(B, dtype=torch.int64, device="cuda"),
                 table=torch.zeros(B, width, dtype=torch.int32, device="cuda"), lens=torch.zeros(B, dtype=torch.int32, device="cuda"),
                 weights=torch.zeros(B, hkv, width * page, device="cuda"), out_table=torch.zeros(B, 2, dtype=torch.int32, device="cuda"),
                 out_slots=torch.zeros(B * budget, dtype=torch.int64, device="cuda"))

    def calls():
        q, k, v = state["x"].split([hkv, hkv, hkv], 1)
        A.kv_append4(k, v, cache, state["slots"])
        out, w = A.paged_attention4(q, cache, state["table"], state["lens"], weights=state["weights"])
        lens, kept, w2 = A.kv_evict4(cache, state["table"], state["lens"], w, state["out_table"], budget, keep_first=1, keep_last=2)
        return (out, w, lens, kept, w2, *A.kv_read4(cache, state["out_slots"]))

    def feed(seed):
        g = gen(seed)
        perm = torch.randperm(pages, generator=g)
        table, out_table = perm[:B * width].reshape(B, width), perm[B * width:].reshape(B, 2)
        lens = torch.randint(1, width * page, (B,), generator=g)
        last = lens - 1
        slots = table.gather(1, (last // page)[:, None])[:, 0] * page + last % page
        i = torch.arange(budget)
        out_slots = out_table[:, i // page] * page + i % page
        new = dict(x=torch.randn(B, 3 * hkv, d, generator=g), slots=slots, table=table, lens=lens, weights=torch.rand(B, hkv, width * page, generator=g),
                   out_table=out_table, out_slots=torch.where(i < lens[:, None], out_slots, -1).flatten())
        for name, t in new.items():
            state[name].copy_(t)
        n = pages * page
        k = torch.randn(2, n, hkv, d, generator=g).cuda()
        A.kv_append4(k[0], k[1], cache, torch.arange(n).cuda())

    feed(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        results = calls()
    for seed in (1, 2, 3):
        feed(seed)
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in results]
        feed(seed)
        for x, y in zip(replayed, calls()):
            assert torch.equal(x, y)
    A.device_status()


# ---- refusals that need tensors on a GPU

def test_refusals(A):
    cache, _, _ = filled(A, 4, 2, 16, 64)
    q, table, lens = torch.randn(2, 4, 64, device="cuda"), torch.zeros(2, 2, dtype=torch.int32, device="cuda"), ints(5, 5)
    w = torch.zeros(2, 2, 32, device="cuda")
    k, slots = torch.randn(2, 2, 64, device="cuda"), torch.zeros(2, dtype=torch.int64, device="cuda")
    from paper_2603_08343_b200.binding import WhtError
    bad = [
        lambda: A.paged_attention4(q.half(), cache, table, lens),
        lambda: A.paged_attention4(q.double(), cache, table, lens),
        lambda: A.paged_attention4(q, cache.int(), table, lens),
        lambda: A.paged_attention4(q, cache[:, :, :, :-16], table, lens),
        lambda: A.paged_attention4(q, cache.transpose(0, 1), table, lens),
        lambda: A.paged_attention4(q, cache, table.long(), lens),
        lambda: A.paged_attention4(q, cache, table[:1], lens),
        lambda: A.paged_attention4(q, cache, table, lens, max_q_len=2),
        lambda: A.paged_attention4(q, cache, table, lens, q_start=ints(0, 2)),
        lambda: A.paged_attention4(q, cache, table, lens, weights=w[:, :, :16].contiguous()),
        lambda: A.paged_attention4(q, cache, table, lens, weights=w.double()),
        lambda: A.paged_attention4(q, cache, table, lens, weights=w, weights_out=w[:1]),
        lambda: A.paged_attention4(q, cache, table, lens, out=torch.empty(2, 4, 64, device="cuda").bfloat16()),
        lambda: A.paged_attention4(q.transpose(1, 2), cache, table, lens),
        lambda: A.paged_attention4(q[:, :3], cache, table, lens),                # 3 heads for 2 key heads
        lambda: A.paged_attention4(q.clone().requires_grad_(), cache, table, lens),
        lambda: A.paged_attention4(q, cache, table, lens, weights=w.clone().requires_grad_()),
        lambda: A.paged_attention4(q, cache, table, lens, scale="much"),
        lambda: A.kv_append4(k, k.bfloat16(), cache, slots),
        lambda: A.kv_append4(k, k, cache, slots.int()),
        lambda: A.kv_append4(k, k, cache, slots, q_out=q),
        lambda: A.kv_append4(k, k, cache, slots, positions=ints(0, 1)),
        lambda: A.kv_append4(k[:, :1], k, cache, slots),
        lambda: A.kv_append4(k.clone().requires_grad_(), k, cache, slots),
        lambda: A.kv_append4(torch.randn(2, 2, 65, device="cuda")[:, :, 1:], k, cache, slots),      # rows off 16-byte boundaries
        lambda: A.kv_read4(cache, slots.int()),
        lambda: A.kv_read4(cache.cpu(), slots),
        lambda: A.kv_evict4(cache, table, lens, w, table, 40),                    # more than the new pages hold
        lambda: A.kv_evict4(cache, table, lens, w, table.clone(), 10, keep_first=6, keep_last=5),
        lambda: A.kv_evict4(cache, table, lens, w, table.clone(), 0),
        lambda: A.kv_evict4(cache, table, lens, w, table.clone(), 10, keep_first=-1),
        lambda: A.kv_evict4(cache, table, lens, w, table, 10),                    # the pages it reads
        lambda: A.kv_evict4(cache, table, lens, w[:, :1], table.clone(), 10),
    ]
    before = cache.clone()
    for i, call in enumerate(bad):
        with pytest.raises((ValueError, WhtError)):
            call()
            raise AssertionError(f"call {i} was not refused")
    assert torch.equal(cache, before)
    with torch.no_grad():
        A.paged_attention4(q.clone().requires_grad_(), cache, table, lens)
    A.device_status()


def test_queries_of_any_size(A):
    """From the smallest normal numbers to 2^100, and rows of zeros: queries enter the products after a shift by a power of two."""
    cache, keys, values = filled(A, 4, 1, 16, 64, seed=11)
    base = torch.randn(1, 4, 64, generator=gen(12))
    table, n = torch.arange(4).int()[None], 60
    for dtype in (BF16, F32):
        for size in (0.0, 2.0 ** -120, 2.0 ** -60, 2.0 ** -12, 1.0):
            q = (base * size).to(dtype)
            want, _ = expected(q, keys, values, table, [n], 16)
            assert close(A.paged_attention4(q.cuda(), cache, table.cuda(), ints(n)), want, q)
        # large ones with a scale that brings the scores back
        q = (base * 2.0 ** 100).to(dtype)
        want, _ = C.attention(q, [keys[:n]], [values[:n]], [n], None, 2.0 ** -103)
        got = A.paged_attention4(q.cuda(), cache, table.cuda(), ints(n), scale=2.0 ** -103)
        assert (got.cpu().double() - want).abs().max().item() <= C.tolerance(q, 8.0, 6.0, 2.0 ** -103)
    assert not math.isnan(A.paged_attention4(torch.zeros(1, 4, 64, device="cuda"), cache, table.cuda(), ints(n)).sum().item())


@pytest.mark.parametrize("tokens", [1, 700])
def test_calls_one_right_behind_the_other_see_what_came_before(A, tokens):
    """Kernels start while the one before them drains: over and over the same slots are overwritten, attended to (few rows, and a prompt on
    tcgen05), evicted from and read back, with and without waiting for each call; both give the same."""
    n, hkv, group, d, page, budget = 5000, 4, 4, 128, 64, 1000
    width, out_width = -(-n // page), -(-budget // page)
    g = gen(tokens)
    k, v = (torch.randn(3, n, hkv, d, generator=g).bfloat16().cuda() for _ in range(2))
    q = torch.randn(tokens, hkv * group, d, generator=g).bfloat16().cuda()
    slots = torch.arange(n).cuda()
    table = torch.arange(width).int().cuda()[None]
    out_table = torch.arange(width, width + out_width).int().cuda()[None]
    start = None if tokens == 1 else ints(0, tokens)

    def rounds(wait):
        cache = A.cache4(width + out_width, hkv, page, d)
        weights = torch.zeros(1, hkv, width * page, device="cuda")
        lens, seen = ints(n), []
        torch.cuda.synchronize()
        for i in range(12):
            if i > 0:
                A.kv_append4(k[i % 3], v[(i + 1) % 3], cache, slots)
                wait()
                out, _ = A.paged_attention4(q, cache, table, lens, q_start=start, max_q_len=tokens, weights=weights, weights_out=weights)
                wait()
                plain = A.paged_attention4(q, cache, table, lens, q_start=start, max_q_len=tokens)
                wait()
            else:
                A.kv_append4(k[0], v[0], cache, slots)
                out = plain = None
                wait()
            left, kept, moved = A.kv_evict4(cache, table, lens, weights, out_table, budget, 3, 20)
            wait()
            keys, values = A.kv_read4(cache, (out_table.long() * page)[0, :, None].add(torch.arange(page).cuda()).flatten()[:budget], torch.bfloat16)
            wait()
            after = A.paged_attention4(q[:1], cache, out_table, left)
            wait()
            seen += [t for t in (out, plain, left, kept, moved, keys, values, after, weights.clone()) if t is not None]
        torch.cuda.synchronize()
        return seen

    patient = rounds(torch.cuda.synchronize)
    for _ in range(4):
        for a, b in zip(rounds(lambda: None), patient):
            assert torch.equal(a, b)
    A.device_status()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("group,counts,d", [(1, (4, 0, 1, 3), 64), (2, (2, 1, 0, 2), 96), (3, (1, 1, 1, 1), 128), (4, (0, 1, 1, 0), 64), (5, (1, 1, 0, 1), 128)])
def test_up_to_four_rows_and_a_few_more(A, dtype, group, counts, d):
    """Four rows a sequence and key head sit in other columns of the products than five; told of more tokens than there are, the same call takes
    the columns of eight."""
    page, hkv, lens = 32, 2, (700, 40, 1, 333)
    width = 22
    cache, keys, values = filled(A, len(lens) * width, hkv, page, d, seed=group)
    table = torch.randperm(len(lens) * width, generator=gen(9)).int().reshape(len(lens), width)
    start = [0]
    for c in counts:
        start.append(start[-1] + c)
    q = torch.randn(start[-1], hkv * group, d, generator=gen(group + 50)).to(dtype)
    want, received = expected(q, keys, values, table, lens, page, start)
    for most in (max(counts), 8):
        out, weights = A.paged_attention4(q.cuda(), cache, table.cuda(), ints(*lens), q_start=ints(*start), max_q_len=most,
                                          weights_out=torch.empty(len(lens), hkv, width * page, device="cuda"))
        assert close(out, want, q)
        for b, n in enumerate(lens):
            assert ((weights[b, :, :n].cpu().double() - received[b]).abs() <= 1e-4 * received[b] + 1e-30).all()
            assert (weights[b, :, n:] == 0).all()
    A.device_status()
