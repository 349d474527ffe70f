"""The serving attention at the edges of its calls: empty ones, tokens of no sequence, other streams, long tables, narrow bounds."""
import pytest
import torch

import attention_ref as R

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def A():
    from paper_2603_08343_b200 import build
    build.build()
    from paper_2603_08343_b200 import attention
    yield attention
    attention.device_status()


def _gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def _randn(shape, dtype, g, scale=1.0):
    return (torch.randn(*shape, generator=g) * scale).to(dtype)


def _cuda(*ts):
    return [t.cuda() if isinstance(t, torch.Tensor) else t for t in ts]


def _ints(*values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


# ---------------------------------------------------------------- calls of no tokens

@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("width,prefix", [(8, 0), (8, 640), (0, 0), (300, 20)])
def test_calls_of_no_tokens(A, dtype, width, prefix):
    kc = _randn((12, 2, 64, 128), dtype, _gen(1)).cuda()
    summary = torch.zeros(12, 2, 2, 128, dtype=torch.int8, device="cuda")
    q = torch.empty(0, 8, 128, dtype=dtype, device="cuda")
    pre = torch.arange(10, dtype=torch.int32, device="cuda")
    for batch, starts in ((0, None), (0, _ints(0)), (4, _ints(0, 0, 0, 0, 0))):
        table = torch.zeros(batch, width, dtype=torch.int32, device="cuda")
        lens = torch.zeros(batch, dtype=torch.int32, device="cuda")
        for max_q in (1,) if starts is None else (1, 40):
            out = A.shared_prefix_attention(q, kc, kc, pre, prefix, table, lens, q_start=starts, max_q_len=max_q)
            assert out.shape == q.shape and out.dtype == dtype
            out, pages = A.selected_page_attention(q, kc, kc, summary, table, lens, 32, q_start=starts, max_q_len=max_q)
            assert out.shape == q.shape and pages.shape == (0, 2, 32)
    A.device_status()


def test_tokens_without_a_sequence_are_refused(A):
    from paper_2603_08343_b200 import binding as B
    kc = _randn((12, 2, 64, 128), BF16, _gen(1)).cuda()
    summary = torch.zeros(12, 2, 2, 128, dtype=torch.int8, device="cuda")
    q = torch.zeros(3, 8, 128, dtype=BF16, device="cuda")
    table, lens = torch.zeros(0, 8, dtype=torch.int32, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda")
    with pytest.raises(B.WhtError) as e:
        A.shared_prefix_attention(q, kc, kc, None, 0, table, lens, q_start=_ints(0), max_q_len=3)
    assert e.value.status == -3
    with pytest.raises(B.WhtError) as e:
        A.selected_page_attention(q, kc, kc, summary, table, lens, 4, q_start=_ints(0), max_q_len=3)
    assert e.value.status == -3


# ---------------------------------------------------------------- tokens that no sequence covers

def _paged(seed, B, hq, hkv, d, page, dtype, prefix, lead, q_lens, tail, kv_lens, width=None):
    """`lead` tokens before the first sequence's and `tail` after the last one's; keys that no token may see are NaN, values infinite."""
    g = _gen(seed)
    width = max([1] + [-(-n // page) for n in kv_lens]) if width is None else width
    n_pre = -(-prefix // page)
    pages = n_pre + sum(-(-n // page) for n in kv_lens) + 1
    perm = torch.randperm(pages, generator=g).to(torch.int32)
    pre, rest = perm[:n_pre].contiguous(), perm[n_pre:].tolist()
    table = torch.full((B, width), -1, dtype=torch.int32)       # beyond a sequence's length: no page at all
    kc, vc = _randn((pages, hkv, page, d), dtype, g), _randn((pages, hkv, page, d), dtype, g)
    seen = torch.zeros(pages, page, dtype=torch.bool)
    for i in range(prefix):
        seen[int(pre[i // page]), i % page] = True
    for b, n in enumerate(kv_lens):
        for j in range(-(-n // page)):
            table[b, j] = rest.pop()
        for i in range(n):
            seen[int(table[b, i // page]), i % page] = True
    dead = ~seen[:, None, :, None].expand_as(kc)
    kc[dead] = float("nan")
    vc[dead] = float("inf")
    T = lead + sum(q_lens) + tail
    starts = torch.tensor([lead] + q_lens).cumsum(0).to(torch.int32)
    return dict(T=T, q=_randn((T, hq, d), dtype, g, 1.5), kc=kc, vc=vc, pre=pre, table=table, lens=torch.tensor(kv_lens, dtype=torch.int32),
                starts=starts, max_q=max(q_lens), vmax=vc[torch.isfinite(vc)].abs().max().item())


def _poison_workspace(nbytes):
    """The next block of this size from the allocator is full of NaN."""
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    if nbytes:
        junk = torch.full((-(-nbytes // 4),), float("nan"), device="cuda")
        torch.cuda.synchronize()
        del junk


UNCOVERED = [
    # B, hq, hkv, d, page, prefix, lead, q_lens, tail, kv_lens
    (2, 4, 2, 64, 16, 0, 2, [1, 1], 3, [20, 5]),                  # own pages alone, nothing to join
    (2, 4, 2, 128, 64, 0, 1, [3, 2], 2, [2000, 900]),             # key ranges, joined
    (2, 4, 2, 64, 16, 40, 0, [2, 1], 1, [9, 30]),                 # one walk over prefix and own pages
    (3, 4, 1, 96, 32, 2000, 3, [1, 4, 2], 0, [50, 4, 70]),        # prefix ranges, own pages, a join
    (4, 16, 2, 128, 64, 1500, 5, [1, 6, 2, 8], 9, [50, 6, 70, 33]),  # the prefix on tcgen05 (bf16)
    (2, 4, 2, 64, 16, 0, 1, [1, 40], 6, [30, 200]),               # prompts
]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("B,hq,hkv,d,page,prefix,lead,q_lens,tail,kv_lens", UNCOVERED)
def test_tokens_of_no_sequence_get_zeros_and_are_reported(A, B, hq, hkv, d, page, prefix, lead, q_lens, tail, kv_lens, dtype):
    from paper_2603_08343_b200 import binding
    c = _paged(30 + B, B, hq, hkv, d, page, dtype, prefix, lead, q_lens, tail, kv_lens)
    q, kc, vc, pre, table, lens, starts = _cuda(c["q"], c["kc"], c["vc"], c["pre"], c["table"], c["lens"], c["starts"])
    code = 0 if dtype == F32 else 1
    out = torch.full_like(q, 7.0)
    _poison_workspace(binding.lib().wht_attn_prefix_workspace_bytes(prefix, table.shape[1], c["T"], B, c["max_q"], hq, hkv, d, page, code))
    A.shared_prefix_attention(q, kc, vc, pre, prefix, table, lens, q_start=starts, max_q_len=c["max_q"], out=out)
    with pytest.raises(binding.WhtError) as e:
        A.device_status()
    assert e.value.status == -11
    want = R.prefix_attention(c["q"], c["kc"], c["vc"], c["pre"], prefix, c["table"], c["lens"], c["starts"], d ** -0.5)
    covered = torch.zeros(c["T"], dtype=torch.bool)
    covered[lead:c["T"] - tail] = True
    assert torch.all(out.cpu()[~covered] == 0)
    assert torch.isfinite(out).all() and (out.cpu().double() - want).abs().max().item() <= R.tolerance(dtype, c["vmax"])


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("select,width", [(3, None), (3, 700), (40, None)])
@pytest.mark.parametrize("q_lens,kv_lens", [([1, 1, 1], [200, 17, 90]), ([30, 1, 7], [200, 17, 90])])
def test_a_selection_s_tokens_of_no_sequence(A, q_lens, kv_lens, select, width, dtype):
    from paper_2603_08343_b200 import binding
    c = _paged(40, 3, 4, 2, 64, 16, dtype, 0, 2, q_lens, 4, kv_lens, width)
    summary = R.page_summary(torch.nan_to_num(c["kc"].float(), nan=0.0), torch.full((2,), 30.0))
    want, want_pages = R.select_attention(c["q"], c["kc"], c["vc"], summary, c["table"], c["lens"], select, c["starts"], 0.125)
    q, kc, vc, sm, table, lens, starts = _cuda(c["q"], c["kc"], c["vc"], summary, c["table"], c["lens"], c["starts"])
    out = torch.full_like(q, 7.0)
    pages = torch.full((c["T"], 2, select), 99, dtype=torch.int32, device="cuda")
    A.selected_page_attention(q, kc, vc, sm, table, lens, select, q_start=starts, max_q_len=c["max_q"], out=out, pages_out=pages)
    with pytest.raises(binding.WhtError) as e:
        A.device_status()
    assert e.value.status == -11
    assert torch.equal(pages.cpu(), want_pages)
    assert torch.all(out.cpu()[:2] == 0) and torch.all(out.cpu()[-4:] == 0)
    assert torch.isfinite(out).all() and (out.cpu().double() - want).abs().max().item() <= R.tolerance(dtype, c["vmax"])


# ---------------------------------------------------------------- one walk over the prefix and the own pages

@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("d,page,prefix,kv_lens", [
    (128, 128, 20, [128, 77, 1]),       # fp32: one stage a warp; slots zeroed for the hole are copied into again at once
    (128, 128, 130, [128, 5, 64]),
    (64, 64, 33, [190, 64, 129]),
    (96, 128, 257, [380, 300, 126]),
])
def test_slots_behind_the_prefix_s_hole_are_used_again(A, d, page, prefix, kv_lens, dtype):
    """The unused end of the prefix's last page lies inside the list; what it holds (NaN and infinities) and the zeros put in its place
    must not reach the chunks that follow in the same shared memory.  Same bits every time."""
    c = _paged(60 + d, 3, 8, 4, d, page, dtype, prefix, 0, [1, 1, 1], 0, kv_lens)
    q, kc, vc, pre, table, lens = _cuda(c["q"], c["kc"], c["vc"], c["pre"], c["table"], c["lens"])
    want = R.prefix_attention(c["q"], c["kc"], c["vc"], c["pre"], prefix, c["table"], c["lens"], None, d ** -0.5)
    outs = [A.shared_prefix_attention(q, kc, vc, pre, prefix, table, lens) for _ in range(20)]
    assert torch.isfinite(outs[0]).all()
    assert (outs[0].cpu().double() - want).abs().max().item() <= R.tolerance(dtype, c["vmax"])
    assert all(torch.equal(o, outs[0]) for o in outs)
    A.device_status()


# ---------------------------------------------------------------- the status of work on other streams

def test_the_status_waits_for_other_streams(A):
    """An error on a side stream (torch's do not wait for the default stream, nor it for them) behind some tenths of a second of work."""
    from paper_2603_08343_b200 import binding
    kc = torch.zeros(4, 1, 16, 64, dtype=BF16, device="cuda")
    k = torch.zeros(1, 1, 64, dtype=BF16, device="cuda")
    past = torch.tensor([4 * 16], device="cuda")                # the first slot behind the cache
    A.kv_append(k, k, kc, kc, torch.tensor([0], device="cuda"))
    A.device_status()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(400_000_000)
        A.kv_append(k, k, kc, kc, past)
    with pytest.raises(binding.WhtError) as e:
        A.device_status()
    assert e.value.status == -11
    A.device_status()


def test_the_older_status_waits_for_other_streams():
    """An expired wait (the library's self-test, 100 ms) on a side stream."""
    from paper_2603_08343_b200 import binding
    torch.cuda.synchronize()
    binding.wht_affine_device_status()
    out = torch.zeros(3, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    binding.wht_affine_selftest_wait_expiry(100_000, out, stream=side)
    with pytest.raises(binding.WhtError) as e:
        binding.wht_affine_device_status()
    assert e.value.status == -9
    binding.wht_affine_device_status()


# ---------------------------------------------------------------- the example at the end of its pages

@pytest.mark.parametrize("select", [0, 2])
def test_a_step_past_the_example_s_pages_is_reported(select):
    """The own pages are looked up in range (an index past them would be a device assertion), the token is dropped, the length reported."""
    import importlib.util
    import os
    from paper_2603_08343_b200 import binding
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serving_step.py")
    spec = importlib.util.spec_from_file_location("serving_step", path)
    E = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(E)
    block = E.Block(2, 4, 2, 64, 16, 16, 20)          # room for 32
    rows = 4 + 2 * 2
    block.write_prefix(torch.zeros(16, rows, 64, dtype=BF16, device="cuda"))
    block.own_lens.fill_(31)
    block.step(torch.ones(2, rows, 64, dtype=BF16, device="cuda"), select)
    E.A.device_status()
    before = block.k_cache.clone()
    block.step(torch.ones(2, rows, 64, dtype=BF16, device="cuda"), select)
    with pytest.raises(binding.WhtError) as e:
        E.A.device_status()
    assert e.value.status == -11
    assert torch.equal(block.k_cache, before)
    for bad in (15, 17):
        with pytest.raises(ValueError):
            block.write_prefix(torch.zeros(bad, rows, 64, dtype=BF16, device="cuda"))
    with pytest.raises(ValueError):
        block.step(torch.ones(3, rows, 64, dtype=BF16, device="cuda"), select)
    with pytest.raises(ValueError):
        E.Block(2, 4, 2, 64, 16, 16, 0)


# ---------------------------------------------------------------- append: what is not used is not checked

@pytest.mark.parametrize("with_summary", [False, True])
def test_positions_of_dropped_tokens_are_not_looked_at(A, with_summary):
    """Padding tokens without a query use no position: one outside the table is no error."""
    g = _gen(50)
    T, page = 70, 16
    kc, vc = (torch.zeros(9, 2, page, 64, dtype=BF16, device="cuda") for _ in range(2))
    k, v = _randn((T, 2, 64), BF16, g), _randn((T, 2, 64), BF16, g)
    slots = torch.arange(T) + 5
    positions = torch.arange(T, dtype=torch.int32)
    slots[[0, 33]], positions[[0, 33]] = -1, torch.tensor([-1, 10 ** 6], dtype=torch.int32)
    slots[40:], positions[40:] = -1, 10 ** 9
    cos, sin = R.inverse_frequencies(64, 50)
    summary = torch.zeros(9, 2, 2, 64, dtype=torch.int8, device="cuda") if with_summary else None
    if with_summary:   # (a dropped token inside a page's tokens would part them)
        slots[33], positions[33] = 38, 33
    kd, vd, sd, pd, cd, nd = _cuda(k, v, slots, positions, cos, sin)
    A.kv_append(kd, vd, kc, vc, sd, positions=pd, cos=cd, sin=nd, summary=summary, summary_scale=torch.full((2,), 30.0, device="cuda"))
    A.device_status()
    live = slots >= 0
    want_k, want_v = torch.zeros(9 * page, 2, 64, dtype=BF16), torch.zeros(9 * page, 2, 64, dtype=BF16)
    want_k[slots[live]] = R.rotate32(k[live], positions[live], cos, sin, False)
    want_v[slots[live]] = v[live]
    assert torch.equal(kc.cpu().transpose(1, 2).reshape(9 * page, 2, 64), want_k)
    assert torch.equal(vc.cpu().transpose(1, 2).reshape(9 * page, 2, 64), want_v)


# ---------------------------------------------------------------- refusals of the Python calls

def test_tensors_that_want_a_gradient_are_refused(A):
    """These operators have no backward: a graph that would end in them without a word is refused, and not under no_grad."""
    kc, summary = torch.zeros(4, 1, 16, 64, dtype=BF16, device="cuda"), torch.zeros(4, 1, 2, 64, dtype=torch.int8, device="cuda")
    k, slots = torch.zeros(1, 1, 64, dtype=BF16, device="cuda"), torch.tensor([0], device="cuda")
    wants = torch.zeros(1, 1, 64, dtype=BF16, device="cuda", requires_grad=True)
    table, lens = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), _ints(1)
    calls = [lambda x: A.kv_append(x, k, kc, kc, slots), lambda x: A.kv_append(k, x, kc, kc, slots),
             lambda x: A.kv_append(k, k, kc, kc, slots, q=x), lambda x: A.shared_prefix_attention(x, kc, kc, None, 0, table, lens),
             lambda x: A.selected_page_attention(x, kc, kc, summary, table, lens, 1)]
    for call in calls:
        with pytest.raises(ValueError, match="no_grad"):
            call(wants)
        with torch.no_grad():
            call(wants)
        call(wants.detach())
    A.device_status()


def test_arguments_of_no_use_are_refused(A):
    """A truth value that is none, and a stream of another device (a stand-in: nothing is launched on it)."""
    kc = torch.zeros(4, 1, 16, 64, dtype=BF16, device="cuda")
    k, slots = torch.zeros(1, 1, 64, dtype=BF16, device="cuda"), torch.tensor([0], device="cuda")
    with pytest.raises(RuntimeError):
        A.kv_append(k, k, kc, kc, slots, interleaved=torch.tensor([True, False]))

    class Elsewhere:
        device_index, cuda_stream = torch.cuda.current_device() + 1, 0
    with pytest.raises(ValueError, match="device"):
        A.kv_append(k, k, kc, kc, slots, stream=Elsewhere())
    side = torch.cuda.Stream()
    A.kv_append(k, k, kc, kc, slots, stream=side)
    A.kv_append(k, k, kc, kc, slots, stream=torch.cuda.default_stream())
    A.device_status()


# ---------------------------------------------------------------- scores of any size

@pytest.mark.parametrize("size", [30.0, 300.0, 5e3, 2e4, 1e6])
@pytest.mark.parametrize("B,d,page,grow", [(9, 128, 16, True), (70, 128, 64, False), (70, 96, 32, True), (300, 64, 16, True)])
def test_scores_of_any_size(A, size, B, d, page, grow):
    """Queries and keys of up to 10^6, scores of up to 10^13: one key takes all the weight (the two best scores of a row lie much
    further apart than fp32 rounds them), so the result is its value, within one rounding."""
    prefix = 700
    g = _gen(70 + B)
    c = _paged(70 + B, B, 2, 1, d, page, BF16, prefix, 0, [1] * B, 0, [1 + i % 3 for i in range(B)])
    scale_of_page = torch.ones(c["kc"].shape[0], 1, 1, 1)
    if grow:   # the best key of a row comes late: its reference moves again and again
        scale_of_page[c["pre"].long()] = (0.1 + torch.arange(len(c["pre"])) / len(c["pre"])).reshape(-1, 1, 1, 1)
    kc = (torch.randn(c["kc"].shape, generator=g) * size * scale_of_page).to(BF16)
    kc[c["kc"].isnan()] = float("nan")
    qs = (torch.randn(c["q"].shape, generator=g) * size).to(BF16)
    want = torch.zeros(c["q"].shape, dtype=torch.float64)
    clear = torch.zeros(B, 2, dtype=torch.bool)
    for b in range(B):
        n = int(c["lens"][b])
        k = torch.cat([R.keys_of(kc, c["pre"], 0, prefix), R.keys_of(kc, c["table"][b], 0, n)]).double()
        v = torch.cat([R.keys_of(c["vc"], c["pre"], 0, prefix), R.keys_of(c["vc"], c["table"][b], 0, n)]).double()
        s = qs[b].double() @ k.T * d ** -0.5
        top = s.topk(2).values
        # fp32: a sum of d products (2^-22 of their magnitudes at most) and a few roundings of the score; 40 = more than any weight that counts
        slack = 2.0 ** -20 * (qs[b].double().abs() @ k.abs().T * d ** -0.5).max(-1).values
        clear[b] = top[:, 0] - top[:, 1] > 40 + 2 * slack
        want[b] = v[s.argmax(-1)]
    if size >= 300:
        assert clear.float().mean() > 0.9
    qd, kd, vd, pre, table, lens = _cuda(qs, kc, c["vc"], c["pre"], c["table"], c["lens"])
    got = A.shared_prefix_attention(qd, kd, vd, pre, prefix, table, lens).cpu()
    assert torch.isfinite(got).all()
    assert torch.equal(got[clear].double(), want[clear])
    A.device_status()


# ---------------------------------------------------------------- calls on another stream

def test_inputs_freed_after_a_call_on_another_stream(A):
    """The call waits on a side stream behind some tenths of a second; its inputs are dropped at once and their memory asked for again."""
    c = _paged(90, 4, 4, 2, 64, 16, BF16, 300, 0, [1] * 4, 0, [40, 3, 17, 60])
    args = _cuda(c["q"], c["kc"], c["vc"], c["pre"], c["table"], c["lens"])
    want = A.shared_prefix_attention(args[0], args[1], args[2], args[3], 300, args[4], args[5])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(400_000_000)
    got = A.shared_prefix_attention(args[0], args[1], args[2], args[3], 300, args[4], args[5], stream=side)
    shapes = [(a.shape, a.dtype) for a in args]
    del args
    junk = [torch.zeros(s, dtype=t, device="cuda") for s, t in shapes for _ in range(4)]
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    del junk
    # and an append: rows and slots
    kc, vc = (torch.zeros(4, 2, 16, 64, dtype=BF16, device="cuda") for _ in range(2))
    k, slots = _cuda(_randn((50, 2, 64), BF16, _gen(91)), torch.arange(50))
    with torch.cuda.stream(side):
        torch.cuda._sleep(400_000_000)
    A.kv_append(k, k, kc, vc, slots, stream=side)
    keep = k.cpu()
    del k, slots
    junk = [torch.zeros(50, 2, 64, dtype=BF16, device="cuda") for _ in range(4)] + [torch.zeros(50, dtype=torch.int64, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    assert torch.equal(kc.cpu().transpose(1, 2).reshape(64, 2, 64)[:50], keep)
    del junk
    A.device_status()


def test_strides_of_dimensions_of_one(A):
    """[tokens, 1, head_dim] out of [tokens, head_dim, 1], and one token out of a tensor with odd strides."""
    c = _paged(95, 3, 1, 1, 64, 16, BF16, 40, 0, [1] * 3, 0, [4, 30, 17])
    q, kc, vc, pre, table, lens = _cuda(c["q"], c["kc"], c["vc"], c["pre"], c["table"], c["lens"])
    odd = q.reshape(3, 64, 1).transpose(1, 2)
    assert odd.stride(1) == 1
    want = A.shared_prefix_attention(q, kc, vc, pre, 40, table, lens)
    assert torch.equal(A.shared_prefix_attention(odd, kc, vc, pre, 40, table, lens), want)
    one = torch.as_strided(q, (1, 1, 64), (3, 5, 1))
    assert torch.equal(A.shared_prefix_attention(one, kc, vc, pre, 40, table[:1], lens[:1]), want[:1])
    cache = torch.zeros_like(kc)
    A.kv_append(one, one, cache, cache, torch.tensor([17], device="cuda"), q=odd[:1])
    assert torch.equal(cache[1, 0, 1], q[0, 0])
    A.device_status()
