"""What the wide bounds of test_attention_gpu.py cannot see: that every key counts exactly once, the rounding that each kernel claims,
long tables, scales of any sign, calls that mix prompts with single tokens, and the tcgen05 kernel next to the own pages in a graph."""
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


def _cuda(*ts):
    return [t.cuda() if isinstance(t, torch.Tensor) else t for t in ts]


def _case(seed, hq, hkv, d, page, dtype, prefix, q_lens, kv_lens, width=None, q_scale=0.5):
    """Queries, a cache of normal keys and values, tables that are -1 beyond a sequence's pages.  What no token may see is NaN."""
    g = _gen(seed)
    B = len(kv_lens)
    need = [-(-n // page) for n in kv_lens]
    n_pre = -(-prefix // page)
    pages = n_pre + sum(need) + 1
    perm = torch.randperm(pages, generator=g).to(torch.int32)
    table = torch.full((B, max([1] + need) if width is None else width), -1, dtype=torch.int32)
    at = n_pre
    kc, vc = (torch.full((pages, hkv, page, d), float("nan"), dtype=dtype) for _ in range(2))
    lists = [(perm[:n_pre], prefix)]
    for b, n in enumerate(need):
        table[b, :n] = perm[at:at + n]
        lists.append((perm[at:at + n], kv_lens[b]))
        at += n
    for ids, n in lists:
        for i, pg in enumerate(ids.tolist()):
            m = min(page, n - i * page)
            kc[pg, :, :m] = torch.randn(hkv, m, d, generator=g).to(dtype)
            vc[pg, :, :m] = torch.randn(hkv, m, d, generator=g).to(dtype)
    T = sum(q_lens)
    starts = torch.tensor([0] + q_lens).cumsum(0).to(torch.int32) if any(n != 1 for n in q_lens) else None
    return dict(q=(torch.randn(T, hq, d, generator=g) * q_scale).to(dtype), kc=kc, vc=vc, pre=perm[:n_pre].contiguous(), prefix=prefix, table=table,
                lens=torch.tensor(kv_lens, dtype=torch.int32), starts=starts, max_q=max(q_lens), hkv=hkv, d=d, T=T)


def _run(A, c, scale=None):
    q, kc, vc, pre, table, lens, starts = _cuda(c["q"], c["kc"], c["vc"], c["pre"], c["table"], c["lens"], c["starts"])
    return A.shared_prefix_attention(q, kc, vc, pre, c["prefix"], table, lens, q_start=starts, max_q_len=c["max_q"], scale=scale)


def _rows(c):
    """(token, key head, keys, values) in 64 bits, for every token."""
    for b, (t0, t1) in enumerate(R.spans(c["starts"], c["T"], len(c["lens"]))):
        for h in range(c["hkv"]):
            n = int(c["lens"][b])
            k, v = (torch.cat([R.keys_of(x, c["pre"], h, c["prefix"]), R.keys_of(x, c["table"][b], h, n)]).double() for x in (c["kc"], c["vc"]))
            for t in range(t0, t1):
                seen = c["prefix"] + max(0, n - (t1 - t0) + (t - t0) + 1)
                yield t, h, k[:seen], v[:seen]


def _exact(c, scale):
    """The result, sum p |v| per element, and per row the largest scale * sum |q| |k| and the number of keys."""
    G = c["q"].shape[1] // c["hkv"]
    out = torch.zeros(c["q"].shape, dtype=torch.float64)
    mass, size = torch.zeros_like(out), torch.zeros(*out.shape[:2], 1, dtype=torch.float64)
    count = torch.zeros_like(size)
    for t, h, k, v in _rows(c):
        if not len(k):
            continue
        s = slice(h * G, (h + 1) * G)
        q = c["q"][t, s].double()
        p = torch.softmax(q @ k.T * scale, -1)
        out[t, s], mass[t, s] = p @ v, p @ v.abs()
        size[t, s, 0] = abs(scale) * (q.abs() @ k.abs().T).max(-1).values
        count[t, s] = len(k)
    return out, mass, size, count


def narrow_bound(dtype, d, out, mass, size, count, tcgen05):
    """|result - out| element by element, from the kernels' arithmetic.  mass = sum p |v|, size = scale sum |q| |k|, n = count keys.

    bf16: products of two bf16 numbers are exact in fp32; a matrix instruction adds 16 of them to its accumulator, each truncated to
    2^-23 of the largest, so a score is off by at most (d + 8) 2^-23 size (the scaling and the difference to the reference: 2^-23 size
    each, taken into d + 16), the weight by as much relatively, and 2^-22 from the exponential; numerator and denominator both: twice.  Adding n values:
    n 17/16 2^-23 mass.  bf16 has 8 significant bits, so rounding to it is off by up to 2^-8: the weights as two bf16 terms 2^-17 mass (half
    a unit of the second); as one (tcgen05), with the sum of the same terms, 2^-8 (mass + |out|); the result 2^-8 |out|.
    fp32: an operand in two tf32 terms is off by 2^-22, the dropped product of the small terms by 2^-22; leading products are added
    eight at a time (9 2^-23) and then with rounding (d / 8 2^-24): 24 2^-23 size covers a score; the same for the values, n 2^-26 for their sum."""
    n = count
    if dtype == BF16:
        weight = (d + 16) * 2.0 ** -23 * size + 2.0 ** -22
        b = mass * (2 * weight + n * 1.0625 * 2.0 ** -23 + 2.0 ** -17) + 2.0 ** -8 * out.abs()
        if tcgen05:
            b = b + 2.0 ** -8 * (mass + out.abs())
    else:
        weight = 24 * 2.0 ** -23 * size + 2.0 ** -21
        b = mass * (2 * weight + 16 * 2.0 ** -23 + n * 2.0 ** -26 + 2.0 ** -21) + 2.0 ** -23 * out.abs()
    return b * (1 + 2.0 ** -6) + 1e-30


FORMS = [
    # hq, hkv, d, page, prefix, q_lens, kv_lens
    (4, 2, 64, 16, 0, [1] * 5, [48, 1, 17, 64, 33]),                # own pages, a few rows
    (16, 1, 128, 64, 0, [1] * 3, [60, 700, 5]),                     # two row tiles
    (32, 1, 96, 32, 0, [1] * 2, [50, 40]),                          # four
    (4, 2, 128, 16, 0, [3, 40], [30, 90]),                          # prompts
    (2, 2, 128, 64, 0, [1] * 2, [9000, 4100]),                      # key ranges and a join
    (8, 4, 128, 128, 130, [1] * 3, [100, 5, 64]),                   # one walk over prefix and own pages
    (4, 2, 64, 32, 2000, [1] * 6, [40, 1, 33, 5, 64, 20]),          # prefix ranges, own pages, a join
    (8, 2, 96, 16, 1000, [5, 1], [40, 20]),
    (4, 4, 128, 16, 300, [1] * 70, [1 + 7 * i % 60 for i in range(70)]),  # from here on tcgen05 (bf16): both tiles the same rows
    (2, 1, 96, 32, 777, [1] * 150, [1 + i % 40 for i in range(150)]),     # two tiles, two blocks of rows
    (6, 2, 64, 64, 5003, [30, 1, 17], [40, 9, 17]),
]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("hq,hkv,d,page,prefix,q_lens,kv_lens", FORMS)
def test_every_key_counts_once(A, hq, hkv, d, page, prefix, q_lens, kv_lens, dtype):
    """Queries of zeros weigh all keys alike, weight 1 exactly; each key's value is 1 in one channel and 0 in the others.  A channel's result is the
    number of its keys over the number of all, where a key dropped or taken twice shows as one in some dozens."""
    c = _case(80, hq, hkv, d, page, dtype, prefix, q_lens, kv_lens)
    c["q"].zero_()
    g = _gen(81)
    channel = torch.randint(0, d, c["vc"].shape[:3], generator=g)
    c["vc"] = torch.where(c["vc"].isnan(), c["vc"], torch.nn.functional.one_hot(channel, d).to(dtype))
    want = _exact(c, 1.0)[0]
    # exact sums of ones; one division, one product and the result's rounding
    got = _run(A, c).cpu().double()
    assert torch.all((got - want).abs() <= want * (2.0 ** -8 * (1 + 2.0 ** -6) if dtype == BF16 else 2.0 ** -22))
    A.device_status()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("hq,hkv,d,page,prefix,q_lens,kv_lens", FORMS)
@pytest.mark.parametrize("q_scale", [0.3, 2.0])
def test_rounding_of_each_form(A, hq, hkv, d, page, prefix, q_lens, kv_lens, q_scale, dtype):
    c = _case(82, hq, hkv, d, page, dtype, prefix, q_lens, kv_lens, q_scale=q_scale)
    scale = d ** -0.5
    want = _exact(c, scale)
    tcgen05 = c["T"] * (hq // hkv) > 32 and prefix >= 256
    got = _run(A, c).cpu().double()
    assert torch.isfinite(got).all()
    worst = ((got - want[0]).abs() / narrow_bound(dtype, d, *want, tcgen05)).max().item()
    assert worst <= 1, worst
    A.device_status()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("scale", [-0.11, 0.0, 0.5])
@pytest.mark.parametrize("form", [0, 3, 5, 6, 8, 9])
def test_scales_of_any_sign(A, form, scale, dtype):
    hq, hkv, d, page, prefix, q_lens, kv_lens = FORMS[form]
    c = _case(83, *FORMS[form][:4], dtype, prefix, q_lens, kv_lens, q_scale=1.0)
    want = _exact(c, scale)
    tcgen05 = c["T"] * (hq // hkv) > 32 and prefix >= 256
    got = _run(A, c, scale).cpu().double()
    assert torch.isfinite(got).all()
    assert ((got - want[0]).abs() / narrow_bound(dtype, d, *want, tcgen05)).max().item() <= 1
    A.device_status()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("times", [4, 32])
@pytest.mark.parametrize("form", [0, 3, 5, 6, 8, 9, 10])
def test_tables_wider_than_their_sequences(A, form, times, dtype):
    """A server's table has room for the longest sequence that it allows; the entries beyond a sequence's pages are never looked at."""
    hq, hkv, d, page, prefix, q_lens, kv_lens = FORMS[form]
    width = max(-(-n // page) for n in kv_lens) * times
    c = _case(84, *FORMS[form][:4], dtype, prefix, q_lens, kv_lens, width=width)
    want = _exact(c, d ** -0.5)
    got = _run(A, c).cpu().double()
    assert ((got - want[0]).abs() / narrow_bound(dtype, d, *want, c["T"] * (hq // hkv) > 32 and prefix >= 256)).max().item() <= 1
    A.device_status()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("times", [1, 4, 32, 200])
@pytest.mark.parametrize("q_lens", [[1, 1, 1], [20, 1, 4]])
def test_selections_from_wide_tables(A, q_lens, times, dtype):
    kv_lens = [300, 40, 77]
    c = _case(85, 4, 2, 64, 16, dtype, 0, q_lens, kv_lens, width=19 * times)
    summary = R.page_summary(torch.nan_to_num(c["kc"].float()), torch.full((2,), 30.0))
    want, want_pages = R.select_attention(c["q"], c["kc"], c["vc"], summary, c["table"], c["lens"], 5, c["starts"], 0.125)
    q, kc, vc, sm, table, lens, starts = _cuda(c["q"], c["kc"], c["vc"], summary, c["table"], c["lens"], c["starts"])
    got, pages = A.selected_page_attention(q, kc, vc, sm, table, lens, 5, q_start=starts, max_q_len=c["max_q"])
    assert torch.equal(pages.cpu(), want_pages)
    # (weights add up to 1 and no value passes 6: the bound of the rounding test with mass = 6, size below 20, 80 keys)
    one = torch.ones_like(want)
    assert torch.all((got.cpu().double() - want).abs() <= narrow_bound(dtype, 64, want, 6 * one, 20 * one, 80 * one, False))
    A.device_status()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("prefix", [0, 1500])
def test_a_prompt_among_single_tokens(A, prefix, dtype):
    """One prompt of 150 tokens in a batch of single tokens, in front, in the middle and at the end; with and without a prefix."""
    for at in (0, 7, 20):
        q_lens, kv_lens = [1] * 20, [1 + 9 * i % 70 for i in range(20)]
        q_lens.insert(at, 150)
        kv_lens.insert(at, 190)
        c = _case(86, 4, 2, 64, 16, dtype, prefix, q_lens, kv_lens)
        want = _exact(c, 0.125)
        got = _run(A, c).cpu().double()
        assert ((got - want[0]).abs() / narrow_bound(dtype, 64, *want, prefix > 0)).max().item() <= 1
    A.device_status()


@pytest.mark.parametrize("form", [0, 1, 2, 6, 8, 9])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
def test_a_query_that_is_no_number_stays_in_its_row(A, form, dtype):
    hq, hkv, d, page, prefix, q_lens, kv_lens = FORMS[form]
    c = _case(87, *FORMS[form][:4], dtype, prefix, q_lens, kv_lens)
    clean = _run(A, c).cpu()
    hit = torch.zeros(c["q"].shape[:2], dtype=torch.bool)
    for t, h, value in ((0, 0, float("nan")), (c["T"] - 1, hq - 1, float("inf")), (c["T"] // 2, hq // 2, float("-inf"))):
        c["q"][t, h, d // 2] = value
        hit[t, h] = True
    got = _run(A, c).cpu()
    assert torch.equal(got[~hit], clean[~hit])
    A.device_status()


@pytest.mark.parametrize("form", [6, 8, 9, 10])
def test_a_graph_with_the_prefix_kernel_beside_the_own_pages(A, form):
    """Captured once and replayed on new queries, keys and lengths."""
    hq, hkv, d, page, prefix, q_lens, kv_lens = FORMS[form]
    c = _case(88, *FORMS[form][:4], BF16, prefix, q_lens, kv_lens)
    q, kc, vc, pre, table, lens, starts = _cuda(c["q"], c["kc"], c["vc"], c["pre"], c["table"], c["lens"], c["starts"])

    def call():
        return A.shared_prefix_attention(q, kc, vc, pre, prefix, table, lens, q_start=starts, max_q_len=c["max_q"])

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = [call() for _ in range(3)]
    for seed in (1, 2):
        g = _gen(seed)
        q.copy_(torch.randn(q.shape, generator=g).to(BF16))
        c["q"] = q.cpu()
        c["lens"] = torch.maximum(c["lens"] - seed, torch.tensor([min(n, m) for n, m in zip(q_lens, kv_lens)], dtype=torch.int32))
        lens.copy_(c["lens"])
        graph.replay()
        torch.cuda.synchronize()
        want = _exact(c, d ** -0.5)
        tcgen05 = c["T"] * (hq // hkv) > 32
        for o in captured:
            assert ((o.cpu().double() - want[0]).abs() / narrow_bound(BF16, d, *want, tcgen05)).max().item() <= 1
            assert torch.equal(o, captured[0])
    A.device_status()
