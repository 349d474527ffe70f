"""The serving attention (paged append, shared prefix, selected pages) against plain 64-bit statements on the CPU."""
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


# ---------------------------------------------------------------- append

def _append_case(seed, T, hq, hkv, d, rot, page, dtype, runs, pad, packed):
    """Tokens of several sequences: runs = [(start place, length)], each on pages of its own."""
    g = _gen(seed)
    assert sum(n for _, n in runs) + pad == T
    pages = sum((s + n - 1) // page - s // page + 1 for s, n in runs) + 2
    perm = torch.randperm(pages, generator=g)
    slots, positions, at = [], [], 0
    for start, n in runs:
        for i in range(n):
            slots.append(int(perm[at + (start + i) // page - start // page]) * page + (start + i) % page)
            positions.append(start + i)
        at += (start + n - 1) // page - start // page + 1
    slots += [-1] * pad
    positions += [0] * pad
    if packed:
        qkv = _randn((T, hq + 2 * hkv, d), dtype, g).cuda()
        q, k, v = qkv.split([hq, hkv, hkv], dim=1)
    else:
        q, k, v = (_randn((T, h, d), dtype, g).cuda() for h in (hq, hkv, hkv))
    kc, vc = _randn((pages, hkv, page, d), dtype, g), _randn((pages, hkv, page, d), dtype, g)
    cos, sin = R.inverse_frequencies(rot, 700) if rot else (None, None)
    lo = torch.randint(-60, 1, (pages, hkv, d), generator=g)
    hi = torch.randint(0, 61, (pages, hkv, d), generator=g)
    return dict(q=q, k=k, v=v, kc=kc, vc=vc, slots=torch.tensor(slots), positions=torch.tensor(positions, dtype=torch.int32), cos=cos, sin=sin,
                summary=torch.stack([lo, hi], 2).to(torch.int8), scale=torch.rand(hkv, generator=g) * 10 + 20)


APPEND = [
    # T, hq, hkv, d, rot, page, dtype, runs, padding, packed, interleaved
    (1, 4, 2, 128, 128, 64, BF16, [(77, 1)], 0, True, False),
    (1, 1, 1, 64, 0, 16, F32, [(0, 1)], 0, False, False),
    (9, 6, 3, 96, 64, 16, BF16, [(15, 1), (16, 1), (5, 1), (0, 1), (31, 1), (300, 1)], 3, True, True),
    (150, 4, 4, 64, 32, 16, BF16, [(0, 40), (7, 100)], 10, False, False),
    (301, 8, 2, 128, 64, 128, BF16, [(100, 200), (3, 101)], 0, True, False),
    (133, 3, 1, 96, 96, 32, F32, [(0, 64), (1, 1), (31, 2), (60, 66)], 0, True, True),
    (700, 5, 5, 64, 64, 64, BF16, [(0, 350), (1, 349)], 1, False, False),
]


@pytest.mark.parametrize("T,hq,hkv,d,rot,page,dtype,runs,pad,packed,interleaved", APPEND)
@pytest.mark.parametrize("with_summary", [False, True])
def test_append(A, T, hq, hkv, d, rot, page, dtype, runs, pad, packed, interleaved, with_summary):
    c = _append_case(5 + T, T, hq, hkv, d, rot, page, dtype, runs, pad, packed)
    kc, vc, summary, scale, slots = _cuda(c["kc"], c["vc"], c["summary"], c["scale"], c["slots"])
    cos, sin, pos = (_cuda(c["cos"], c["sin"], c["positions"]) if rot else (None, None, None))
    out = A.kv_append(c["k"], c["v"], kc, vc, slots, positions=pos, cos=cos, sin=sin, q=c["q"], interleaved=interleaved,
                      summary=summary if with_summary else None, summary_scale=scale if with_summary else None)
    torch.cuda.synchronize()
    q, k, v = (c[n].cpu() for n in "qkv")
    want_q, want_k = (R.rotate32(x, c["positions"], c["cos"], c["sin"], interleaved) if rot else x for x in (q, k))
    assert torch.equal(out.cpu(), want_q)
    if rot:  # and the rotation is the formula's: one rounding of each product and sum, one to the type
        exact = R.rotate(q, c["positions"], c["cos"], c["sin"], interleaved)
        eps = 2 ** -8 if dtype == BF16 else 0.0
        assert torch.all((out.cpu().double() - exact).abs() <= exact.abs() * eps + 2 ** -22 * q.double().abs().amax() * 2)
    want_kc, want_vc = c["kc"].clone(), c["vc"].clone()
    want_s = c["summary"].clone()
    for t in range(T):
        s = int(c["slots"][t])
        if s < 0:
            continue
        want_kc[s // page, :, s % page] = want_k[t]
        want_vc[s // page, :, s % page] = v[t]
        k8 = (want_k[t].float() * c["scale"][:, None]).round().clamp(-127, 127).to(torch.int8)
        if s % page == 0:
            want_s[s // page, :, 0] = k8
            want_s[s // page, :, 1] = k8
        else:
            want_s[s // page, :, 0] = torch.minimum(want_s[s // page, :, 0], k8)
            want_s[s // page, :, 1] = torch.maximum(want_s[s // page, :, 1], k8)
    assert torch.equal(kc.cpu(), want_kc) and torch.equal(vc.cpu(), want_vc)
    assert torch.equal(summary.cpu(), want_s if with_summary else c["summary"])
    A.device_status()


def test_append_in_place_and_empty(A):
    c = _append_case(3, 20, 2, 1, 64, 64, 16, BF16, [(5, 20)], 0, False)
    kc, vc, slots, cos, sin, pos = _cuda(c["kc"], c["vc"], c["slots"], c["cos"], c["sin"], c["positions"])
    want = A.kv_append(c["k"], c["v"], kc, vc, slots, positions=pos, cos=cos, sin=sin, q=c["q"])
    q = c["q"].clone()
    assert A.kv_append(c["k"], c["v"], kc, vc, slots, positions=pos, cos=cos, sin=sin, q=q, q_out=q) is q
    assert torch.equal(q, want)
    before = kc.clone()
    assert A.kv_append(c["k"][:0], c["v"][:0], kc, vc, slots[:0]) is None
    assert torch.equal(kc, before)


def test_append_reports_what_is_out_of_range(A):
    from paper_2603_08343_b200 import binding as B
    c = _append_case(4, 4, 1, 1, 64, 64, 16, BF16, [(5, 4)], 0, False)
    kc, vc, cos, sin = _cuda(c["kc"], c["vc"], c["cos"], c["sin"])
    slots = c["slots"].clone()
    slots[2] = kc.shape[0] * 16  # the first slot past the cache
    A.kv_append(c["k"], c["v"], kc, vc, slots.cuda(), positions=c["positions"].cuda(), cos=cos, sin=sin)
    with pytest.raises(B.WhtError) as e:
        A.device_status()
    assert e.value.status == -11
    A.device_status()
    live = [t for t in range(4) if t != 2]
    for t in live:
        s = int(slots[t])
        assert torch.equal(vc[s // 16, :, s % 16].cpu(), c["v"][t].cpu())
    pos = c["positions"].clone()
    pos[1] = cos.shape[0]
    A.kv_append(c["k"], c["v"], kc, vc, c["slots"].cuda(), positions=pos.cuda(), cos=cos, sin=sin)
    with pytest.raises(B.WhtError):
        A.device_status()


# ---------------------------------------------------------------- shared prefix

def _paged(seed, B, hq, hkv, d, page, dtype, prefix, q_lens, kv_lens, width=None, poison=True, q_scale=1.5):
    """A cache in which everything that no token may see is NaN or infinite."""
    g = _gen(seed)
    tokens = sum(q_lens)
    width = max([1] + [-(-n // page) for n in kv_lens]) if width is None else width
    n_pre = -(-prefix // page)
    pages = n_pre + B * width + 1
    perm = torch.randperm(pages, generator=g).to(torch.int32)
    pre, table = perm[:n_pre].contiguous(), perm[n_pre:n_pre + B * width].reshape(B, width).contiguous()
    kc, vc = _randn((pages, hkv, page, d), dtype, g), _randn((pages, hkv, page, d), dtype, g)
    if poison:
        seen = torch.zeros(pages, page, dtype=torch.bool)
        for row, n in [(pre, prefix)] + [(table[b], kv_lens[b]) for b in range(B)]:
            for i in range(n):
                seen[int(row[i // page]), i % page] = True
        dead = ~seen[:, None, :, None].expand_as(kc)
        kc[dead] = float("nan")
        vc[dead] = float("inf")
    starts = None
    if any(n != 1 for n in q_lens):
        starts = torch.tensor([0] + q_lens).cumsum(0).to(torch.int32)
    return dict(q=_randn((tokens, hq, d), dtype, g, q_scale), kc=kc, vc=vc, pre=pre, table=table, lens=torch.tensor(kv_lens, dtype=torch.int32), starts=starts,
                max_q=max(q_lens))


def _check(got, want, dtype, vmax, what=""):
    got = got.double().cpu()
    assert torch.isfinite(got).all(), what
    err = (got - want).abs().max().item()
    assert err <= R.tolerance(dtype, vmax), f"{what}: {err} > {R.tolerance(dtype, vmax)}"


def _run_prefix(A, c, prefix, scale, q=None, **kw):
    q, kc, vc, pre, table, lens, starts = _cuda(c["q"] if q is None else q, c["kc"], c["vc"], c["pre"], c["table"], c["lens"], c["starts"])
    return A.shared_prefix_attention(q, kc, vc, pre, prefix, table, lens, q_start=starts, max_q_len=c["max_q"], scale=scale, **kw)


PREFIX = [
    # B, hq, hkv, d, page, prefix, q_lens, kv_lens
    (1, 1, 1, 64, 16, 0, [1], [1]),
    (1, 4, 4, 128, 64, 1, [1], [1]),
    (3, 4, 2, 64, 16, 0, [1, 1, 1], [0, 1, 37]),                    # a row with nothing to see
    (3, 4, 2, 128, 32, 65, [1, 1, 1], [0, 33, 64]),
    (2, 8, 1, 96, 16, 100, [1, 1], [15, 17]),
    (5, 6, 3, 64, 128, 300, [1] * 5, [1, 127, 128, 129, 200]),
    (2, 2, 2, 128, 64, 1000, [1, 1], [700, 3]),                      # both split over blocks
    (3, 2, 1, 64, 16, 33, [5, 1, 9], [5, 40, 12]),                   # several tokens, each sees up to itself
    (3, 4, 4, 96, 32, 0, [3, 2, 20], [1, 2, 20]),                    # tokens before the first key: empty rows
    (2, 16, 2, 128, 64, 257, [17, 40], [20, 100]),                   # more rows than a block holds
    (4, 48, 1, 64, 32, 200, [1] * 4, [10, 20, 30, 40]),              # 48 query heads for one key head
    (40, 4, 2, 128, 16, 513, [1] * 40, [(7 * i) % 90 for i in range(40)]),
    (70, 2, 2, 64, 64, 190, [1] * 70, [(5 * i) % 40 + 1 for i in range(70)]),
    (33, 4, 1, 128, 128, 640, [1] * 33, [(11 * i) % 60 + 1 for i in range(33)]),
    (6, 8, 4, 128, 32, 385, [30, 1, 25, 7, 64, 2], [30, 1, 60, 20, 64, 5]),
    # rows enough for the tcgen05 kernel: one tile of rows twice, two tiles, more than one block of rows; whole and ragged key tiles
    (66, 2, 2, 64, 16, 256, [1] * 66, [(3 * i) % 20 for i in range(66)]),
    (70, 1, 1, 64, 64, 1111, [1] * 70, [1] * 70),
    (65, 2, 1, 64, 128, 1280, [1] * 65, [2] * 65),
    (100, 3, 1, 96, 32, 700, [1] * 100, [5] * 100),
    (65, 1, 1, 96, 128, 300, [1] * 65, [9] * 65),
    (300, 2, 2, 128, 16, 401, [1] * 300, [3] * 300),
    (128, 1, 1, 128, 64, 5000, [1] * 128, [3] * 128),
    (129, 2, 2, 128, 128, 4096, [1] * 129, [2] * 129),
    (2, 16, 1, 64, 32, 600, [40, 3], [41, 3]),
    # key ranges of one tile: all copies of a block are asked for before its queries are loaded
    (140, 1, 1, 128, 64, 300, [1] * 140, [2] * 140),
    (300, 2, 2, 64, 128, 640, [1] * 300, [1] * 300),
]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("B,hq,hkv,d,page,prefix,q_lens,kv_lens", PREFIX)
def test_shared_prefix(A, B, hq, hkv, d, page, prefix, q_lens, kv_lens, dtype):
    c = _paged(100 + B, B, hq, hkv, d, page, dtype, prefix, q_lens, kv_lens)
    want = R.prefix_attention(c["q"], c["kc"], c["vc"], c["pre"], prefix, c["table"], c["lens"], c["starts"], d ** -0.5)
    vmax = c["vc"][torch.isfinite(c["vc"])].abs().max().item()
    _check(_run_prefix(A, c, prefix, None), want, dtype, vmax)
    A.device_status()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("B", [9, 70])
def test_shared_prefix_large_scores(A, dtype, B):
    # scores of both signs in the hundreds: one key takes all the weight, or all weights would underflow without the maximum
    c = _paged(7, B, 4, 2, 128, 16, dtype, 300, [1] * B, [20] * B, q_scale=40.0)
    # keys that grow along the prefix: the running maximum moves again and again
    for i, pg in enumerate(c["pre"].tolist()):
        c["kc"][pg] *= 0.2 + 0.05 * i
    want = R.prefix_attention(c["q"], c["kc"], c["vc"], c["pre"], 300, c["table"], c["lens"], None, 0.5)
    got = _run_prefix(A, c, 300, 0.5).double().cpu()
    assert torch.isfinite(got).all()
    # the scores' own fp32 rounding (|score| up to ~2^10, 2^-23 relative of a sum of 128 terms) moves weights by up to 2^-10
    assert (got - want).abs().max().item() <= R.tolerance(BF16, 5.0)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("d,prefix,lens", [(64, 0, [20, 37]), (128, 21, [18, 300]), (96, 700, [40, 18])])
def test_later_tokens_values_stay_out_of_earlier_ones(A, dtype, d, prefix, lens):
    """Values that are infinite or NaN at a token's place do not reach the tokens of the same call that do not see it."""
    q_lens = [18, 18]
    c = _paged(12, 2, 6, 2, d, 16, dtype, prefix, q_lens, lens)
    clean = _run_prefix(A, c, prefix, None).cpu()
    bad = [int(n) - 7 for n in lens]                    # seen by the last seven tokens of each sequence only
    for b, (j, value) in enumerate(zip(bad, (float("inf"), float("nan")))):
        c["vc"][int(c["table"][b, j // 16]), :, j % 16] = value
    got = _run_prefix(A, c, prefix, None).cpu()
    for b in range(2):
        first, last = 18 * b, 18 * (b + 1) - 7
        assert not torch.isfinite(got[last:18 * (b + 1)].float()).any()
        assert (got[first:last].double() - clean[first:last].double()).abs().max() <= 2 * R.tolerance(dtype, 6.0)
    A.device_status()


def test_shared_prefix_strides_out_and_stream(A):
    c = _paged(8, 6, 4, 2, 64, 16, BF16, 100, [1] * 6, [9, 1, 30, 4, 5, 6])
    wide = torch.zeros(6, 9, 64, dtype=BF16).cuda()
    wide[:, 2:6] = c["q"].cuda()
    base = _run_prefix(A, c, 100, None)
    assert torch.equal(_run_prefix(A, c, 100, None, q=wide[:, 2:6]), base)
    every_second = torch.zeros(6, 8, 64, dtype=BF16).cuda()
    every_second[:, ::2] = c["q"].cuda()
    assert torch.equal(_run_prefix(A, c, 100, None, q=every_second[:, ::2]), base)
    out = torch.empty_like(base)
    assert _run_prefix(A, c, 100, None, out=out) is out and torch.equal(out, base)
    s = torch.cuda.Stream()
    other = _run_prefix(A, c, 100, None, stream=s)
    s.synchronize()
    assert torch.equal(other, base)
    # the same call again gives the same bits
    assert torch.equal(_run_prefix(A, c, 100, None), base)


def test_shared_prefix_equals_its_parts_in_one(A):
    """The prefix copied in front of each sequence's own pages gives the same as the shared one."""
    B, page, d = 5, 16, 128
    c = _paged(9, B, 8, 2, d, page, BF16, 64, [1] * B, [40, 3, 64, 17, 1], poison=False)
    shared = _run_prefix(A, c, 64, None)
    joined = torch.cat([c["pre"][None].expand(B, -1), c["table"]], 1).contiguous()
    q, kc, vc, table, lens = _cuda(c["q"], c["kc"], c["vc"], joined, c["lens"] + 64)
    alone = A.shared_prefix_attention(q, kc, vc, None, 0, table, lens)
    _check(shared, alone.double().cpu(), BF16, c["vc"].abs().max().item())


@pytest.mark.parametrize("B,h,d,page", [(70, 16, 64, 64), (128, 16, 128, 128), (200, 8, 96, 32), (256, 8, 128, 16)])
def test_long_prefix_by_both_kernels(A, B, h, d, page):
    """Many key tiles per block of the tensor-core kernel, against the paged kernel on the prefix as everyone's own pages."""
    prefix = 20011
    g = torch.Generator(device="cuda")
    g.manual_seed(B)
    n_pre = -(-prefix // page)
    kc = torch.empty(n_pre, h, page, d, device="cuda", dtype=BF16).normal_(generator=g)
    vc = torch.empty_like(kc).normal_(generator=g)
    q = torch.empty(B, h, d, device="cuda", dtype=BF16).normal_(generator=g) * 3
    pre = torch.randperm(n_pre, device="cuda", generator=g).to(torch.int32)
    none = torch.zeros(B, dtype=torch.int32, device="cuda")
    for _ in range(3):
        shared = A.shared_prefix_attention(q, kc, vc, pre, prefix, pre[:1].expand(B, 1).contiguous(), none)
        own = A.shared_prefix_attention(q, kc, vc, None, 0, pre[None].expand(B, -1).contiguous(), none + prefix)
        # each is within the bound of the exact result
        assert torch.isfinite(shared).all()
        assert (shared.float() - own.float()).abs().max().item() <= 2 * R.tolerance(BF16, vc.abs().max().item())
    A.device_status()


def test_shared_prefix_reports_bad_pages_and_lengths(A):
    from paper_2603_08343_b200 import binding as B
    c = _paged(10, 2, 2, 1, 64, 16, BF16, 40, [1, 1], [20, 30], poison=False)
    for which, at, value in (("pre", 1, 10 ** 6), ("table", (1, 0), -3), ("lens", 0, 10 ** 6)):
        broken = dict(c)
        broken[which] = c[which].clone()
        broken[which][at] = value
        _run_prefix(A, broken, 40, None)
        with pytest.raises(B.WhtError) as e:
            A.device_status()
        assert e.value.status == -11
    _run_prefix(A, c, 40, None)
    A.device_status()


# ---------------------------------------------------------------- selected pages

SELECT = [
    # B, hq, hkv, d, page, select, q_lens, kv_lens
    (1, 1, 1, 64, 16, 1, [1], [1]),
    (2, 4, 2, 128, 16, 1, [1, 1], [40, 0]),                           # only its own page; a row with nothing to see
    (3, 4, 1, 96, 16, 4, [1] * 3, [64, 65, 300]),
    (2, 8, 8, 64, 32, 3, [1, 1], [31, 500]),
    (4, 8, 2, 128, 64, 5, [1] * 4, [1000, 321, 640, 5]),
    (2, 32, 1, 128, 16, 6, [1, 1], [333, 200]),                       # two row tiles
    (2, 4, 2, 64, 16, 4, [40, 7], [200, 7]),                          # prompts
    (1, 6, 2, 128, 16, 3, [33], [20]),                                # tokens before the first key
    (1, 2, 1, 64, 16, 40, [1], [3000]),                               # more pages than a block scores at once
    (1, 2, 1, 64, 16, 5, [18], [24700]),                              # a prompt whose scores no block holds: two kernels
    (1, 2, 2, 64, 16, 600, [1], [20000]),                             # a long list out of a long table
    (2, 4, 2, 64, 16, 1024, [1, 3], [90, 500]),                       # room for more pages than there are
    (20, 8, 8, 64, 16, 20, [1] * 20, [(37 * i) % 700 for i in range(20)]),  # units beyond one block an SM
]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("B,hq,hkv,d,page,select,q_lens,kv_lens", SELECT)
def test_selected_pages(A, B, hq, hkv, d, page, select, q_lens, kv_lens, dtype):
    c = _paged(200 + B, B, hq, hkv, d, page, dtype, 0, q_lens, kv_lens)
    scale8 = torch.full((hkv,), 30.0)
    summary = R.page_summary(torch.nan_to_num(c["kc"].float(), nan=0.0), scale8)
    want, want_pages = R.select_attention(c["q"], c["kc"], c["vc"], summary, c["table"], c["lens"], select, c["starts"], d ** -0.5)
    q, kc, vc, sm, table, lens, starts = _cuda(c["q"], c["kc"], c["vc"], summary, c["table"], c["lens"], c["starts"])
    got, pages = A.selected_page_attention(q, kc, vc, sm, table, lens, select, q_start=starts, max_q_len=c["max_q"])
    assert torch.equal(pages.cpu(), want_pages)
    vmax = c["vc"][torch.isfinite(c["vc"])].abs().max().item()
    _check(got, want, dtype, vmax)
    A.device_status()


@pytest.mark.parametrize("n_pages", [30, 1500])
def test_ties_go_to_the_lowest_page(A, n_pages):
    """Equal summaries, and a few better ones: the better ones and then the first of the equal ones."""
    page, d, select = 16, 64, 9
    g = _gen(3)
    summary = torch.zeros(n_pages, 1, 2, d, dtype=torch.int8)
    summary[:, :, 0], summary[:, :, 1] = -20, 20
    better = [n_pages - 2, 7, 19]
    summary[better, :, 1] = 21
    kc, vc = _randn((n_pages, 1, page, d), BF16, g), _randn((n_pages, 1, page, d), BF16, g)
    q = torch.rand(1, 2, d, generator=g).to(BF16) + 0.5
    table = torch.arange(n_pages, dtype=torch.int32)[None]
    lens = torch.tensor([n_pages * page], dtype=torch.int32)
    _, pages = A.selected_page_attention(*_cuda(q, kc, vc, summary, table, lens), select)
    rest = [i for i in range(n_pages) if i not in better][:select - 1 - len(better)]
    assert pages.cpu().flatten().tolist() == sorted(better + rest) + [n_pages - 1]
    # all equal: simply the first
    summary[better, :, 1] = 20
    _, pages = A.selected_page_attention(*_cuda(q, kc, vc, summary, table, lens), select)
    assert pages.cpu().flatten().tolist() == list(range(select - 1)) + [n_pages - 1]
    # a query of zeros scores every page 0
    _, pages = A.selected_page_attention(*_cuda(torch.zeros_like(q), kc, vc, summary, table, lens), select)
    assert pages.cpu().flatten().tolist() == list(range(select - 1)) + [n_pages - 1]


def test_scores_at_the_ends_of_their_range(A):
    """Largest group and channels, all bytes at their ends: the digits and sums must not overflow."""
    n_pages, page, d, G = 40, 16, 128, 64
    summary = torch.full((n_pages, 1, 2, d), 127, dtype=torch.int8)
    summary[:, :, 0] = -127
    for i in range(n_pages):
        summary[i, :, 1, :i + 1] = 127 - i
    g = _gen(6)
    q = torch.where(torch.rand(1, G, d, generator=g) < 0.5, -3.0, 3.0).to(BF16)
    kc, vc = _randn((n_pages, 1, page, d), BF16, g), _randn((n_pages, 1, page, d), BF16, g)
    table, lens = torch.arange(n_pages, dtype=torch.int32)[None], torch.tensor([n_pages * page], dtype=torch.int32)
    want, want_pages = R.select_attention(q, kc, vc, summary, table, lens, 8, None, d ** -0.5)
    got, pages = A.selected_page_attention(*_cuda(q, kc, vc, summary, table, lens), 8)
    assert torch.equal(pages.cpu(), want_pages)
    _check(got, want, BF16, vc.abs().max().item())


def test_selecting_every_page_is_plain_attention(A):
    B, page, d = 3, 16, 128
    c = _paged(11, B, 4, 2, d, page, BF16, 0, [1] * B, [100, 5, 77], poison=False)
    q, kc, vc, table, lens = _cuda(c["q"], c["kc"], c["vc"], c["table"], c["lens"])
    summary = torch.zeros(kc.shape[0], 2, 2, d, dtype=torch.int8, device="cuda")
    got, _ = A.selected_page_attention(q, kc, vc, summary, table, lens, 7)
    plain = A.shared_prefix_attention(q, kc, vc, None, 0, table, lens)
    _check(got, plain.double().cpu(), BF16, c["vc"].abs().max().item())


def test_the_summary_that_append_keeps_is_the_cache_s(A):
    """A prompt and then single tokens: the summaries are those of the cache's keys."""
    g = _gen(12)
    page, d, hkv, n = 16, 64, 2, 75
    kc, vc = (torch.zeros(8, hkv, page, d, dtype=BF16, device="cuda") for _ in range(2))
    summary = torch.full((8, hkv, 2, d), 99, dtype=torch.int8, device="cuda")
    scale = torch.tensor([25.0, 40.0])
    table = torch.randperm(8, generator=g)[:5]
    k = _randn((n, hkv, d), BF16, g).cuda()
    slots = torch.tensor([int(table[i // page]) * page + i % page for i in range(n)]).cuda()
    A.kv_append(k[:50], k[:50], kc, vc, slots[:50], summary=summary, summary_scale=scale.cuda())
    for i in range(50, n):
        A.kv_append(k[i:i + 1], k[i:i + 1], kc, vc, slots[i:i + 1], summary=summary, summary_scale=scale.cuda())
    lens = torch.zeros(8, dtype=torch.int64)
    for j in range(5):
        lens[table[j]] = min(page, n - j * page)
    want = R.page_summary(kc.cpu(), scale, lens)
    for j in table.tolist():
        assert torch.equal(summary.cpu()[j], want[j])


def test_cache_offsets_past_32_bits(A):
    """Pages whose element offset passes 2^31 and whose byte offset passes 2^32."""
    page, hkv, d = 128, 16, 128
    pages = (2 ** 31) // (page * hkv * d) + 40
    kc = torch.zeros(pages, hkv, page, d, dtype=BF16, device="cuda")
    vc = torch.zeros(pages, hkv, page, d, dtype=BF16, device="cuda")
    summary = torch.zeros(pages, hkv, 2, d, dtype=torch.int8, device="cuda")
    g = _gen(13)
    n = 200
    mine = [pages - 1, pages - 3]
    slots = torch.tensor([mine[i // page] * page + i % page for i in range(n)]).cuda()
    k, v = _randn((n, hkv, d), BF16, g), _randn((n, hkv, d), BF16, g)
    A.kv_append(k.cuda(), v.cuda(), kc, vc, slots, summary=summary, summary_scale=torch.full((hkv,), 30.0).cuda())
    q = _randn((1, hkv, d), BF16, g)
    table, lens = torch.tensor([mine], dtype=torch.int32), torch.tensor([n], dtype=torch.int32)
    want = torch.stack([R.attend(q[0, h:h + 1], k[:, h], v[:, h], d ** -0.5)[0] for h in range(hkv)])[None]
    vmax = v.abs().max().item()
    qd, td, ld = _cuda(q, table, lens)
    _check(A.shared_prefix_attention(qd, kc, vc, None, 0, td, ld), want, BF16, vmax)
    _check(A.shared_prefix_attention(qd, kc, vc, td[0], n, td, torch.zeros_like(ld)), want, BF16, vmax)
    _check(A.selected_page_attention(qd, kc, vc, summary, td, ld, 2)[0], want, BF16, vmax)
    A.device_status()


def test_all_in_a_graph(A):
    """A decode step captured once and replayed on new data gives what the calls give."""
    B, hq, hkv, d, page = 4, 4, 2, 64, 16
    c = _paged(14, B, hq, hkv, d, page, BF16, 50, [1] * B, [20, 33, 1, 16], poison=False)
    q, kc, vc, pre, table, lens = _cuda(c["q"], c["kc"], c["vc"], c["pre"], c["table"], c["lens"])
    summary = torch.zeros(kc.shape[0], hkv, 2, d, dtype=torch.int8, device="cuda")
    scale = torch.full((hkv,), 30.0, device="cuda")
    k, v = _randn((B, hkv, d), BF16, _gen(1)).cuda(), _randn((B, hkv, d), BF16, _gen(2)).cuda()
    slots = torch.tensor([int(table[b, (int(lens[b]) - 1) // page]) * page + (int(lens[b]) - 1) % page for b in range(B)], device="cuda")

    def step():
        A.kv_append(k, v, kc, vc, slots, summary=summary, summary_scale=scale)
        o = A.shared_prefix_attention(q, kc, vc, pre, 50, table, lens)
        return o, *A.selected_page_attention(q, kc, vc, summary, table, lens, 2)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    q.copy_(_randn(q.shape, BF16, _gen(15)))
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(captured, step()):
        assert torch.equal(a, b)
