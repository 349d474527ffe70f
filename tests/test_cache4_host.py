"""The 4-bit cache without a GPU: exports, refusals before any CUDA work, the division of the work, and the plain statements themselves."""
import ctypes
import os
import re

import pytest
import torch

import cache4_ref as C

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, NULL, DIM, BAD_T, DTYPE, MISALIGNED = 0, -1, -2, -3, -4, -5


@pytest.fixture(scope="module")
def lib():
    from paper_2603_08343_b200 import build
    build.build()
    from paper_2603_08343_b200 import binding
    return binding.lib()


def test_every_declared_symbol_is_exported(lib):
    from paper_2603_08343_b200 import binding
    text = open(os.path.join(ROOT, "include", "wht_cache4.h")).read()
    names = sorted(set(re.findall(r"\b(wht_[a-z_0-9]+)\s*\(", re.sub(r"/\*.*?\*/", "", text, flags=re.S))))
    assert sorted(binding.CACHE4_EXPORTS) == names
    for name in names:
        assert hasattr(lib, name)


def _pointers():
    buf = (ctypes.c_char * 4096)()
    p = ctypes.c_void_p((ctypes.addressof(buf) + 15) & ~15)
    return buf, p, ctypes.c_void_p(p.value + 8)


def _append(lib, p, **kw):
    a = dict(k=p, k_st=128, k_sh=64, v=p, v_st=128, v_sh=64, q=p, q_st=256, q_sh=64, q_out=p, slots=p, positions=p, cos=p, sin=p, cache=p,
             T=3, hq=4, hkv=2, d=64, rot=64, inter=0, max_pos=10, pages=5, page=16, dtype=1, stream=None)
    assert set(kw) <= set(a)
    a.update(kw)
    return lib.wht_kv_append4(*a.values())


def test_append_refusals(lib):
    keep, p, off = _pointers()
    for kw, want in [
        (dict(dtype=2), DTYPE), (dict(d=80), DIM), (dict(d=256), DIM), (dict(hq=3), DIM), (dict(hkv=0), DIM), (dict(hq=130, hkv=2), DIM),
        (dict(page=48), DIM), (dict(pages=-1), DIM), (dict(rot=8), DIM), (dict(rot=80), DIM), (dict(rot=-16), DIM), (dict(max_pos=0), DIM),
        (dict(T=-1), BAD_T), (dict(T=1 << 40), BAD_T), (dict(k=None), NULL), (dict(slots=None), NULL), (dict(cache=None), NULL),
        (dict(q_out=None), NULL), (dict(q=None), NULL), (dict(cos=None), NULL), (dict(positions=None), NULL), (dict(k=off), MISALIGNED),
        (dict(q_out=off), MISALIGNED), (dict(cache=off), MISALIGNED), (dict(k_st=100), MISALIGNED), (dict(q_sh=68), MISALIGNED),
        (dict(sin=off), MISALIGNED), (dict(T=0), OK), (dict(T=0, k=None, slots=None), OK),
    ]:
        assert _append(lib, p, **kw) == want, kw


def test_read_refusals(lib):
    keep, p, off = _pointers()

    def read(cache=p, slots=p, k=p, v=p, n=3, hkv=2, d=64, pages=5, page=16, dtype=0):
        return lib.wht_kv_read4(cache, slots, k, v, n, hkv, d, pages, page, dtype, None)
    assert [read(dtype=5), read(d=65), read(page=8), read(n=-1), read(cache=None), read(slots=None), read(v=None), read(k=off), read(n=0)] == \
        [DTYPE, DIM, DIM, BAD_T, NULL, NULL, NULL, MISALIGNED, OK]


def _attend(lib, p, **kw):
    a = dict(q=p, q_st=256, q_sh=64, cache=p, table=p, width=4, lens=p, start=None, out=p, weights=None, weights_out=None, T=3, B=3, max_q=1,
             hq=4, hkv=2, d=64, pages=9, page=16, scale=0.125, dtype=1, ws=p, ws_bytes=0, stream=None)
    assert set(kw) <= set(a)
    a.update(kw)
    return lib.wht_attn_paged4(*a.values())


def test_attention_refusals(lib):
    keep, p, off = _pointers()
    for kw, want in [
        (dict(dtype=2), DTYPE), (dict(d=72), DIM), (dict(hq=5), DIM), (dict(page=8), DIM), (dict(width=-1), DIM), (dict(max_q=0), DIM),
        (dict(width=1 << 30), DIM), (dict(T=-1), BAD_T), (dict(T=4), BAD_T), (dict(max_q=2), BAD_T), (dict(q=None), NULL), (dict(cache=None), NULL),
        (dict(out=None), NULL), (dict(lens=None), NULL), (dict(table=None), NULL), (dict(weights=p), NULL), (dict(cache=off), MISALIGNED),
        (dict(out=off), MISALIGNED), (dict(weights_out=off), MISALIGNED), (dict(weights=off, weights_out=p), MISALIGNED), (dict(q_st=100), MISALIGNED),
        (dict(ws=off), MISALIGNED), (dict(T=0, B=0), OK), (dict(T=0, B=0, weights_out=p), OK),
    ]:
        assert _attend(lib, p, **kw) == want, kw


def _evict(lib, p, **kw):
    other = [ctypes.c_void_p(p.value + 16 * (i + 1)) for i in range(6)]
    a = dict(cache=p, table=other[0], width=4, lens=other[1], weights=other[2], out_table=other[3], out_width=2, lens_out=other[4],
             weights_out=other[5], kept=p, B=3, hkv=2, d=64, pages=9, page=16, budget=20, first=2, last=3, stream=None)
    assert set(kw) <= set(a)
    a.update(kw)
    return lib.wht_kv_evict4(*a.values())


def test_eviction_refusals(lib):
    keep, p, off = _pointers()
    for kw, want in [
        (dict(d=72), DIM), (dict(page=8), DIM), (dict(hkv=0), DIM), (dict(width=-1), DIM), (dict(width=1 << 27), DIM), (dict(out_width=1), DIM),
        (dict(budget=0), DIM), (dict(budget=33), DIM), (dict(first=-1), DIM), (dict(first=18), DIM), (dict(first=(1 << 31) - 1, last=(1 << 31) - 1), DIM),
        (dict(B=-1), BAD_T), (dict(cache=None), NULL), (dict(table=None), NULL), (dict(lens=None), NULL), (dict(weights=None), NULL),
        (dict(out_table=None), NULL), (dict(lens_out=None), NULL), (dict(weights_out=None), NULL), (dict(kept=None), NULL),
        (dict(cache=off), MISALIGNED), (dict(weights=off), MISALIGNED), (dict(weights_out=off), MISALIGNED), (dict(B=0), OK),
        (dict(lens_out=ctypes.c_void_p(p.value + 32)), DIM),          # written while other blocks read it
    ]:
        assert _evict(lib, p, **kw) == want, kw


def test_python_calls_refuse_what_is_not_a_cache_on_a_gpu(lib):
    from paper_2603_08343_b200 import attention as A
    cache = A.cache4(4, 2, 16, 64, device="cpu")
    assert cache.shape == (4, 2, 1, 16 * 64 + 128) and cache.dtype == torch.uint8
    k = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    table, lens, slots = torch.zeros(3, 1, dtype=torch.int32), torch.ones(3, dtype=torch.int32), torch.zeros(3, dtype=torch.int64)
    for call in (lambda: A.kv_append4(k, k, cache, slots), lambda: A.kv_read4(cache, slots), lambda: A.paged_attention4(k, cache, table, lens),
                 lambda: A.kv_evict4(cache, table, lens, torch.zeros(3, 2, 16), table, 4), lambda: A.kv_read4(cache, slots, dtype=torch.float16),
                 lambda: A.paged_attention4(k.half(), cache, table, lens), lambda: A.cache4(4, 2, 24, 64), lambda: A.cache4(4, 2, 16, 80)):
        with pytest.raises(ValueError):
            call()


# ---- the plain statements themselves

def test_a_held_row_is_within_half_a_step():
    g = torch.Generator()
    g.manual_seed(0)
    x = torch.randn(200, 96, generator=g) * 10.0 ** torch.randint(-5, 6, (200, 1), generator=g)
    held = C.hold(x)
    spread = x.amax(-1) - x.amin(-1)
    assert ((x - held).abs().amax(-1) <= spread / 30 + 2 ** -8 * (x.abs().amax(-1) + spread)).all()
    assert all(len(set(row.tolist())) <= 16 for row in held)
    assert torch.equal(C.hold(torch.full((1, 64), 1.5)), torch.full((1, 64), 1.5))


def test_reference_keeps_the_heaviest():
    w = [5.0, 1.0, 3.0, 3.0, 0.0, 3.0, 9.0, 2.0]
    assert C.keep(w, 8, 8, 0, 0) == list(range(8))
    assert C.keep(w, 8, 4, 0, 0) == [0, 2, 3, 6]
    assert C.keep(w, 8, 4, 0, 2) == [0, 2, 6, 7]
    assert C.keep(w, 8, 3, 2, 1) == [0, 1, 7]
    assert C.keep([1.0, float("nan"), -1.0], 3, 2, 0, 0) == [0, 2]


def test_reference_weights_sum_to_the_rows():
    q, k = torch.randn(5, 4, 64), [torch.randn(7, 2, 64), torch.randn(3, 2, 64)]
    _, received = C.attention(q, k, k, [7, 3], torch.tensor([0, 2, 5]), 0.1)
    assert abs(received[0].sum().item() - 8) < 1e-9 and abs(received[1].sum().item() - 12) < 1e-9
