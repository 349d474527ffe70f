"""Serving attention without a GPU: every declared function is exported, and bad arguments are refused before any
CUDA work, by the C entry points and by the Python calls."""
import ctypes
import os
import re

import pytest
import torch

import attention_ref as R

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
    text = open(os.path.join(ROOT, "include", "wht_attention.h")).read()
    names = sorted(set(re.findall(r"\b(wht_[a-z_0-9]+)\s*\(", re.sub(r"/\*.*?\*/", "", text, flags=re.S))))
    assert sorted(binding.ATTENTION_EXPORTS) == names
    for name in names:
        assert hasattr(lib, name)
    assert b"out of range" in lib.wht_affine_status_string(-11)


def _pointers():
    buf = (ctypes.c_char * 4096)()
    p = ctypes.c_void_p((ctypes.addressof(buf) + 15) & ~15)
    return buf, p, ctypes.c_void_p(p.value + 8)


def _append(lib, p, **kw):
    a = dict(k=p, k_st=128, k_sh=64, v=p, v_st=128, v_sh=64, q=p, q_st=256, q_sh=64, q_out=p, slots=p, positions=p, cos=p, sin=p, kc=p, vc=p,
             summary=p, scale=p, T=3, hq=4, hkv=2, d=64, rot=64, inter=0, max_pos=10, pages=5, page=16, dtype=1, stream=None)
    assert set(kw) <= set(a)
    a.update(kw)
    return lib.wht_kv_append(*a.values())


def test_append_refusals(lib):
    keep, p, off = _pointers()
    for kw, want in [
        (dict(dtype=2), DTYPE), (dict(dtype=7), DTYPE), (dict(d=80), DIM), (dict(d=256), DIM), (dict(hq=3), DIM), (dict(hkv=0), DIM),
        (dict(hq=130, hkv=2), DIM), (dict(page=48), DIM), (dict(page=256), DIM), (dict(pages=-1), DIM), (dict(rot=8), DIM), (dict(rot=80), DIM),
        (dict(rot=-16), DIM), (dict(max_pos=0), DIM), (dict(T=-1), BAD_T), (dict(T=1 << 40), BAD_T), (dict(k=None), NULL), (dict(slots=None), NULL),
        (dict(vc=None), NULL), (dict(q_out=None), NULL), (dict(q=None), NULL), (dict(cos=None), NULL), (dict(positions=None), NULL),
        (dict(scale=None), NULL), (dict(k=off), MISALIGNED), (dict(q_out=off), MISALIGNED), (dict(k_st=100), MISALIGNED), (dict(q_sh=68), MISALIGNED),
        (dict(sin=off), MISALIGNED), (dict(summary=off), MISALIGNED), (dict(T=0), OK), (dict(T=0, k=None, slots=None), OK),
    ]:
        assert _append(lib, p, **kw) == want, kw


def _attend(lib, name, p, **kw):
    a = dict(q=p, q_st=256, q_sh=64, kc=p, vc=p)
    if name == "wht_attn_prefix":
        a.update(pre=p, prefix=100, table=p, width=4, lens=p, start=None, out=p)
    else:
        a.update(summary=p, table=p, width=4, lens=p, start=None, select=2, out=p, pages_out=p)
    a.update(T=3, B=3, max_q=1, hq=4, hkv=2, d=64, pages=9, page=16, scale=0.125, dtype=1, ws=p, ws_bytes=0, stream=None)
    assert set(kw) <= set(a)
    a.update(kw)
    return getattr(lib, name)(*a.values())


@pytest.mark.parametrize("name", ["wht_attn_prefix", "wht_attn_select"])
def test_attention_refusals(lib, name):
    keep, p, off = _pointers()
    cases = [
        (dict(dtype=2), DTYPE), (dict(d=72), DIM), (dict(hq=5), DIM), (dict(page=8), DIM), (dict(width=-1), DIM), (dict(max_q=0), DIM),
        (dict(width=1 << 30), DIM), (dict(T=-1), BAD_T), (dict(T=4), BAD_T), (dict(max_q=2), BAD_T), (dict(q=None), NULL), (dict(kc=None), NULL),
        (dict(out=None), NULL), (dict(lens=None), NULL), (dict(table=None), NULL), (dict(vc=off), MISALIGNED), (dict(out=off), MISALIGNED),
        (dict(q_st=100), MISALIGNED), (dict(T=0, B=0), OK),
    ]
    if name == "wht_attn_prefix":
        cases += [(dict(prefix=-1), BAD_T), (dict(pre=None), NULL)]
    else:
        cases += [(dict(select=0), DIM), (dict(select=1025), DIM), (dict(width=50000), DIM), (dict(summary=None), NULL), (dict(pages_out=None), NULL),
                  (dict(summary=off), MISALIGNED)]
    for kw, want in cases:
        assert _attend(lib, name, p, **kw) == want, kw


def test_python_calls_refuse_tensors_that_are_not_on_a_gpu(lib):
    from paper_2603_08343_b200 import attention as A
    kc = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    k = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        A.kv_append(k, k, kc, kc, torch.zeros(3, dtype=torch.int64))
    with pytest.raises(ValueError):
        A.shared_prefix_attention(k, kc, kc[:, :1], None, 0, torch.zeros(3, 1, dtype=torch.int32), torch.ones(3, dtype=torch.int32))
    with pytest.raises(ValueError):
        A.kv_append(k, k, kc.half(), kc.half(), torch.zeros(3, dtype=torch.int64))


# ---- the plain statements themselves

def test_reference_rotation_turns_pairs():
    cos, sin = R.inverse_frequencies(16, 4)
    x = torch.randn(4, 1, 32)
    y = R.rotate(x, torch.arange(4), cos, sin, False)
    assert torch.allclose(y.norm(dim=-1), x.double().norm(dim=-1), atol=1e-5)
    assert torch.equal(y[0], x[0].double()) and torch.equal(y[..., 16:], x[..., 16:].double())
    # scores of rotated pairs depend on the distance alone
    q = R.rotate(x[:1].expand(4, 1, 32), torch.arange(4), cos, sin, True)
    k = R.rotate(x[1:2].expand(4, 1, 32), torch.arange(4), cos, sin, True)
    assert abs((q[2, 0] @ k[1, 0]) - (q[3, 0] @ k[2, 0])) < 1e-5


def test_reference_selection_bounds_every_key():
    """A page's score is at least the whole-number score of each of its keys."""
    g = torch.Generator()
    g.manual_seed(1)
    kc = torch.randn(5, 1, 16, 64, generator=g)
    scale = torch.tensor([30.0])
    s = R.page_summary(kc, scale)
    q8 = R.whole_queries(torch.randn(4, 64, generator=g))
    k8 = (kc[:, 0] * 30.0).round().clamp(-127, 127).to(torch.int64)
    low, high = s[:, 0, 0].to(torch.int64), s[:, 0, 1].to(torch.int64)
    for p in range(5):
        bound = torch.maximum(q8 * low[p], q8 * high[p]).sum()
        assert (q8.sum(0) * k8[p]).sum(-1).max() <= bound
