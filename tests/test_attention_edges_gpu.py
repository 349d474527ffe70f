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
