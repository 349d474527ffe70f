"""What the 4-bit cache holds, to the last bit: bf16 reads, and how far a held row may be from what was appended."""
import pytest
import torch

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


def nearest_bf16(x):
    """fp64 numbers (normal ones in bf16's range, and zeros) to the nearest of 8 bits, ties to even: one rounding, where .bfloat16() has two."""
    m, e = torch.frexp(x)
    return torch.ldexp(torch.round(torch.ldexp(m, torch.tensor(8))), e - 8)


def parts(x):
    """lo, step and codes of rows [n, d], as their definition has them, in 64 bits."""
    lo = x.float().amin(-1).bfloat16().float()
    step = ((x.float().amax(-1) - lo) * torch.tensor(1.0 / 15.0)).bfloat16().float()
    codes = ((x.float() - lo[:, None]) * (1.0 / step)[:, None]).round().clamp(0, 15)
    return lo.double()[:, None], step.double()[:, None], codes.double()


@pytest.mark.parametrize("d", [64, 96, 128])
def test_bf16_reads_are_rounded_once(A, d):
    """Least values far below the step, of either sign: products of nine bits and more lie half way between two bf16 numbers, and the least value
    says which it is."""
    rows = []
    for i, step in enumerate((129 / 128, 131 / 128, 1.5, 255 / 128, 2.0 ** -30 * 137 / 128)):
        for tiny in (0.0, 2.0 ** -22, 2.0 ** -33, -2.0 ** -26, -2.0 ** -36):
            x = torch.arange(d).remainder(16).double().roll(i) * step
            x[x == 0] = tiny * step
            rows.append(x)
    g = torch.Generator()
    g.manual_seed(d)
    x = torch.cat([torch.stack(rows), torch.randn(200, d, generator=g).double(), torch.rand(200, d, generator=g).double() * 3 + 1e-9]).float()
    n = x.shape[0]
    lo, step, codes = parts(x)
    cache = A.cache4(n // 16 + 1, 1, 16, d)
    slots = torch.arange(n, device="cuda")
    A.kv_append4(x[:, None].cuda(), x.flip(0)[:, None].contiguous().cuda(), cache, slots)
    want = nearest_bf16(lo + step * codes)                  # (8 + 12 bits up to 2^40 apart: exact in 64 bits)
    k, v = A.kv_read4(cache, slots, BF16)
    assert torch.equal(k[:, 0].cpu().double(), want) and torch.equal(v[:, 0].cpu().double(), want.flip(0))
    k, _ = A.kv_read4(cache, slots, F32)
    assert torch.equal(k[:, 0].cpu(), C.hold(x))
    assert (k[:, 0].cpu().bfloat16().double() != want).any()  # (so the rows do tell the two apart)


@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_channel_is_held_to_half_a_step_or_the_rounding_of_the_least_value(A, dtype, d):
    """... and to the roundings of fp32 on the way: of the reciprocal, the difference and its product, 2^-22 of 15 steps, and of the held value,
    two of 2^-24."""
    g = torch.Generator()
    g.manual_seed(d)
    rows = [torch.rand(d, generator=g) * 0.3 + 100.3]
    for offset in (0.0, 1.0, -1.0, 37.0, -300.3, 1e4, -1e6):
        for spread in (1.0, 0.01, 20.0):
            rows += [torch.randn(d, generator=g) * spread + offset, torch.rand(d, generator=g) * spread + offset]
    x = torch.stack(rows).to(dtype)
    n = x.shape[0]
    cache = A.cache4(n // 16 + 1, 1, 16, d)
    slots = torch.arange(n, device="cuda")
    A.kv_append4(x[:, None].cuda(), x[:, None].cuda(), cache, slots)
    k, _ = A.kv_read4(cache, slots)
    x, k = x.double(), k[:, 0].cpu().double()
    lo = x.amin(-1).float().bfloat16().double()
    step = ((x.amax(-1) - lo).clamp(min=0) / 15) * (1 + 2.0 ** -8)
    least = (2.0 ** -8 * x.amin(-1).abs())
    bound = torch.maximum(step * (0.5 + 15 * 2.0 ** -22), least) + 2.0 ** -23 * k.abs().amax(-1) + 15 * 2.0 ** -100
    assert ((k - x).abs().amax(-1) <= bound).all()
    if dtype == F32:                                        # the row from 100.3 to 100.6: below 100.5 nothing is told apart
        assert (k[0][x[0] < 100.5] == 100.5).all()
