"""Tables so wide, of so many sequences, that the attention over the 4-bit cache counts its work in larger grains."""
import os
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PAGE, PAGES, HKV, D = 128, 48, 32, 64
# table width, sequences, most tokens of one, heads of a key head, type, grain (log2 of its tiles of 16 keys; 1 and, in the tcgen05 kernel, 2 elsewhere)
CALLS = [(262144, 64, 1, 4, "bf16", 2), (262144, 64, 1, 8, "bf16", 2), (262144, 64, 3, 4, "fp32", 2), (131072, 150, 1, 2, "fp32", 2), (900000, 64, 1, 1, "bf16", 3),
         (262144, 64, 3, 4, "bf16", 2), (900000, 64, 32, 4, "bf16", 3), (900000, 64, 9, 4, "bf16", 5)]


@pytest.mark.parametrize("width,batch,tokens,group,dtype,grain", CALLS)
def test_these_calls_do(tmp_path, width, batch, tokens, group, dtype, grain):
    exe = str(tmp_path / "probe")
    subprocess.run(["g++", "-std=c++17", "-O1", os.path.join(ROOT, "tests", "cache4_plan_probe.cpp"), "-o", exe], check=True)
    numbers = (width, batch * tokens, batch, tokens, group * HKV, HKV, D, PAGE, 1 if dtype == "bf16" else 0, 0)
    words = subprocess.run([exe], input=" ".join(map(str, numbers)) + "\n", capture_output=True, text=True, check=True).stdout.split()
    plan = {k: int(v) for k, v in (word.split("=") for word in words)}
    assert plan["grain"] == grain and plan["umma"] == (tokens == 32)


@pytest.mark.gpu
@pytest.mark.parametrize("width,batch,tokens,group,dtype,grain", CALLS)
def test_results_of_wide_and_narrow_tables(width, batch, tokens, group, dtype, grain):
    """Short and ragged sequences, what lies behind them no pages at all.  The runs divide otherwise than with a narrow table: bf16 results are two roundings
    apart at most (2^-7 of the norm), fp32 ones what weights of 22 bits and fp32 sums come to (2^-17)."""
    from paper_2603_08343_b200 import build
    build.build()
    from paper_2603_08343_b200 import attention as A
    g = torch.Generator(device="cuda")
    g.manual_seed(width + tokens)
    cache = A.cache4(PAGES, HKV, PAGE, D)
    k, v = (torch.randn(PAGES * PAGE, HKV, D, device="cuda", generator=g) for _ in range(2))
    A.kv_append4(k, v, cache, torch.arange(PAGES * PAGE, device="cuda"))
    kind = torch.bfloat16 if dtype == "bf16" else torch.float32
    narrow = torch.randint(0, PAGES, (batch, 40), device="cuda", generator=g).int()
    lens = torch.randint(1, 40 * PAGE + 1, (batch,), device="cuda", generator=g).int()
    counts = torch.randint(0, tokens + 1, (batch,), device="cuda", generator=g) if tokens > 1 else torch.ones(batch, dtype=torch.int64, device="cuda")
    counts[3:5] = tokens
    lens[:4] = torch.tensor([0, 1, 40 * PAGE, 17], dtype=torch.int32)
    starts = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), counts.cumsum(0)]).int()
    T = int(starts[-1])
    q = torch.randn(T, HKV * group, D, device="cuda", generator=g).to(kind)
    wide = torch.full((batch, width), 1 << 30, dtype=torch.int32, device="cuda")
    wide[:, :40] = narrow
    wide[torch.arange(width, device="cuda")[None, :40].expand(batch, 40).ge(-(-lens[:, None] // PAGE)).nonzero(as_tuple=True)] = -1
    args = dict(q_start=None if tokens == 1 else starts, max_q_len=tokens)
    want = A.paged_attention4(q, cache, narrow, lens, **args)
    got = A.paged_attention4(q, cache, wide, lens, **args)
    A.device_status()
    assert (got - want).norm(dtype=torch.float64) <= (2.0 ** -7 if dtype == "bf16" else 2.0 ** -17) * want.norm(dtype=torch.float64)
    assert torch.isfinite(got).all() and torch.equal(got, A.paged_attention4(q, cache, wide, lens, **args))
