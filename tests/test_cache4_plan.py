"""How the attention over the 4-bit cache divides its work (csrc/cache4_plan.h), without a GPU: the header is host arithmetic alone and is
compiled here with the host compiler, for 148 SMs; the kernel's part of the division is restated below."""
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF16, F32 = 1, 0


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("plan") / "probe")
    proc = subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", os.path.join(ROOT, "tests", "cache4_plan_probe.cpp"), "-o", exe],
                          capture_output=True, text=True)
    assert proc.returncode == 0, proc.stderr

    def run(*numbers):
        proc = subprocess.run([exe], input=" ".join(map(str, numbers)) + "\n", capture_output=True, text=True)
        assert proc.returncode == 0
        return {k: int(v) for k, v in (word.split("=") for word in proc.stdout.split())}
    return run


def div_up(a, b):
    return -(-a // b)


def unit_rows(f):
    return 256 if f["umma"] else 8 * f["row_tiles"]


def division(f, lens, counts, group, hkv):
    """Runs of the kernel: (total grains, grains of a run, grains of each unit)."""
    units = []
    for n, c in zip(lens, counts):
        grains = max(1, div_up(n, 16 << f["grain"]))
        units += [grains] * (hkv * div_up(c * group, unit_rows(f)))
    total = sum(units)
    return total, max(div_up(total, f["warps"]), f["least"]), units


@pytest.mark.parametrize("seed", range(40))
def test_every_part_has_its_place(plan, seed):
    r = random.Random(seed)
    B, hkv, group = r.choice([1, 2, 7, 64, 300]), r.choice([1, 2, 8, 32]), r.choice([1, 3, 4, 16])
    page, width, max_q = r.choice([16, 64, 128]), r.choice([1, 5, 100, 2000]), r.choice([1, 1, 2, 33])
    dtype, D = r.choice([BF16, F32]), r.choice([64, 96, 128])
    counts = [r.randint(0, max_q) if max_q > 1 else 1 for _ in range(B)]
    lens = [r.randint(0, width * page) for _ in range(B)]
    f = plan(width, sum(counts), B, max_q, group * hkv, hkv, D, page, dtype, 1)
    if sum(counts) == 0:
        assert f["bytes"] == 0
        return
    total, run, units = division(f, lens, counts, group, hkv)
    assert total < 2 ** 31 and run * f["warps"] < 2 ** 32
    assert div_up(total, run) <= f["warps"]                       # every grain has a run
    # parts of units that lie in several runs: the first in its run's second place, the others in their runs' first
    at, used = 0, set()
    for grains in units:
        first, last = at // run, (at + grains - 1) // run
        if last > first:
            for w in range(first, last + 1):
                slot = 2 * w + (1 if w == first else 0)
                assert slot not in used and slot < 2 * f["warps"]
                used.add(slot)
        at += grains
    assert f["part_rows"] >= min(unit_rows(f), max(counts) * group)
    slots = 2 * f["warps"] * f["part_rows"]
    assert f["ml_bytes"] >= slots * 8 and f["o_bytes"] >= slots * D * 4
    assert f["lse_bytes"] >= sum(counts) * group * hkv * 4
    assert f["bytes"] >= f["ml_bytes"] + f["o_bytes"] + f["lse_bytes"] + f["scores_bytes"]
    if f["scores_bytes"]:
        assert f["row_tiles"] == 1 and f["scores_bytes"] >= 4 * B * hkv * width * page * f["part_rows"]


@pytest.mark.parametrize("B,hkv,width,page,max_q,group", [
    (4096, 32, 16000, 128, 1, 4), (1, 1, 16777214, 128, 1, 1), (4096, 64, 16777214, 128, 1, 64), (1000, 8, 100000, 16, 1 << 20, 64)])
def test_grains_fit_32_bits(plan, B, hkv, width, page, max_q, group):
    """At the widest tables, all full."""
    T = B if max_q == 1 else 1000
    f = plan(width, T, B, max_q, group * hkv, hkv, 128, page, BF16, 0)
    units = hkv * min(B * div_up(min(max_q, T) * group, unit_rows(f)), div_up(T * group, unit_rows(f)) + B)
    total = units * max(1, div_up(width * page, 16 << f["grain"]))
    run = max(div_up(total, f["warps"]), f["least"])
    assert total < 2 ** 31 + units and total < 2 ** 32 and run * f["warps"] < 2 ** 32


def test_which_kernel(plan):
    """Single tokens, short prompts and fp32 rows on the kernel of few rows, long prompts over long contexts on tcgen05."""
    def umma(width, T, B, max_q, hq, hkv, dtype=BF16):
        return plan(width, T, B, max_q, hq, hkv, 128, 64, dtype, 0)["umma"] == 1
    assert umma(469, 128, 1, 128, 32, 8) and umma(63, 2048, 1, 2048, 32, 8)
    assert not umma(469, 128, 1, 128, 32, 8, F32)
    assert not umma(256, 64, 64, 1, 32, 8) and not umma(16, 300, 1, 300, 8, 8) and not umma(79, 260, 8, 64, 16, 4)


def test_the_workspace_does_not_grow_with_the_table(plan):
    """(The scores for the received weight do, up to a gigabyte.)"""
    small = plan(100, 64, 64, 1, 32, 8, 128, 64, BF16, 0)["bytes"]
    assert plan(100000, 64, 64, 1, 32, 8, 128, 64, BF16, 0)["bytes"] <= small <= 2 * 148 * 16 * 4 * (128 * 4 + 8) + 512
    assert plan(1000, 64, 64, 1, 32, 8, 128, 64, BF16, 1)["scores_bytes"] == 4 * 4 * 64 * 8 * 64000
    assert plan(100000, 64, 64, 1, 32, 8, 128, 64, BF16, 1)["scores_bytes"] == 0
    assert plan(10, 64, 64, 4, 32, 8, 128, 64, BF16, 1)["scores_bytes"] == 0
    assert plan(1000, 0, 64, 4, 32, 8, 128, 64, BF16, 1)["bytes"] == 0


@pytest.mark.parametrize("d,hq,hkv,page,lens,counts", [
    (128, 32, 8, 64, [5000], [600]), (128, 8, 2, 128, [16001, 9000, 700], [513, 1, 700]), (96, 12, 4, 32, [7000, 0, 40, 4000], [800, 3, 64, 1]),
    (64, 16, 16, 16, [3000, 2999], [900, 411]), (64, 64, 1, 64, [12000], [77]), (128, 16, 4, 64, [6000], [500]), (96, 16, 4, 64, [5000], [500]),
    (128, 8, 2, 64, [5000], [600]), (128, 32, 8, 64, [5000, 4000], [600, 500])])
def test_the_sizes_of_the_prompt_tests(plan, d, hq, hkv, page, lens, counts):
    """They are to reach the tcgen05 kernel (test_cache4_prompts_gpu.py)."""
    width = max(1, max(div_up(n, page) for n in lens))
    assert plan(width, sum(counts), len(lens), max(counts), hq, hkv, d, page, BF16, 0)["umma"] == 1
