"""How the serving attention divides its work (csrc/attn_plan.h), without a GPU: the header is host arithmetic alone and is
compiled here with the host compiler, for 148 SMs."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF16, F32 = 1, 0


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("plan") / "probe")
    proc = subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", os.path.join(ROOT, "tests", "attn_plan_probe.cpp"), "-o", exe],
                          capture_output=True, text=True)
    assert proc.returncode == 0, proc.stderr

    def run(kind, *numbers):
        line = " ".join([kind, *map(str, numbers)] + ["0"] * (11 - len(numbers)))
        proc = subprocess.run([exe], input=line + "\n", capture_output=True, text=True)
        assert proc.returncode == 0, f"{line}: ended with {proc.returncode}"
        return {k: int(v) for k, v in (word.split("=") for word in proc.stdout.split())}
    return run


EMPTY_PREFIX = [
    # prefix_len, width, T, B, max_q_len, Hq, Hkv, D, page, dtype, tcgen05
    (0, 8, 0, 0, 1, 32, 8, 128, 64, BF16, 1),
    (8192, 8, 0, 0, 1, 32, 8, 128, 64, BF16, 1),
    (8192, 8, 0, 4, 16, 32, 8, 128, 64, BF16, 1),
    (8192, 8, 0, 4, 16, 32, 8, 128, 64, BF16, 0),
    (1000, 4, 0, 0, 1, 12, 12, 64, 16, F32, 0),
    (0, 512, 0, 0, 1, 32, 1, 128, 128, F32, 0),
    (40, 1, 0, 0, 1, 2, 2, 64, 16, BF16, 1),
]


@pytest.mark.parametrize("call", EMPTY_PREFIX)
def test_a_prefix_call_of_no_tokens_needs_nothing(plan, call):
    assert plan("prefix", *call)["bytes"] == 0


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("width,select,hq", [(512, 32, 32), (8, 1024, 8), (2048, 600, 64), (0, 4, 8)])
def test_a_selection_of_no_tokens_needs_nothing(plan, width, select, hq, dtype):
    assert plan("select", width, select, 0, 0, 1, hq, 8, 128, 64, dtype)["bytes"] == 0


@pytest.fixture(scope="module")
def lib():
    from paper_2603_08343_b200 import build
    build.build()
    from paper_2603_08343_b200 import binding
    return binding.lib()


@pytest.fixture(scope="module")
def p():
    import ctypes
    buf = (ctypes.c_char * 4096)()
    yield ctypes.c_void_p((ctypes.addressof(buf) + 15) & ~15)
    del buf


def test_tokens_without_a_sequence_are_refused(lib, p):
    """Through the C entry points, which check before any CUDA work: T = 3 tokens, B = 0 sequences, q_start given."""
    rest = (3, 0, 1, 4, 2, 64, 9, 16, 0.125, BF16, p, 0, None)
    assert lib.wht_attn_prefix(p, 256, 64, p, p, p, 100, p, 4, p, p, p, *rest) == -3
    assert lib.wht_attn_select(p, 256, 64, p, p, p, p, 4, p, p, 2, p, p, *rest) == -3
    assert lib.wht_attn_prefix_workspace_bytes(1000, 64, 3, 0, 1, 4, 2, 64, 16, BF16) == 0
    assert lib.wht_attn_select_workspace_bytes(64, 32, 3, 0, 1, 4, 2, 64, 16, BF16) == 0


def test_the_stride_of_a_dimension_of_one_may_be_anything(lib, p):
    """(Without a GPU the calls then end at the device query.)"""
    def append(T, hkv, st, sh):
        return lib.wht_kv_append(p, st, sh, p, st, sh, p, st, sh, p, p, p, p, p, p, p, None, None, T, hkv, hkv, 64, 64, 0, 10, 5, 16, BF16, None)

    def prefix(T, hkv, st, sh):
        return lib.wht_attn_prefix(p, st, sh, p, p, p, 100, p, 4, p, None, p, T, T, 1, hkv, hkv, 64, 9, 16, 0.125, BF16, p, 0, None)
    import torch
    if not torch.cuda.is_available():   # (host memory stands in for tensors: nothing may run)
        for call in (append, prefix):
            assert call(1, 2, 3, 64) != -5 and call(3, 1, 64, 1) != -5 and call(1, 1, 7, 9) != -5
    for call in (append, prefix):
        assert call(2, 1, 100, 1) == -5 and call(1, 2, 128, 9) == -5


@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_lists_whose_rounded_length_passes_31_bits_are_refused(lib, p, page):
    """A list's keys are rounded up to whole tiles of 128 in 31 bits."""
    for width in ((2 ** 31 - 1) // page, (2 ** 31 - 128) // page):
        rest = (3, 3, 1, 4, 2, 64, 9, page, 0.125, BF16, p, 0, None)
        assert lib.wht_attn_prefix(p, 256, 64, p, p, p, 100, p, width, p, None, p, *rest) == -2
    assert lib.wht_attn_prefix(p, 256, 64, p, p, p, 2 ** 31 - 128, p, 4, p, None, p, *rest) == -3


@pytest.mark.parametrize("width,select,T,B,max_q,hkv,page", [
    (1500, 32, 32768, 1, 32768, 8, 16),     # a long prompt: 1.5 GB of scores that nobody would read
    (512, 32, 64, 64, 1, 8, 64),
    (64, 16, 1, 1, 1, 8, 64),
    (2048, 32, 64, 64, 1, 8, 16),
])
def test_scores_that_stay_in_shared_memory_need_no_workspace(plan, width, select, T, B, max_q, hkv, page):
    f = plan("select", width, select, T, B, max_q, 4 * hkv, hkv, 128, page, BF16)
    assert f["scores_bytes"] == 0
    parts = f["splits"] * T * 4 * hkv * (128 * 4 + 8) if f["splits"] > 1 else 0
    assert f["bytes"] <= parts + 256


@pytest.mark.parametrize("width,T,B,max_q", [(1024, 1, 1, 1), (2048, 4, 4, 1), (1600, 300, 1, 300), (49152, 200, 200, 1)])
def test_scores_of_the_two_kernels_do(plan, width, T, B, max_q):
    f = plan("select", width, 32, T, B, max_q, 32, 8, 128, 16, BF16)
    assert f["scores_bytes"] >= T * 8 * width * 4


def test_the_example_refuses_more_steps_than_it_has_pages_for():
    """(On the host: an index past the own pages would be a device assertion.)"""
    import sys
    for steps, own in ((513, 512), (0, 512), (1, 0)):
        proc = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "serving_step.py"), "--steps", str(steps), "--own", str(own)],
                              capture_output=True, text=True, env={**os.environ, "CUDA_VISIBLE_DEVICES": ""})
        assert proc.returncode == 2 and "--steps" in proc.stderr, proc.stderr
