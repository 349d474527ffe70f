"""The bounded-cache example (4-bit append, attention with received weight, eviction, head mixing) against a plain statement of the whole block."""
import importlib.util
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import attention_ref as R
import cache4_ref as C
import oracle

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PATH = os.path.join(ROOT, "examples", "bounded_cache_step.py")


@pytest.mark.parametrize("batch,heads,kv_heads,head_dim,page,budget,slack", [(2, 8, 2, 64, 16, 20, 9), (3, 4, 4, 128, 32, 33, 40)])
def test_steps_of_a_block(batch, heads, kv_heads, head_dim, page, budget, slack):
    spec = importlib.util.spec_from_file_location("bounded_cache_step", PATH)
    E = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(E)
    g = torch.Generator()
    g.manual_seed(budget)
    width = heads * head_dim
    a, b = torch.randn(width, generator=g), torch.randn(width, generator=g)
    block = E.BoundedBlock(batch, heads, kv_heads, head_dim, page, budget, slack, 200, keep_first=2, keep_last=5, a=a.cuda(), b=b.cuda())
    cos, sin = block.cos.cpu(), block.sin.cpu()
    keys = [torch.zeros(0, kv_heads, head_dim) for _ in range(batch)]
    values = [torch.zeros(0, kv_heads, head_dim) for _ in range(batch)]
    half, held = 0, 0
    for step in range(budget + 2 * slack + 3):
        if held == block.most:
            kept = block.evict(half).cpu().long()          # (exactness of the choice: test_cache4_gpu.py)
            assert kept.shape == (batch, kv_heads, budget) and (kept >= 0).all() and (kept.diff(dim=-1) > 0).all()
            for s in range(batch):
                keys[s], values[s] = (torch.stack([x[s][kept[s, h], h] for h in range(kv_heads)], 1) for x in (keys, values))
            half, held = 1 - half, budget
        qkv = torch.randn(batch, heads + 2 * kv_heads, head_dim, generator=g).bfloat16()
        y = block.step(qkv.cuda(), half).cpu()
        held += 1
        q, k, v = qkv.split([heads, kv_heads, kv_heads], 1)
        at = torch.full((batch,), step).int()
        q = R.rotate32(q, at, cos, sin, False)
        k, v = C.hold(C.rotated(k, at, cos, sin, False)), C.hold(v.float())
        for s in range(batch):
            keys[s], values[s] = torch.cat([keys[s], k[s:s + 1]]), torch.cat([values[s], v[s:s + 1]])
        want, _ = C.attention(q, keys, values, [held] * batch, None, head_dim ** -0.5)
        mixed = oracle.wht_affine_fwd(want.reshape(batch, -1).numpy(), a.double().numpy(), b.double().numpy())
        spread = max((x.amax(-1) - x.amin(-1)).max().item() for x in keys)
        vmax = max(x.abs().max().item() for x in values)
        # heads within their tolerance; the mixing adds `width` of them with signs, over sqrt(width), times |a|, and rounds once more
        slack_y = C.tolerance(q, spread, vmax, head_dim ** -0.5) * width ** 0.5 * a.abs().numpy() + 2 ** -8 * np.abs(mixed)
        assert np.all(np.abs(y.double().numpy() - mixed) <= slack_y)
    assert block.lens.tolist() == [held] * batch and half == 0        # evicted twice
    E.A.device_status()


def test_the_example_runs():
    proc = subprocess.run([sys.executable, PATH, "--batch", "4", "--budget", "96", "--slack", "40", "--steps", "200"], capture_output=True, text=True, timeout=300)
    assert proc.returncode == 0, proc.stderr
    assert "2 evictions" in proc.stdout
