"""The serving example (append, both ways to attend, head mixing) against a plain 64-bit statement of the whole block."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import attention_ref as R
import oracle

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def E():
    from paper_2603_08343_b200 import build
    build.build()
    spec = importlib.util.spec_from_file_location("serving_step", os.path.join(ROOT, "examples", "serving_step.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("select", [0, 3])
@pytest.mark.parametrize("batch,heads,kv_heads,head_dim,page,prefix", [(3, 8, 2, 64, 16, 48), (40, 4, 4, 128, 32, 256)])
def test_steps_of_a_block(E, batch, heads, kv_heads, head_dim, page, prefix, select):
    g = torch.Generator()
    g.manual_seed(batch)
    width = heads * head_dim
    a, b = torch.randn(width, generator=g), torch.randn(width, generator=g)
    steps, own = 5, 40
    block = E.Block(batch, heads, kv_heads, head_dim, page, prefix, own, a=a.cuda(), b=b.cuda())
    rows = heads + 2 * kv_heads
    document = torch.randn(prefix, rows, head_dim, generator=g).bfloat16()
    first = block.write_prefix(document.cuda())
    outs, tokens = [], []
    for _ in range(steps):
        tokens.append(torch.randn(batch, rows, head_dim, generator=g).bfloat16())
        outs.append(block.step(tokens[-1].cuda(), select).cpu())
    torch.cuda.synchronize()
    E.A.device_status()

    # the same in 64 bits, sequence by sequence, from the stored values of the definition
    cos, sin = block.cos.cpu(), block.sin.cpu()
    scale8 = block.summary_scale.cpu()

    def mixed(h):  # [n, heads, head_dim] fp64
        return oracle.wht_affine_fwd(h.reshape(h.shape[0], -1).numpy(), a.double().numpy(), b.double().numpy())

    def turned(x, positions):
        return R.rotate32(x, positions, cos, sin, False)

    def close(got, want, vmax):
        # heads within their tolerance and rounded to bf16 (2^-8 of vmax); the mixing adds `width` of them with signs, over sqrt(width),
        # times |a|, and rounds once more
        slack = (R.tolerance(torch.bfloat16, vmax) + vmax * 2 ** -8) * width ** 0.5 * a.abs().numpy() + 2 ** -8 * np.abs(want)
        assert np.all(np.abs(got.double().numpy() - want) <= slack)

    q, k, v = document.split([heads, kv_heads, kv_heads], dim=1)
    place = torch.arange(prefix)
    q, doc_k = turned(q, place), turned(k, place)
    G = heads // kv_heads
    want = torch.stack([torch.cat([R.attend(q[t, h * G:(h + 1) * G], doc_k[:t + 1, h], v[:t + 1, h], head_dim ** -0.5) for h in range(kv_heads)])
                        for t in range(prefix)])
    close(first.cpu(), mixed(want), v.abs().max().item())

    doc_v, vmax = v, max(t.abs().max().item() for t in tokens + [document])
    ks, vs = [doc_k.clone() for _ in range(batch)], [doc_v.clone() for _ in range(batch)]
    for i in range(steps):
        q, k, v = tokens[i].split([heads, kv_heads, kv_heads], dim=1)
        at = torch.full((batch,), prefix + i)
        q, k = turned(q, at), turned(k, at)
        want = torch.zeros(batch, heads, head_dim, dtype=torch.float64)
        for s in range(batch):
            ks[s], vs[s] = torch.cat([ks[s], k[s:s + 1]]), torch.cat([vs[s], v[s:s + 1]])
            n = prefix + i + 1
            for h in range(kv_heads):
                keys = torch.arange(n)
                if select:
                    c = (ks[s][:, h].float() * scale8[h]).round().clamp(-127, 127).long()
                    q8 = R.whole_queries(q[s, h * G:(h + 1) * G])
                    scores = []
                    for p in range((n - 1) // page):
                        lo, hi = c[p * page:(p + 1) * page].min(0).values, c[p * page:(p + 1) * page].max(0).values
                        scores.append(int(torch.maximum(q8 * lo, q8 * hi).sum()))
                    best = sorted(range(len(scores)), key=lambda p: (-scores[p], p))[:select - 1]
                    keys = torch.cat([torch.arange(p * page, min(n, (p + 1) * page)) for p in sorted(best) + [(n - 1) // page]])
                want[s, h * G:(h + 1) * G] = R.attend(q[s, h * G:(h + 1) * G], ks[s][keys, h], vs[s][keys, h], head_dim ** -0.5)
        close(outs[i], mixed(want), vmax)
