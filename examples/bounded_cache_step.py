"""One attention block in serving with a bounded cache: 4-bit keys and values, eviction by received weight, head mixing.

    python examples/bounded_cache_step.py [--batch 32] [--budget 2048] [--slack 256] [--steps 512]

Every sequence decodes one token a step.  Keys and values are appended in 4 bits; the attention keeps the weight that each key
receives.  Once the sequences hold budget + slack keys, the heaviest `budget` of each (the first 4 and the last 256 always among them) move
into the other half of the pages, whose turn it then is.  Positions go on counting from what a sequence has seen.  Steps and evictions
are captured in CUDA graphs; the fused projection's outputs are random.
"""
import argparse
import os
import sys

import torch

if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2603_08343_b200 import attention as A
from paper_2603_08343_b200 import binding as B


def rope_tables(max_pos, rot, base=10000.0):
    """cos, sin [max_pos, rot/2] fp32."""
    angle = torch.arange(max_pos, dtype=torch.float64)[:, None] * base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    return angle.cos().float().cuda(), angle.sin().float().cuda()


class BoundedBlock:
    """A block whose sequences hold at most budget + slack keys each, in two sets of pages that take turns."""

    def __init__(self, batch, heads, kv_heads, head_dim, page, budget, slack, max_pos, keep_first=4, keep_last=256, a=None, b=None):
        if slack < 1 or keep_first + keep_last > budget:
            raise ValueError("a sequence needs room for a token, and a budget for what is always kept")
        self.batch, self.heads, self.kv_heads, self.head_dim, self.page = batch, heads, kv_heads, head_dim, page
        self.budget, self.most, self.keep_first, self.keep_last = budget, budget + slack, keep_first, keep_last
        width = -(-self.most // page)
        self.cache = A.cache4(2 * batch * width, kv_heads, page, head_dim)
        order = torch.randperm(2 * batch * width, device="cuda").to(torch.int32)   # pages come from a pool in any order
        self.tables = [t.contiguous() for t in order.reshape(2, batch, width)]
        self.lens = torch.zeros(batch, dtype=torch.int32, device="cuda")
        self.position = torch.zeros(batch, dtype=torch.int32, device="cuda")
        self.weights = torch.zeros(batch, kv_heads, width * page, device="cuda")
        self.cos, self.sin = rope_tables(max_pos, head_dim)
        self.a = torch.ones(heads * head_dim, device="cuda") if a is None else a
        self.b = torch.zeros(heads * head_dim, device="cuda") if b is None else b

    def step(self, qkv, half):
        """One token per sequence on pages `half`: qkv [batch, heads + 2 kv_heads, head_dim] -> [batch, heads * head_dim]."""
        q, k, v = qkv.split([self.heads, self.kv_heads, self.kv_heads], dim=1)
        place = self.lens.long()
        page = self.tables[half].gather(1, (place // self.page).clamp(max=self.tables[half].shape[1] - 1)[:, None])[:, 0].long()
        slots = torch.where(place < self.most, page * self.page + place % self.page, -1)     # (a token that finds no room is dropped)
        q = A.kv_append4(k, v, self.cache, slots, positions=self.position, cos=self.cos, sin=self.sin, q=q)
        self.lens += 1
        self.position += 1
        heads, _ = A.paged_attention4(q, self.cache, self.tables[half], self.lens, weights=self.weights, weights_out=self.weights)
        return B.forward(heads.flatten(1), self.a, self.b, decode=heads.shape[0] <= 256)

    def evict(self, half):
        """Moves what is kept from pages `half` to the others; returns which keys stayed [batch, kv_heads, budget]."""
        lens, kept, weights = A.kv_evict4(self.cache, self.tables[half], self.lens, self.weights, self.tables[1 - half], self.budget,
                                          keep_first=self.keep_first, keep_last=self.keep_last)
        self.lens.copy_(lens)
        self.weights.copy_(weights)
        return kept


def main():
    ap = argparse.ArgumentParser()
    for name, value in (("batch", 32), ("heads", 32), ("kv-heads", 8), ("head-dim", 128), ("page", 64), ("budget", 2048), ("slack", 256), ("steps", 4096)):
        ap.add_argument(f"--{name}", type=int, default=value)
    o = ap.parse_args()
    torch.manual_seed(0)
    block = BoundedBlock(o.batch, o.heads, o.kv_heads, o.head_dim, o.page, o.budget, o.slack, max_pos=o.steps, keep_last=min(256, o.budget // 2))
    qkv = torch.randn(o.batch, o.heads + 2 * o.kv_heads, o.head_dim, device="cuda").bfloat16()
    block.step(qkv, 0)                                                              # warm-up, before the captures
    block.evict(0)
    torch.cuda.synchronize()
    steps, evictions = [torch.cuda.CUDAGraph() for _ in range(2)], [torch.cuda.CUDAGraph() for _ in range(2)]
    for half in range(2):
        with torch.cuda.graph(steps[half]):
            y = block.step(qkv, half)
        with torch.cuda.graph(evictions[half]):
            block.evict(half)
    block.lens.zero_()
    block.position.zero_()
    block.weights.zero_()
    held, half, moved = 0, 0, 0
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    for _ in range(o.steps):
        if held == block.most:
            evictions[half].replay()
            held, half, moved = block.budget, 1 - half, moved + 1
        qkv.normal_()
        steps[half].replay()
        held += 1
    end.record()
    torch.cuda.synchronize()
    A.device_status()
    assert torch.isfinite(y).all() and int(block.lens.max()) == held
    print(f"{begin.elapsed_time(end) / o.steps * 1e3:.1f} us a step ({o.batch} sequences of up to {block.most} keys, {moved} evictions)")


if __name__ == "__main__":
    main()
