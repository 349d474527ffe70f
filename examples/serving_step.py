"""One attention block in serving: paged cache, shared prefix, selected pages, head mixing.

    python examples/serving_step.py [--batch 64] [--prefix 8192] [--own 512] [--steps 32] [--select 32]

A document of `prefix` tokens is written into the cache once.  A batch of sequences then answers questions about it:
each decode step rotates and appends the new tokens' keys and values, attends (to the shared prefix and the sequence's own
pages, or to the pages that the summaries select) and mixes the heads.  The step is captured in a CUDA graph; the fused
projection's outputs are random.
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


class Block:
    """The cache of one attention block and its parameters a, b; `prefix` tokens (whole pages) that all sequences share."""

    def __init__(self, batch, heads, kv_heads, head_dim, page, prefix, own, dtype=torch.bfloat16, summary_scale=28.0, a=None, b=None):
        if prefix % page:
            raise ValueError("the shared prefix takes whole pages")
        if own < 1:
            raise ValueError("a sequence needs room for one token of its own at least")
        self.batch, self.heads, self.kv_heads, self.head_dim, self.page, self.prefix = batch, heads, kv_heads, head_dim, page, prefix
        n_prefix, n_own = prefix // page, -(-own // page)
        pages = n_prefix + batch * n_own
        self.k_cache = torch.zeros(pages, kv_heads, page, head_dim, dtype=dtype, device="cuda")
        self.v_cache = torch.zeros_like(self.k_cache)
        self.summary = torch.zeros(pages, kv_heads, 2, head_dim, dtype=torch.int8, device="cuda")
        self.summary_scale = torch.full((kv_heads,), summary_scale, device="cuda")
        order = torch.randperm(pages, device="cuda").to(torch.int32)      # pages come from a pool in any order
        self.prefix_pages = order[:n_prefix].contiguous()
        self.own_pages = order[n_prefix:].reshape(batch, n_own).contiguous()
        self.all_pages = torch.cat([self.prefix_pages.expand(batch, -1), self.own_pages], 1).contiguous()
        self.own_lens = torch.zeros(batch, dtype=torch.int32, device="cuda")
        self.capacity = n_own * page                                       # tokens of its own that a sequence has room for
        self.cos, self.sin = rope_tables(prefix + self.capacity, head_dim)
        self.a = torch.ones(heads * head_dim, device="cuda") if a is None else a
        self.b = torch.zeros(heads * head_dim, device="cuda") if b is None else b

    def _append(self, qkv, slots, positions):
        q, k, v = qkv.split([self.heads, self.kv_heads, self.kv_heads], dim=1)
        return A.kv_append(k, v, self.k_cache, self.v_cache, slots, positions=positions, cos=self.cos, sin=self.sin, q=q,
                           summary=self.summary, summary_scale=self.summary_scale)

    def _mix(self, heads):
        return B.forward(heads.flatten(1), self.a, self.b, decode=heads.shape[0] <= 256)

    def write_prefix(self, qkv):
        """The shared document, once: qkv [prefix, heads + 2 kv_heads, head_dim]; returns its tokens' block outputs."""
        n = qkv.shape[0]
        if n != self.prefix:
            raise ValueError(f"{n} tokens for a document of {self.prefix}")
        place = torch.arange(n, device="cuda")
        slots = self.prefix_pages.long()[place // self.page] * self.page + place % self.page
        q = self._append(qkv, slots, place.int())
        starts = torch.tensor([0, n], dtype=torch.int32, device="cuda")
        lens = torch.tensor([n], dtype=torch.int32, device="cuda")
        return self._mix(A.shared_prefix_attention(q, self.k_cache, self.v_cache, None, 0, self.prefix_pages[None], lens, q_start=starts, max_q_len=n))

    def step(self, qkv, select=0):
        """One token per sequence: qkv [batch, heads + 2 kv_heads, head_dim] -> [batch, heads * head_dim].  select: 0 reads all keys,
        the shared ones once for the whole batch; otherwise each token reads that many pages.  A token that finds its sequence's pages
        full is dropped, and the attention reports the length (`device_status`)."""
        if qkv.shape[0] != self.batch:
            raise ValueError(f"{qkv.shape[0]} tokens for {self.batch} sequences")
        place = self.own_lens.long()
        page = self.own_pages.gather(1, (place // self.page).clamp(max=self.own_pages.shape[1] - 1)[:, None])[:, 0].long()
        slots = torch.where(place < self.capacity, page * self.page + place % self.page, -1)
        q = self._append(qkv, slots, self.own_lens + self.prefix)
        self.own_lens += 1
        if select:
            heads, _ = A.selected_page_attention(q, self.k_cache, self.v_cache, self.summary, self.all_pages, self.own_lens + self.prefix, select)
        else:
            heads = A.shared_prefix_attention(q, self.k_cache, self.v_cache, self.prefix_pages, self.prefix, self.own_pages, self.own_lens)
        return self._mix(heads)


def main():
    ap = argparse.ArgumentParser()
    for name, value in (("batch", 64), ("heads", 32), ("kv-heads", 8), ("head-dim", 128), ("page", 64), ("prefix", 8192), ("own", 512),
                        ("steps", 32), ("select", 32)):
        ap.add_argument(f"--{name}", type=int, default=value)
    o = ap.parse_args()
    if not 1 <= o.steps <= o.own:
        ap.error(f"--steps {o.steps}: the sequences have room for 1 to --own {o.own} tokens")
    torch.manual_seed(0)
    rows = o.heads + 2 * o.kv_heads
    block = Block(o.batch, o.heads, o.kv_heads, o.head_dim, o.page, o.prefix, o.own)
    block.write_prefix(torch.randn(o.prefix, rows, o.head_dim, device="cuda").bfloat16())
    qkv = torch.randn(o.batch, rows, o.head_dim, device="cuda").bfloat16()
    for select in (0, o.select):
        block.own_lens.zero_()
        block.step(qkv, select)                                           # warm-up, before the capture
        block.own_lens.zero_()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = block.step(qkv, select)
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        for _ in range(o.steps):
            qkv.normal_()
            graph.replay()
        end.record()
        torch.cuda.synchronize()
        A.device_status()
        assert torch.isfinite(y).all()
        what = f"{select} selected pages" if select else "shared prefix"
        print(f"{what}: {begin.elapsed_time(end) / o.steps * 1e3:.1f} us a step ({o.batch} sequences, {o.prefix} + up to {o.steps} keys)")


if __name__ == "__main__":
    main()
