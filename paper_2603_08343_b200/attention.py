"""Serving attention in front of the head mixing: a paged cache, what writes it and two ways to read it.

    from paper_2603_08343_b200 import attention as A, binding as B

    q = A.kv_append(k, v, k_cache, v_cache, slots, positions=pos, cos=cos, sin=sin, q=q)     # rotate, write the cache
    heads = A.shared_prefix_attention(q, k_cache, v_cache, prefix_pages, prefix_len, page_table, kv_lens)
    y = B.forward(heads.flatten(1), a, b, decode=True)                                       # head mixing

    # long contexts: only the pages that a score over their summaries selects for each query
    heads, pages = A.selected_page_attention(q, k_cache, v_cache, summary, page_table, kv_lens, select=32)

Caches are [num_pages, kv_heads, page, head_dim] (page 16, 32, 64 or 128; head_dim 64, 96 or 128), queries
[tokens, heads, head_dim]; all tensors of a call are bf16 or all are fp32.  Query, key and value tensors may be slices of a
fused projection.  Argument checks and marshalling only: the work is the library's (include/wht_attention.h).
The calls run on the current stream of the tensors' device, or on `stream`; they do not synchronise.  Page
numbers, slots and lengths are checked on the device: device_status() reports what was out of range.  There is no backward:
tensors that require a gradient are refused unless gradients are off.
"""
from __future__ import annotations

import importlib.util
import os

import torch

from . import binding as _B

PAGE_SIZES = (16, 32, 64, 128)
HEAD_DIMS = (64, 96, 128)


def _load():
    """The CPython module that checks the arguments and calls the library (csrc/attn_python.cpp)."""
    path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "_attention.so")
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build it with `python -m paper_2603_08343_b200.build` (there is no CPU fallback)")
    spec = importlib.util.spec_from_file_location("_attention", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    module.raise_with(_B._check)
    return module


_native = _load()


def _raw(stream):
    if stream is None:
        return None
    if stream.device_index != torch.cuda.current_device():
        raise ValueError(f"the stream is on device {stream.device_index}, the call on the current one, {torch.cuda.current_device()}")
    # outputs and scratch come from the current stream's pool, which may hand out memory that stream still uses
    stream.wait_stream(torch.cuda.current_stream())
    return stream.cuda_stream


def kv_append(k, v, k_cache, v_cache, slots, positions=None, cos=None, sin=None, q=None, q_out=None, summary=None,
              summary_scale=None, interleaved: bool = False, stream=None):
    """Writes new keys and values into the paged cache, rotating queries and keys by their positions; returns the
    rotated queries (`q_out`, allocated if None; may be q itself) or None without q.

    k, v [tokens, kv_heads, head_dim], q [tokens, heads, head_dim]; slots [tokens] int64 (page * page_size + place, negative
    for padding); positions [tokens] int32 and cos, sin [max_pos, rot/2] fp32, or all three None for no rotation.  Pairs are
    (i, i + rot/2), or (2i, 2i + 1) with `interleaved`.  summary [num_pages, kv_heads, 2, head_dim] int8 with
    summary_scale [kv_heads] fp32 keeps each page's least and largest clamp(rint(key * scale), -127, 127) per channel; it
    needs a page's tokens next to each other, in the order of their slots.
    """
    return _native.kv_append(k, v, k_cache, v_cache, slots, positions, cos, sin, q, q_out, summary, summary_scale, interleaved, _raw(stream))


def shared_prefix_attention(q, k_cache, v_cache, prefix_pages, prefix_len: int, page_table, kv_lens, q_start=None, max_q_len: int = 1,
                            scale: float | None = None, out=None, stream=None):
    """Attention of a batch behind one shared prefix: each token sees the `prefix_len` keys of `prefix_pages` and its
    sequence's own keys up to itself.  Returns [tokens, heads, head_dim].

    page_table [batch, pages] int32 and kv_lens [batch] int32: the sequences' own pages and how many keys they hold, this
    call's tokens included (the work is divided by the table's width: one about as wide as the longest sequence is fastest).
    q_start [batch + 1] int32: sequence b's tokens are q_start[b]..q_start[b+1]-1, at most max_q_len; None = one token per
    sequence.  prefix_len = 0 gives plain attention over the own pages.  scale: 1/sqrt(head_dim).
    """
    return _native.shared_prefix_attention(q, k_cache, v_cache, prefix_pages, prefix_len, page_table, kv_lens, q_start, max_q_len, scale,
                                           out, _raw(stream))


def selected_page_attention(q, k_cache, v_cache, summary, page_table, kv_lens, select: int, q_start=None, max_q_len: int = 1,
                            scale: float | None = None, out=None, pages_out=None, stream=None):
    """Attention of each query to its own page and to the `select` - 1 earlier pages of its sequence that score highest
    by their summaries (the summary that kv_append keeps).  Returns (out [tokens, heads, head_dim], pages [tokens, kv_heads,
    select] int32: the pages read, ascending, then -1).  Tables of up to 49152 pages; the other arguments are those of
    shared_prefix_attention."""
    return _native.selected_page_attention(q, k_cache, v_cache, summary, page_table, kv_lens, select, q_start, max_q_len, scale, out,
                                           pages_out, _raw(stream))


def device_status() -> None:
    """Synchronises with the device, all streams, and raises WhtError if a kernel met an index out of range (a token that no
    sequence covers included) since the last query."""
    _B._check(_B.lib().wht_attn_device_status(), "wht_attn_device_status")
