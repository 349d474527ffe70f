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
numbers, slots and lengths are checked on the device: device_status() reports what was out of range.
"""
from __future__ import annotations

import functools

import torch

from . import binding as _B
from .workloads import WHT_BF16, WHT_F32

_lib = _B.lib()
_CODES = {torch.bfloat16: WHT_BF16, torch.float32: WHT_F32}
_raw_stream = torch._C._cuda_getCurrentRawStream

PAGE_SIZES = (16, 32, 64, 128)
HEAD_DIMS = (64, 96, 128)


def _fail(what: str):
    raise ValueError(what)


def _caches(k_cache, v_cache):
    """(dtype code, device index, num_pages, kv_heads, page, head_dim) of a pair of caches."""
    shape = k_cache.shape
    if len(shape) != 4 or v_cache.shape != shape:
        _fail("k_cache and v_cache must be [num_pages, kv_heads, page, head_dim] and of one shape")
    code = _CODES.get(k_cache.dtype)
    if code is None or v_cache.dtype is not k_cache.dtype:
        _fail(f"unsupported storage types k_cache={k_cache.dtype}, v_cache={v_cache.dtype}: both bf16 or both fp32")
    if not (k_cache.is_cuda and k_cache.is_contiguous() and v_cache.is_contiguous()):
        _fail("caches must be contiguous tensors on a CUDA device")
    device = k_cache.get_device()
    if v_cache.get_device() != device or device != torch.cuda.current_device():
        _fail("all tensors must live on the current CUDA device")
    if shape[2] not in PAGE_SIZES or shape[3] not in HEAD_DIMS:
        _fail(f"page must be one of {PAGE_SIZES} and head_dim one of {HEAD_DIMS}, got {shape[2]} and {shape[3]}")
    return code, device, *shape


def _rows(t, name, heads, dim, dtype, device, tokens=None):
    """Checks a [tokens, heads, head_dim] tensor (strides allowed, channels contiguous); its token and head strides."""
    if t.dim() != 3 or t.shape[2] != dim or (heads is not None and t.shape[1] != heads) or (tokens is not None and t.shape[0] != tokens):
        _fail(f"{name} must be [{'tokens' if tokens is None else tokens}, {'heads' if heads is None else heads}, {dim}], got {tuple(t.shape)}")
    if t.dtype is not dtype or t.get_device() != device:
        _fail(f"{name} must be a {dtype} tensor on the caches' device")
    st, sh, sd = t.stride()
    if sd != 1:
        _fail(f"{name} must have contiguous channels")
    return st, sh


def _vector(t, name, dtype, device, shape):
    if t.dtype is not dtype or t.get_device() != device or t.shape != shape or not t.is_contiguous():
        _fail(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on the caches' device")
    return t.data_ptr()


def _batch(q, page_table, kv_lens, q_start, max_q_len, device):
    if page_table.dim() != 2:
        _fail("page_table must be [batch, pages]")
    batch, width = page_table.shape
    table = _vector(page_table, "page_table", torch.int32, device, (batch, width))
    lens = _vector(kv_lens, "kv_lens", torch.int32, device, (batch,))
    if q_start is None:
        if q.shape[0] != batch or max_q_len != 1:
            _fail(f"without q_start every sequence has one token: got {q.shape[0]} tokens for {batch} sequences, max_q_len {max_q_len}")
        return batch, width, table, lens, None
    return batch, width, table, lens, _vector(q_start, "q_start", torch.int32, device, (batch + 1,))


def _outputs(stream, device, *made):
    """The raw stream of the call; tensors made on the current stream are marked as in use on another one."""
    current = _raw_stream(device)
    if stream is None or stream.cuda_stream == current:
        return current
    stream.wait_stream(torch.cuda.current_stream())  # the allocator may hand out memory that the current stream still uses
    for t in made:
        if t is not None:
            t.record_stream(stream)
    return stream.cuda_stream


@functools.lru_cache(maxsize=4096)
def _workspace_bytes(name: str, device: int, *args) -> int:
    return int(getattr(_lib, name)(*args))


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
    code, device, pages, hkv, page, dim = _caches(k_cache, v_cache)
    dtype = k_cache.dtype
    tokens = k.shape[0]
    k_st, k_sh = _rows(k, "k", hkv, dim, dtype, device)
    v_st, v_sh = _rows(v, "v", hkv, dim, dtype, device, tokens)
    slots_p = _vector(slots, "slots", torch.int64, device, (tokens,))
    rot = max_pos = 0
    pos_p = cos_p = sin_p = q_p = out_p = sum_p = scale_p = None
    if positions is not None or cos is not None or sin is not None:
        if positions is None or cos is None or sin is None or cos.dim() != 2:
            _fail("positions, cos and sin [max_pos, rot/2] come together")
        max_pos, half = cos.shape
        rot = 2 * half
        if rot % 16 or rot > dim or max_pos < 1:
            _fail(f"rot = {rot} must be a multiple of 16 up to head_dim, with at least one position")
        cos_p = _vector(cos, "cos", torch.float32, device, (max_pos, half))
        sin_p = _vector(sin, "sin", torch.float32, device, (max_pos, half))
        pos_p = _vector(positions, "positions", torch.int32, device, (tokens,))
    made = None
    hq, q_st, q_sh = hkv, 0, 0
    if q is not None:
        q_st, q_sh = _rows(q, "q", None, dim, dtype, device, tokens)
        hq = q.shape[1]
        if q_out is None:
            q_out = made = torch.empty((tokens, hq, dim), dtype=dtype, device=q.device)
        elif q_out.shape != q.shape or q_out.dtype is not dtype or q_out.get_device() != device or not q_out.is_contiguous():
            _fail("q_out must be contiguous and match q")
        q_p, out_p = q.data_ptr(), q_out.data_ptr()
    elif q_out is not None:
        _fail("q_out without q")
    if summary is not None:
        if summary_scale is None:
            _fail("summary needs summary_scale")
        sum_p = _vector(summary, "summary", torch.int8, device, (pages, hkv, 2, dim))
        scale_p = _vector(summary_scale, "summary_scale", torch.float32, device, (hkv,))
    rc = _lib.wht_kv_append(k.data_ptr(), k_st, k_sh, v.data_ptr(), v_st, v_sh, q_p, q_st, q_sh, out_p, slots_p, pos_p, cos_p, sin_p,
                            k_cache.data_ptr(), v_cache.data_ptr(), sum_p, scale_p, tokens, hq, hkv, dim, rot, int(interleaved),
                            max_pos, pages, page, code, _outputs(stream, device, made))
    if rc:
        raise _B.WhtError(rc, "wht_kv_append")
    return q_out


def _attention_out(q, out, device):
    if out is None:
        return torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if out.shape != q.shape or out.dtype is not q.dtype or out.get_device() != device or not out.is_contiguous():
        _fail("out must be contiguous and match q")
    return out


def _scratch(name, device, q, *args):
    need = _workspace_bytes(name, device, *args)
    return (None, 0) if need == 0 else (torch.empty(need, dtype=torch.uint8, device=q.device), need)


def shared_prefix_attention(q, k_cache, v_cache, prefix_pages, prefix_len: int, page_table, kv_lens, q_start=None, max_q_len: int = 1,
                            scale: float | None = None, out=None, stream=None):
    """Attention of a batch behind one shared prefix: each token sees the `prefix_len` keys of `prefix_pages` and its
    sequence's own keys up to itself.  Returns [tokens, heads, head_dim].

    page_table [batch, pages] int32 and kv_lens [batch] int32: the sequences' own pages and how many keys they hold, this
    call's tokens included.  q_start [batch + 1] int32: sequence b's tokens are q_start[b]..q_start[b+1]-1, at most
    max_q_len; None = one token per sequence.  prefix_len = 0 gives plain attention over the own pages.  scale: 1/sqrt(head_dim).
    """
    code, device, pages, hkv, page, dim = _caches(k_cache, v_cache)
    q_st, q_sh = _rows(q, "q", None, dim, k_cache.dtype, device)
    tokens, hq, _ = q.shape
    batch, width, table_p, lens_p, start_p = _batch(q, page_table, kv_lens, q_start, max_q_len, device)
    if prefix_len < 0:
        _fail("prefix_len must be >= 0")
    prefix_p = None
    if prefix_len:
        if prefix_pages.shape[0] * page < prefix_len:
            _fail(f"{prefix_pages.shape[0]} prefix pages do not hold {prefix_len} keys")
        prefix_p = _vector(prefix_pages, "prefix_pages", torch.int32, device, prefix_pages.shape)
    given = out
    out = _attention_out(q, out, device)
    work, need = _scratch("wht_attn_prefix_workspace_bytes", device, q, prefix_len, width, tokens, batch, max_q_len, hq, hkv, dim, page, code)
    rc = _lib.wht_attn_prefix(q.data_ptr(), q_st, q_sh, k_cache.data_ptr(), v_cache.data_ptr(), prefix_p, prefix_len, table_p, width,
                              lens_p, start_p, out.data_ptr(), tokens, batch, max_q_len, hq, hkv, dim, pages, page,
                              dim ** -0.5 if scale is None else scale, code, None if work is None else work.data_ptr(), need,
                              _outputs(stream, device, work, None if given is not None else out))
    if rc:
        raise _B.WhtError(rc, "wht_attn_prefix")
    return out


def selected_page_attention(q, k_cache, v_cache, summary, page_table, kv_lens, select: int, q_start=None, max_q_len: int = 1,
                            scale: float | None = None, out=None, pages_out=None, stream=None):
    """Attention of each query to its own page and to the `select` - 1 earlier pages of its sequence that score highest
    by their summaries (the summary that kv_append keeps).  Returns (out [tokens, heads, head_dim], pages [tokens, kv_heads,
    select] int32: the pages read, ascending, then -1).  The other arguments are those of shared_prefix_attention."""
    code, device, pages, hkv, page, dim = _caches(k_cache, v_cache)
    q_st, q_sh = _rows(q, "q", None, dim, k_cache.dtype, device)
    tokens, hq, _ = q.shape
    batch, width, table_p, lens_p, start_p = _batch(q, page_table, kv_lens, q_start, max_q_len, device)
    sum_p = _vector(summary, "summary", torch.int8, device, (pages, hkv, 2, dim))
    if select < 1:
        _fail("select must be >= 1")
    given, given_pages = out, pages_out
    out = _attention_out(q, out, device)
    if pages_out is None:
        pages_out = torch.empty((tokens, hkv, select), dtype=torch.int32, device=q.device)
    pages_p = _vector(pages_out, "pages_out", torch.int32, device, (tokens, hkv, select))
    work, need = _scratch("wht_attn_select_workspace_bytes", device, q, width, select, tokens, batch, max_q_len, hq, hkv, dim, page, code)
    rc = _lib.wht_attn_select(q.data_ptr(), q_st, q_sh, k_cache.data_ptr(), v_cache.data_ptr(), sum_p, table_p, width, lens_p, start_p,
                              select, out.data_ptr(), pages_p, tokens, batch, max_q_len, hq, hkv, dim, pages, page,
                              dim ** -0.5 if scale is None else scale, code, None if work is None else work.data_ptr(), need,
                              _outputs(stream, device, work, None if given is not None else out,
                                       None if given_pages is not None else pages_out))
    if rc:
        raise _B.WhtError(rc, "wht_attn_select")
    return out, pages_out


def device_status() -> None:
    """Synchronises and raises WhtError if a kernel met an index out of range since the last query."""
    rc = _lib.wht_attn_device_status()
    if rc:
        raise _B.WhtError(rc, "wht_attn_device_status")
