"""A key/value cache held in four bits and the attention over it (``include/moa_kv4.h``).

A cache is a uint8 tensor [num_pages, heads, page_bytes] (``kv4_cache``).  ``seq_lens`` int32 [B]
counts the tokens of every sequence, the call's new ones included; ``page_table`` int32
[B, max_pages] names the pages of each (None: sequence b has page b alone); ``new_lens`` int32 [B]
says how many of a call's N rows per sequence are real (None: all).  Row i of sequence b is token
``seq_lens[b] - new_lens[b] + i``.
"""
from __future__ import annotations

import functools
import math

import torch

from . import MOA_BF16, MOA_F32, _DTYPE_CODES
from ._call import check_list, check_rows, ci, done, f32, function, handle, i64, on, ptr, same_device, strides, sz, vp

moa_kv4_page_bytes = function("moa_kv4_page_bytes", [i64] * 2, sz)
_ROWS = [vp] * 6 + [i64] * 7 + [vp, vp, ci, vp]
moa_kv4_write = function("moa_kv4_write", _ROWS)
moa_kv4_read = function("moa_kv4_read", _ROWS)
_SPLIT = [i64] * 8 + [ci]
moa_kv4_attn_num_splits = function("moa_kv4_attn_num_splits", _SPLIT)
moa_kv4_attn_workspace_bytes = function("moa_kv4_attn_workspace_bytes", _SPLIT, sz)
moa_kv4_attn_fwd = function(
    "moa_kv4_attn_fwd", [vp] * 7 + [i64] * 9 + [vp, vp, f32, ci, ci, vp, sz, ci, vp])

_ws_bytes = functools.lru_cache(maxsize=1024)(moa_kv4_attn_workspace_bytes)


def kv4_cache(num_pages, heads, page, d, device="cuda"):
    """An empty cache of ``num_pages`` pages of ``page`` tokens (a multiple of 64) of ``heads``
    key/value heads of size d (64 or 128).  Its contents need not be set."""
    n = moa_kv4_page_bytes(page, d)
    if n == 0:
        raise ValueError("page must be a multiple of 64 up to 2^20, d 64 or 128")
    return torch.empty((num_pages, heads, n), dtype=torch.uint8, device=device)


def _place(cache, d, B, seq_lens, new_lens, page_table, device):
    """Checks the cache and the lists: (heads, page, num_pages, max_pages)."""
    if cache.dim() != 3 or cache.dtype != torch.uint8 or not cache.is_contiguous() or not cache.is_cuda:
        raise ValueError("cache must be a contiguous uint8 device tensor [num_pages, heads, page_bytes]")
    num_pages, heads, n = cache.shape
    page = n // (d + d // 16) if d in (64, 128) else 0
    if page == 0 or moa_kv4_page_bytes(page, d) != n:
        raise ValueError(f"cache: {n} bytes are no page of heads of size {d}")
    if cache.device != device:
        raise ValueError(f"tensors on {device} and on {cache.device} in one call")
    check_list("seq_lens", seq_lens, (B,), torch.int32, device)
    if new_lens is not None:
        check_list("new_lens", new_lens, (B,), torch.int32, device)
    if page_table is None:
        if num_pages < B:
            raise ValueError("a cache without a page table needs a page for every sequence")
        return heads, page, num_pages, 1
    max_pages = page_table.shape[-1] if page_table.dim() == 2 else -1
    check_list("page_table", page_table, (B, max_pages), torch.int32, device)
    return heads, page, num_pages, max_pages


def kv4_write(k, v, cache, seq_lens, page_table=None, new_lens=None, stream=None):
    """Quantises new keys and values k, v [B, heads, N, d] (bf16 or fp32, any views with contiguous
    heads) into ``cache``, in place.  Raises ``MoaAttnError`` on a rejected call."""
    check_rows("k", k)
    check_rows("v", v, k.shape)
    if k.dtype != v.dtype:
        raise TypeError("k and v must share one dtype")
    B, Hk, N, d = k.shape
    device = same_device(k, v)
    heads, page, num_pages, max_pages = _place(cache, d, B, seq_lens, new_lens, page_table, device)
    if Hk != heads:
        raise ValueError(f"k has {Hk} heads, the cache {heads}")
    with on(device):
        done(moa_kv4_write(k.data_ptr(), v.data_ptr(), cache.data_ptr(), seq_lens.data_ptr(), ptr(new_lens),
                           ptr(page_table), B, Hk, N, d, page, num_pages, max_pages, strides(k), strides(v),
                           _DTYPE_CODES[k.dtype], handle(stream, k)))


def kv4_read(cache, N, d, seq_lens, page_table=None, new_lens=None, out_dtype=None, k_out=None, v_out=None,
             stream=None):
    """The keys and values [B, heads, N, d] that ``cache`` holds for N rows per sequence, as
    ``out_dtype`` (default bf16; exact).  Rows behind ``new_lens`` are left as they are in ``k_out``
    and ``v_out`` (in new tensors: unset).  ``new_lens=seq_lens`` reads whole sequences."""
    B = seq_lens.shape[0] if seq_lens.dim() == 1 else -1
    device = cache.device
    heads, page, num_pages, max_pages = _place(cache, d, B, seq_lens, new_lens, page_table, device)
    dt = out_dtype or (k_out.dtype if k_out is not None else torch.bfloat16)
    if dt not in _DTYPE_CODES:
        raise TypeError(f"unsupported dtype {dt}; use torch.float32 or torch.bfloat16")
    outs = []
    for name, t in (("k_out", k_out), ("v_out", v_out)):
        if t is None:
            t = torch.empty((B, heads, N, d), dtype=dt, device=device)
        else:
            check_rows(name, t, (B, heads, N, d))
            if t.dtype != dt or t.device != device:
                raise ValueError(f"{name} must be of {dt} on {device}")
        outs.append(t)
    k, v = outs
    with on(device):
        done(moa_kv4_read(cache.data_ptr(), k.data_ptr(), v.data_ptr(), seq_lens.data_ptr(), ptr(new_lens),
                          ptr(page_table), B, heads, N, d, page, num_pages, max_pages, strides(k), strides(v),
                          _DTYPE_CODES[dt], handle(stream, cache)))
    return k, v


def kv4_attn_fwd(q, cache, seq_lens, page_table=None, new_lens=None, scale=None, causal=False, max_len=0,
                 out_dtype=None, return_lse=False, num_splits=0, out=None, workspace=None, stream=None):
    """Attention of new queries q [B, Hq, N, d] (bf16) over ``cache``, whose heads each serve
    Hq / heads successive query heads.  ``causal``: query i sees the tokens up to its own,
    ``seq_lens[b] - new_lens[b] + i``; otherwise all ``seq_lens[b]``.  A row that sees nothing gets
    O = 0 and LSE = -inf; rows behind ``new_lens`` are left as they are.  ``max_len``: the longest
    sequence, where the caller knows it (it guides the key splits only; 0: the table's capacity).
    ``scale`` defaults to 1/sqrt(d).  Returns O [B, Hq, N, d] (and LSE [B, Hq, N] fp32 when
    ``return_lse``).  Raises ``MoaAttnError`` on a rejected call."""
    check_rows("q", q)
    if q.dtype != torch.bfloat16:
        raise TypeError("q must be torch.bfloat16")
    B, Hq, N, d = q.shape
    device = q.device
    heads, page, num_pages, max_pages = _place(cache, d, B, seq_lens, new_lens, page_table, device)
    odt = torch.bfloat16 if out_dtype is None else out_dtype
    if odt not in _DTYPE_CODES:
        raise TypeError(f"unsupported dtype {odt}; use torch.float32 or torch.bfloat16")
    if out is None:
        out = torch.empty((B, Hq, N, d), dtype=odt, device=device)
    else:
        check_rows("out", out, q.shape)
        if out.dtype != odt or out.device != device:
            raise ValueError("out must be a [B, Hq, N, d] tensor of the output dtype")
    lse = torch.empty((B, Hq, N), dtype=torch.float32, device=device) if return_lse else None
    if scale is None:
        scale = 1.0 / math.sqrt(d)
    if workspace is None:
        n = _ws_bytes(B, Hq, heads, N, d, page, max_pages, max_len, num_splits)
        if n:
            workspace = torch.empty(n, dtype=torch.uint8, device=device)
    else:
        same_device(q, workspace)
    ws_n = 0 if workspace is None else workspace.numel() * workspace.element_size()
    with on(device):
        done(moa_kv4_attn_fwd(q.data_ptr(), cache.data_ptr(), out.data_ptr(), ptr(lse), seq_lens.data_ptr(),
                              ptr(new_lens), ptr(page_table), B, Hq, heads, N, d, page, num_pages, max_pages,
                              max_len, strides(q), strides(out), float(scale), int(causal),
                              MOA_F32 if odt == torch.float32 else MOA_BF16, ptr(workspace), ws_n, num_splits,
                              handle(stream, q)))
    return (out, lse) if return_lse else out
