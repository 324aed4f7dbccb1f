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

from . import MOA_BF16, MOA_F32, _DTYPE_CODES, _stream_handle, _torch as torch
from ._call import (Function, Packed, check_list, check_rows, ci, f32, i64, is_list, new_like, on_stream, run, sz, vp,
                    workspace as _workspace)

moa_kv4_page_bytes = Function("moa_kv4_page_bytes", [i64] * 2, sz)
_ROWS = [vp] * 6 + [i64] * 7 + [vp, vp, ci, vp]
moa_kv4_write = Function("moa_kv4_write", _ROWS)
moa_kv4_read = Function("moa_kv4_read", _ROWS)
_SPLIT = [i64] * 8 + [ci]
moa_kv4_attn_num_splits = Function("moa_kv4_attn_num_splits", _SPLIT)
moa_kv4_attn_workspace_bytes = Function("moa_kv4_attn_workspace_bytes", _SPLIT, sz)
moa_kv4_attn_fwd = Function(
    "moa_kv4_attn_fwd", [vp] * 7 + [i64] * 9 + [vp, vp, f32, ci, ci, vp, sz, ci, vp])

_write = Packed("moa_packed_kv4_write", "6q 7q 8q 2q")
_read = Packed("moa_packed_kv4_read", "6q 7q 8q 2q")
_attn = Packed("moa_packed_kv4_attn_fwd", "7q 9q 8q d 2q 4q")
_ws_bytes = functools.lru_cache(maxsize=1024)(moa_kv4_attn_workspace_bytes)
if torch is not None:   # the C functions above need none
    _int32, _uint8, _bf16 = torch.int32, torch.uint8, torch.bfloat16


@functools.lru_cache(maxsize=256)
def _page_of(n, d):
    """Tokens of a page of n bytes of a head of size d."""
    page = n // (d + d // 16) if d in (64, 128) else 0
    if page == 0 or moa_kv4_page_bytes(page, d) != n:
        raise ValueError(f"cache: {n} bytes are no page of heads of size {d}")
    return page


def kv4_cache(num_pages, heads, page, d, device="cuda"):
    """An empty cache of ``num_pages`` pages of ``page`` tokens (a multiple of 64) of ``heads``
    key/value heads of size d (64 or 128).  Its contents need not be set."""
    n = moa_kv4_page_bytes(page, d)
    if n == 0:
        raise ValueError("page must be a multiple of 64 up to 2^20, d 64 or 128")
    return torch.empty((num_pages, heads, n), dtype=torch.uint8, device=device)


def _place(cache, d, B, seq_lens, new_lens, page_table, device):
    """Checks the cache and the lists.  (heads, page, num_pages, max_pages, addresses of the cache,
    seq_lens, new_lens and page_table)."""
    n = cache.shape
    if len(n) != 3 or cache.dtype is not _uint8 or not cache.is_contiguous() or cache.get_device() != device:
        raise ValueError("cache must be a contiguous uint8 tensor [num_pages, heads, page_bytes] on the other tensors' device")
    num_pages, heads, size = n
    page = _page_of(size, d)
    if not is_list(seq_lens, (B,), _int32, device):
        check_list("seq_lens", seq_lens, (B,), _int32, device)
    new = table = 0
    if new_lens is not None:
        check_list("new_lens", new_lens, (B,), _int32, device)
        new = new_lens.data_ptr()
    max_pages = 1
    if page_table is not None:
        max_pages = page_table.shape[-1] if page_table.dim() == 2 else -1
        if not is_list(page_table, (B, max_pages), _int32, device):
            check_list("page_table", page_table, (B, max_pages), _int32, device)
        table = page_table.data_ptr()
    elif num_pages < B:
        raise ValueError("a cache without a page table needs a page for every sequence")
    return heads, page, num_pages, max_pages, cache.data_ptr(), seq_lens.data_ptr(), new, table


def kv4_write(k, v, cache, seq_lens, page_table=None, new_lens=None, stream=None):
    """Quantises new keys and values k, v [B, heads, N, d] (bf16 or fp32, any views with contiguous
    heads) into ``cache``, in place.  Raises ``MoaAttnError`` on a rejected call."""
    if stream is not None:
        with on_stream(stream, k):
            return kv4_write(k, v, cache, seq_lens, page_table, new_lens)
    n, ks, vs = k.shape, k.stride(), v.stride()
    device = k.get_device()
    if len(n) != 4 or device < 0 or k.dtype not in _DTYPE_CODES or ks[3] != 1:
        check_rows("k", k)
    if v.shape != n or v.dtype is not k.dtype or v.get_device() != device or vs[3] != 1:
        check_rows("v", v, n, k.dtype, device)
    B, Hk, N, d = n
    heads, page, num_pages, max_pages, pool, lens, new, table = _place(cache, d, B, seq_lens, new_lens, page_table, device)
    if Hk != heads:
        raise ValueError(f"k has {Hk} heads, the cache {heads}")
    run(_write, device, k.data_ptr(), v.data_ptr(), pool, lens, new, table, B, Hk, N, d, page, num_pages, max_pages,
        *ks, *vs, _DTYPE_CODES[k.dtype], _stream_handle(None, k))


def kv4_read(cache, N, d, seq_lens, page_table=None, new_lens=None, out_dtype=None, k_out=None, v_out=None,
             stream=None):
    """The keys and values [B, heads, N, d] that ``cache`` holds for N rows per sequence, as
    ``out_dtype`` (default bf16; exact).  Rows behind ``new_lens`` are left as they are in ``k_out``
    and ``v_out`` (in new tensors: unset).  ``new_lens=seq_lens`` with N at least the longest reads
    whole sequences, token i to row i."""
    if stream is not None:
        with on_stream(stream, cache):
            return kv4_read(cache, N, d, seq_lens, page_table, new_lens, out_dtype, k_out, v_out)
    B = seq_lens.shape[0] if seq_lens.dim() == 1 else -1
    device = cache.get_device()
    if device < 0:
        raise ValueError("cache must be a device tensor")
    heads, page, num_pages, max_pages, pool, lens, new, table = _place(cache, d, B, seq_lens, new_lens, page_table, device)
    dt = out_dtype or (_bf16 if k_out is None else k_out.dtype)
    if dt not in _DTYPE_CODES:
        raise TypeError(f"unsupported dtype {dt}; use torch.float32 or torch.bfloat16")
    n = (B, heads, N, d)
    if k_out is None:
        k_out = cache.new_empty(n, dtype=dt)
    else:
        check_rows("k_out", k_out, n, dt, device)
    if v_out is None:
        v_out = new_like(k_out)
    else:
        check_rows("v_out", v_out, n, dt, device)
    run(_read, device, pool, k_out.data_ptr(), v_out.data_ptr(), lens, new, table, B, heads, N, d, page, num_pages,
        max_pages, *k_out.stride(), *v_out.stride(), _DTYPE_CODES[dt], _stream_handle(None, cache))
    return k_out, v_out


def kv4_attn_fwd(q, cache, seq_lens, page_table=None, new_lens=None, scale=None, causal=False, max_len=0,
                 out_dtype=None, return_lse=False, num_splits=0, out=None, workspace=None, stream=None):
    """Attention of new queries q [B, Hq, N, d] (bf16) over ``cache``, whose heads each serve
    Hq / heads successive query heads.  ``causal``: query i sees the tokens up to its own,
    ``seq_lens[b] - new_lens[b] + i``; otherwise all ``seq_lens[b]``.  A row that sees nothing gets
    O = 0 and LSE = -inf; rows behind ``new_lens`` are left as they are.  ``max_len``: the longest
    sequence, where the caller knows it (it guides the key splits only; 0: the table's capacity).
    ``scale`` defaults to 1/sqrt(d).  Returns O [B, Hq, N, d] (and LSE [B, Hq, N] fp32 when
    ``return_lse``).  Raises ``MoaAttnError`` on a rejected call."""
    if stream is not None:
        with on_stream(stream, q):
            return kv4_attn_fwd(q, cache, seq_lens, page_table, new_lens, scale, causal, max_len, out_dtype, return_lse,
                                num_splits, out, workspace)
    n, qs = q.shape, q.stride()
    device = q.get_device()
    if len(n) != 4 or device < 0 or q.dtype is not _bf16 or qs[3] != 1:
        check_rows("q", q, dtype=_bf16)
    B, Hq, N, d = n
    heads, page, num_pages, max_pages, pool, lens, new, table = _place(cache, d, B, seq_lens, new_lens, page_table, device)
    odt = out_dtype or _bf16
    if odt not in _DTYPE_CODES:
        raise TypeError(f"unsupported dtype {odt}; use torch.float32 or torch.bfloat16")
    if out is None:
        out = new_like(q) if odt is _bf16 else q.new_empty(n, dtype=odt)
    else:
        check_rows("out", out, n, odt, device)
    lse = q.new_empty((B, Hq, N), dtype=torch.float32) if return_lse else None
    if workspace is None:
        need = _ws_bytes(B, Hq, heads, N, d, page, max_pages, max_len, num_splits)
        if need:
            workspace = q.new_empty(need, dtype=_uint8)
    ws, ws_n = _workspace(workspace, device)
    run(_attn, device, q.data_ptr(), pool, out.data_ptr(), lse.data_ptr() if return_lse else 0, lens, new, table, B, Hq,
        heads, N, d, page, num_pages, max_pages, max_len, *qs, *out.stride(),
        1.0 / math.sqrt(d) if scale is None else scale, causal, MOA_F32 if odt is torch.float32 else MOA_BF16, ws, ws_n,
        num_splits, _stream_handle(None, q))
    return (out, lse) if return_lse else out
