"""A paged key/value cache in bf16: appending to it and the attention over it (``include/moa_paged.h``).

A cache is two bf16 tensors [num_pages, heads, page, d] (``paged_cache``; any views with contiguous
heads), page a power of two from 16 on.  ``seq_lens`` int32 [B] counts the tokens of every sequence,
the call's new ones included; ``page_table`` int32 [B, max_pages] names the pages of each (None:
sequence b has page b alone); ``new_lens`` int32 [B] says how many of a call's N rows per sequence
are real (None: all).  Row i of sequence b is token ``seq_lens[b] - new_lens[b] + i``.
"""
from __future__ import annotations

import functools
import math

from . import MOA_BF16, MOA_F32, _DTYPE_CODES, _stream_handle, _torch as torch
from ._call import (Function, Packed, check_list, check_rows, ci, f32, i64, is_list, new_like, on_stream, run, sz, vp,
                    workspace as _workspace)
from .rope import _HOW, _common

_SPLIT = [i64] * 11 + [ci]
moa_paged_attn_num_splits = Function("moa_paged_attn_num_splits", _SPLIT)
moa_paged_attn_workspace_bytes = Function("moa_paged_attn_workspace_bytes", _SPLIT, sz)
moa_paged_attn_fwd = Function(
    "moa_paged_attn_fwd", [vp] * 8 + [i64] * 9 + [vp] * 4 + [i64] * 3 + [f32, ci, vp, sz, ci, vp])
moa_paged_append = Function(
    "moa_paged_append", [vp] * 13 + [i64] * 9 + [vp] * 6 + [ci, vp, ci, f32, ci, ci, vp])

_append = Packed("moa_packed_paged_append", "13q 9q 24q" + _HOW + "q")
_attn = Packed("moa_packed_paged_attn_fwd", "8q 9q 16q 3q d 5q")
_ws_bytes = functools.lru_cache(maxsize=1024)(moa_paged_attn_workspace_bytes)
if torch is not None:   # the C functions above need none
    _int32, _uint8, _bf16 = torch.int32, torch.uint8, torch.bfloat16


def paged_cache(num_pages, heads, page, d, device="cuda"):
    """The two pools of an empty cache, ``num_pages`` pages of ``page`` tokens (a power of two from
    16 on) of ``heads`` key/value heads of size d (64 or 128).  Their contents need not be set."""
    if page < 16 or page > 1 << 20 or page & (page - 1) or d not in (64, 128):
        raise ValueError("page must be a power of two in 16..2^20, d 64 or 128")
    return tuple(torch.empty((num_pages, heads, page, d), dtype=torch.bfloat16, device=device) for _ in range(2))


def _place(k_pool, v_pool, d, B, seq_lens, new_lens, page_table, device):
    """Checks the pools and the lists.  (heads, page, num_pages, max_pages, strides of both pools,
    addresses of the pools, seq_lens, new_lens and page_table)."""
    n, ks, vs = k_pool.shape, k_pool.stride(), v_pool.stride()
    if len(n) != 4 or n[3] != d or k_pool.dtype is not _bf16 or k_pool.get_device() != device or ks[3] != 1:
        raise ValueError(f"k_pool must be a bf16 tensor [num_pages, heads, page, {d}] with contiguous heads on the other "
                         "tensors' device")
    if v_pool.shape != n or v_pool.dtype is not _bf16 or v_pool.get_device() != device or vs[3] != 1:
        raise ValueError("v_pool must be a tensor like k_pool")
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
    elif n[0] < B:
        raise ValueError("a cache without a page table needs a page for every sequence")
    return (n[1], n[2], n[0], max_pages, ks, vs, k_pool.data_ptr(), v_pool.data_ptr(), seq_lens.data_ptr(), new, table)


def paged_append(q, k, v, k_pool, v_pool, seq_lens, page_table=None, new_lens=None, positions=None, inv_freq=None,
                 q_weight=None, k_weight=None, eps=1e-6, interleaved=False, sections=None, q_out=None, stream=None):
    """New tokens into the cache: head rows of q [B, Hq, N, d] and k [B, heads, N, d] normed with
    ``q_weight`` and ``k_weight`` and turned by position as ``qk_norm_rope`` does (None: no norm, no
    rotation), keys and values v [B, heads, N, d] written to their pages.  q, k, v are bf16 or fp32,
    any views with contiguous heads; q may be None.  ``positions``: contiguous int64 [B, N], or
    [axes, B, N] with ``sections``; None: every token's place in its sequence.  Returns the turned
    queries, bf16 ``q_out`` (which may be a bf16 q); rows behind ``new_lens`` are left as they are
    (in a new tensor: unset).  Raises ``MoaAttnError`` on a rejected call."""
    if stream is not None:
        with on_stream(stream, k):
            return paged_append(q, k, v, k_pool, v_pool, seq_lens, page_table, new_lens, positions, inv_freq, q_weight,
                                k_weight, eps, interleaved, sections, q_out)
    if q is None:
        if q_weight is not None or q_out is not None:
            raise ValueError("q_weight and q_out go with q")
        kn, _, ks, _, device, rot, axes, sec, wcode, (kp, _, wk, _, pos, freq) = _common(
            k, None, positions, inv_freq, k_weight, None, sections)
        Hq, qs, qos, qp, qop, wq = 0, ks, ks, 0, 0, 0
    else:
        qn, kn, qs, ks, device, rot, axes, sec, wcode, (qp, kp, wq, wk, pos, freq) = _common(
            q, k, positions, inv_freq, q_weight, k_weight, sections)
        Hq = qn[1]
        if q_out is None:
            q_out = new_like(q) if q.dtype is _bf16 else q.new_empty(qn, dtype=_bf16)
        qos = q_out.stride()
        if q_out.shape != qn or q_out.dtype is not _bf16 or q_out.get_device() != device or qos[3] != 1:
            check_rows("q_out", q_out, qn, _bf16, device)
        qop = q_out.data_ptr()
    vs = v.stride()
    if v.shape != kn or v.dtype is not k.dtype or v.get_device() != device or vs[-1] != 1:
        check_rows("v", v, kn, k.dtype, device)
    B, Hk, N, d = kn
    heads, page, num_pages, max_pages, kps, vps, kpp, vpp, lens, new, table = _place(
        k_pool, v_pool, d, B, seq_lens, new_lens, page_table, device)
    if Hk != heads:
        raise ValueError(f"k has {Hk} heads, the cache {heads}")
    run(_append, device, qp, kp, v.data_ptr(), qop, kpp, vpp, wq, wk, pos, freq, lens, new, table, B, Hq, Hk, N, d, rot, page,
        num_pages, max_pages, *qs, *ks, *vs, *qos, *kps, *vps, axes, *sec, interleaved, eps, _DTYPE_CODES[k.dtype], wcode,
        _stream_handle(None, k))
    return q_out


def paged_attn_fwd(q, k_pool, v_pool, seq_lens, page_table=None, new_lens=None, left=-1, right=-1, sinks=0, scale=None,
                   max_len=0, out_dtype=None, return_lse=False, num_splits=0, out=None, workspace=None, stream=None):
    """Attention of new queries q [B, Hq, N, d] (bf16) over the cache, whose heads each serve
    Hq / heads successive query heads.  Query i of sequence b stands at its token's position p and
    sees the tokens j <= p + right with j >= p - left or j < sinks; a negative left or right is no
    limit on that side (right=0: the causal mask).  Tokens on a page outside the pool (an entry of
    -1) are not visible; a row that sees nothing gets O = 0 and LSE = -inf; rows behind ``new_lens``
    are left as they are.  ``max_len``: the longest sequence, where the caller knows it (it guides the
    key splits only; 0: the table's capacity).  ``scale`` defaults to 1/sqrt(d).  Returns O
    [B, Hq, N, d] (and LSE [B, Hq, N] fp32 when ``return_lse``).  Raises ``MoaAttnError`` on a
    rejected call."""
    if stream is not None:
        with on_stream(stream, q):
            return paged_attn_fwd(q, k_pool, v_pool, seq_lens, page_table, new_lens, left, right, sinks, scale, max_len,
                                  out_dtype, return_lse, num_splits, out, workspace)
    n, qs = q.shape, q.stride()
    device = q.get_device()
    if len(n) != 4 or device < 0 or q.dtype is not _bf16 or qs[3] != 1:
        check_rows("q", q, dtype=_bf16)
    B, Hq, N, d = n
    heads, page, num_pages, max_pages, ks, vs, kp, vp_, lens, new, table = _place(
        k_pool, v_pool, d, B, seq_lens, new_lens, page_table, device)
    odt = out_dtype or _bf16
    if odt not in _DTYPE_CODES:
        raise TypeError(f"unsupported dtype {odt}; use torch.float32 or torch.bfloat16")
    if out is None:
        out = new_like(q) if odt is _bf16 else q.new_empty(n, dtype=odt)
    else:
        check_rows("out", out, n, odt, device)
    lse = q.new_empty((B, Hq, N), dtype=torch.float32) if return_lse else None
    if workspace is None:
        need = _ws_bytes(B, Hq, heads, N, d, page, max_pages, max_len, left, right, sinks, num_splits)
        if need:
            workspace = q.new_empty(need, dtype=_uint8)
    ws, ws_n = _workspace(workspace, device)
    run(_attn, device, q.data_ptr(), kp, vp_, out.data_ptr(), lse.data_ptr() if return_lse else 0, lens, new, table, B, Hq,
        heads, N, d, page, num_pages, max_pages, max_len, *qs, *ks, *vs, *out.stride(), left, right, sinks,
        1.0 / math.sqrt(d) if scale is None else scale, MOA_F32 if odt is torch.float32 else MOA_BF16, ws, ws_n, num_splits,
        _stream_handle(None, q))
    return (out, lse) if return_lse else out
