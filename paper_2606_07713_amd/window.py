"""Attention in a sliding window with first tokens that stay visible, and its gradients (``include/moa_window.h``).

Query i of Nq stands at position p = i + Nk - Nq and sees the keys j <= p + right with j >= p - left
or j < sinks; a negative left or right is no limit on that side (left=-1, right=0: the causal mask).
Query heads may share key/value heads: q [B, Hq, Nq, d], k and v [B, Hk, Nk, d], Hq a multiple of Hk.
"""
from __future__ import annotations

import functools
import math

from . import MOA_BF16, MOA_F32, _DTYPE_CODES, _stream_handle, _torch as torch
from ._call import (Function, Packed, check_list, check_rows, ci, f32, i64, is_list, new_like, on_stream, run, sz, vp,
                    workspace as _workspace)

_SPLIT = [i64] * 9 + [ci]
moa_win_attn_num_splits = Function("moa_win_attn_num_splits", _SPLIT)
moa_win_attn_workspace_bytes = Function("moa_win_attn_workspace_bytes", _SPLIT, sz)
moa_win_attn_fwd = Function(
    "moa_win_attn_fwd", [vp] * 5 + [i64] * 6 + [vp] * 4 + [i64] * 3 + [f32, ci, vp, sz, ci, vp])

moa_win_attn_bwd_workspace_bytes = Function("moa_win_attn_bwd_workspace_bytes", [i64] * 9, sz)
moa_win_attn_bwd = Function(
    "moa_win_attn_bwd", [vp] * 9 + [i64] * 6 + [vp] * 8 + [i64] * 3 + [f32, ci, vp, sz, vp])

_fwd = Packed("moa_packed_win_attn_fwd", "5q 6q 16q 3q d 5q")
_bwd = Packed("moa_packed_win_attn_bwd", "9q 6q 32q 3q d 4q")
_ws_bytes = functools.lru_cache(maxsize=1024)(moa_win_attn_workspace_bytes)
_bwd_ws_bytes = functools.lru_cache(maxsize=1024)(moa_win_attn_bwd_workspace_bytes)
if torch is not None:   # the C functions above need none
    _uint8, _bf16, _float32 = torch.uint8, torch.bfloat16, torch.float32


def _rows(name, t, shape, device):
    """t is a bf16 tensor of this shape on that device: its strides."""
    s = t.stride()
    if t.shape != shape or t.dtype is not _bf16 or t.get_device() != device or s[-1] != 1:
        check_rows(name, t, shape, _bf16, device)
    return s


def _common(q, k, v):
    """Checks what forward and backward share.  (sizes of q, of k, strides of q, k, v, device)."""
    qn, kn, qs = q.shape, k.shape, q.stride()
    device = q.get_device()
    if len(qn) != 4 or device < 0 or q.dtype is not _bf16 or qs[3] != 1:
        check_rows("q", q, dtype=_bf16)
    if len(kn) != 4 or kn[0] != qn[0] or kn[3] != qn[3]:
        raise ValueError(f"k must be [B, Hk, Nk, d] with q's B and d, got {tuple(kn)} for {tuple(qn)}")
    return qn, kn, qs, _rows("k", k, kn, device), _rows("v", v, kn, device), device


def win_attn_fwd(q, k, v, left=-1, right=-1, sinks=0, scale=None, out_dtype=None, return_lse=False, num_splits=0,
                 out=None, workspace=None, stream=None):
    """Attention of q [B, Hq, Nq, d] over k, v [B, Hk, Nk, d] (bf16, any views with contiguous heads)
    in a window.  ``scale`` defaults to 1/sqrt(d).  Returns O [B, Hq, Nq, d] of ``out_dtype`` (default
    bf16), and LSE [B, Hq, Nq] fp32 when ``return_lse``; a row that sees nothing gets O = 0 and LSE =
    -inf.  Raises ``MoaAttnError`` on a rejected call."""
    if stream is not None:
        with on_stream(stream, q):
            return win_attn_fwd(q, k, v, left, right, sinks, scale, out_dtype, return_lse, num_splits, out, workspace)
    qn, kn, qs, ks, vs, device = _common(q, k, v)
    B, Hq, Nq, d = qn
    odt = out_dtype or _bf16
    if odt not in _DTYPE_CODES:
        raise TypeError(f"unsupported dtype {odt}; use torch.float32 or torch.bfloat16")
    if out is None:
        out = new_like(q) if odt is _bf16 else q.new_empty(qn, dtype=odt)
    else:
        check_rows("out", out, qn, odt, device)
    lse = q.new_empty((B, Hq, Nq), dtype=torch.float32) if return_lse else None
    if workspace is None:
        need = _ws_bytes(B, Hq, kn[1], Nq, kn[2], d, left, right, sinks, num_splits)
        if need:
            workspace = q.new_empty(need, dtype=_uint8)
    ws, ws_n = _workspace(workspace, device)
    run(_fwd, device, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse.data_ptr() if return_lse else 0, B, Hq,
        kn[1], Nq, kn[2], d, *qs, *ks, *vs, *out.stride(), left, right, sinks, 1.0 / math.sqrt(d) if scale is None else scale,
        MOA_F32 if odt is torch.float32 else MOA_BF16, ws, ws_n, num_splits, _stream_handle(None, q))
    return (out, lse) if return_lse else out


def win_attn_bwd(q, k, v, o, do, lse, left=-1, right=-1, sinks=0, scale=None, dq=None, dk=None, dv=None, workspace=None,
                 stream=None):
    """Gradients of ``win_attn_fwd``: (dq, dk, dv), bf16, from its inputs, its outputs o (bf16 or fp32)
    and lse, and the gradient do [B, Hq, Nq, d] (bf16) of o; dk and dv are summed over the query heads
    that share a key/value head.  All tensors may be views with contiguous heads; dq, dk and dv may be
    given.  The other arguments must be the forward's."""
    if stream is not None:
        with on_stream(stream, q):
            return win_attn_bwd(q, k, v, o, do, lse, left, right, sinks, scale, dq, dk, dv, workspace)
    qn, kn, qs, ks, vs, device = _common(q, k, v)
    B, Hq, Nq, d = qn
    gs, os = _rows("do", do, qn, device), o.stride()
    if o.shape != qn or o.dtype not in _DTYPE_CODES or o.get_device() != device or os[-1] != 1:
        check_rows("o", o, qn, None, device)
    if not is_list(lse, (B, Hq, Nq), _float32, device):
        check_list("lse", lse, (B, Hq, Nq), _float32, device)
    dq, dk, dv = (new_like(x) if t is None else t for t, x in ((dq, q), (dk, k), (dv, v)))
    dqs, dks, dvs = _rows("dq", dq, qn, device), _rows("dk", dk, kn, device), _rows("dv", dv, kn, device)
    if workspace is None:
        need = _bwd_ws_bytes(B, Hq, kn[1], Nq, kn[2], d, left, right, sinks)
        if need:
            workspace = q.new_empty(need, dtype=_uint8)
    ws, ws_n = _workspace(workspace, device)
    run(_bwd, device, q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), do.data_ptr(), lse.data_ptr(), dq.data_ptr(),
        dk.data_ptr(), dv.data_ptr(), B, Hq, kn[1], Nq, kn[2], d, *qs, *ks, *vs, *os, *gs, *dqs, *dks, *dvs, left, right, sinks,
        1.0 / math.sqrt(d) if scale is None else scale, _DTYPE_CODES[o.dtype], ws, ws_n, _stream_handle(None, q))
    return dq, dk, dv
