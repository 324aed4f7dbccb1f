"""Norms of queries and keys for each head with the rotation by position (``include/moa_rope.h``)."""
from __future__ import annotations

import torch

from . import _DTYPE_CODES
from ._call import (array, check_list, check_rows, ci, done, f32, function, handle, i64, on, ptr, same_device,
                    strides, sz, vp)

_ARGS = [i64] * 6
moa_qk_norm_rope = function(
    "moa_qk_norm_rope",
    [vp] * 8 + _ARGS + [vp] * 4 + [ci, vp, ci, f32, ci, ci, vp])
moa_qk_norm_rope_bwd = function(
    "moa_qk_norm_rope_bwd",
    [vp] * 12 + _ARGS + [vp] * 6 + [ci, vp, ci, f32, ci, ci, vp, sz, vp])
moa_qk_norm_rope_bwd_workspace_bytes = function("moa_qk_norm_rope_bwd_workspace_bytes", [i64] * 5, sz)


def _common(q, k, positions, inv_freq, q_weight, k_weight, sections):
    """Checks what forward and backward share: (B, Hq, Hk, N, d, rot, axes, weight type)."""
    check_rows("q", q)
    B, Hq, N, d = q.shape
    Hk = 0
    if k is not None:
        check_rows("k", k, (B, k.shape[1] if k.dim() == 4 else -1, N, d))
        Hk = k.shape[1]
        if k.dtype != q.dtype:
            raise TypeError("q and k must share one dtype")
    elif k_weight is not None:
        raise ValueError("k_weight without k")
    device = same_device(q, k, positions, inv_freq, q_weight, k_weight)
    wdt = None
    for name, w in (("q_weight", q_weight), ("k_weight", k_weight)):
        if w is None:
            continue
        if w.dtype not in _DTYPE_CODES or (wdt is not None and w.dtype != wdt):
            raise TypeError("q_weight and k_weight must both be torch.float32 or both torch.bfloat16")
        wdt = w.dtype
        check_list(name, w, (d,), wdt, device)
    rot = 0
    if inv_freq is not None:
        rot = 2 * inv_freq.numel()
        check_list("inv_freq", inv_freq, (rot // 2,), torch.float32, device)
    axes = 1 if sections is None else len(sections)
    if positions is not None:
        shape = (B, N) if sections is None else (axes, B, N)
        check_list("positions", positions, shape, torch.int64, device)
    return B, Hq, Hk, N, d, rot, axes, 0 if wdt is None else _DTYPE_CODES[wdt]


def _output(name, out, like):
    if out is None:
        return torch.empty(like.shape, dtype=like.dtype, device=like.device)
    check_rows(name, out, like.shape)
    if out.dtype != like.dtype or out.device != like.device:
        raise ValueError(f"{name} must have the input's dtype and device")
    return out


def qk_norm_rope(q, k=None, positions=None, inv_freq=None, q_weight=None, k_weight=None, eps=1e-6,
                 interleaved=False, sections=None, q_out=None, k_out=None, stream=None):
    """RMS norm of every head row of q [B, Hq, N, d] and k [B, Hk, N, d] with ``q_weight`` and
    ``k_weight`` [d] (None: no norm), then the rotation of its first ``2 * len(inv_freq)``
    elements by position (None: no rotation).

    q, k: bf16 or fp32 device tensors, any views with contiguous heads (slices of a packed
    projection output, ``[B, N, H, d]`` transposed); k may be None.  ``positions``: int64 [B, N],
    or [axes, B, N] with ``sections`` = rotated pairs of each axis (time, height, width, ...);
    None: 0 .. N-1.  ``inv_freq``: fp32 [rot/2], radians per position.  Pairs are (i, i + rot/2),
    or (2i, 2i + 1) when ``interleaved``.  ``q_out`` and ``k_out`` may be q and k (in place).
    Returns (q_out, k_out).  Raises ``MoaAttnError`` on a rejected call.
    """
    B, Hq, Hk, N, d, rot, axes, wcode = _common(q, k, positions, inv_freq, q_weight, k_weight, sections)
    qo = _output("q_out", q_out, q)
    ko = None if k is None else _output("k_out", k_out, k)
    with on(q.device):
        done(moa_qk_norm_rope(q.data_ptr(), ptr(k), qo.data_ptr(), ptr(ko), ptr(q_weight), ptr(k_weight),
                              ptr(positions), ptr(inv_freq), B, Hq, Hk, N, d, rot, strides(q), strides(k),
                              strides(qo), strides(ko), axes, array(sections), int(interleaved), float(eps),
                              _DTYPE_CODES[q.dtype], wcode, handle(stream, q)))
    return qo, ko


def qk_norm_rope_bwd(q, k, dq_out, dk_out, positions=None, inv_freq=None, q_weight=None, k_weight=None,
                     eps=1e-6, interleaved=False, sections=None, dq=None, dk=None, workspace=None,
                     stream=None):
    """Gradients of ``qk_norm_rope``: (dq, dk, dq_weight, dk_weight) from its inputs q and k and
    the gradients of its outputs (k and dk_out may be None).  dq and dk have q's dtype and may be
    given (also dq_out and dk_out themselves); the weights' gradients are fp32 [d], None where
    there is no weight.  The other arguments must be the forward's."""
    B, Hq, Hk, N, d, rot, axes, wcode = _common(q, k, positions, inv_freq, q_weight, k_weight, sections)
    if (k is None) != (dk_out is None):
        raise ValueError("k and dk_out go together")
    for name, g, x in (("dq_out", dq_out, q), ("dk_out", dk_out, k)):
        if x is None:
            continue
        check_rows(name, g, x.shape)
        if g.dtype != x.dtype or g.device != x.device:
            raise ValueError(f"{name} must have the input's dtype and device")
    dq = _output("dq", dq, q)
    dk = None if k is None else _output("dk", dk, k)
    dwq = None if q_weight is None else torch.empty(d, dtype=torch.float32, device=q.device)
    dwk = None if k_weight is None else torch.empty(d, dtype=torch.float32, device=q.device)
    if workspace is None and (dwq is not None or dwk is not None):
        n = moa_qk_norm_rope_bwd_workspace_bytes(B, Hq, Hk, N, d)
        workspace = torch.empty(n, dtype=torch.uint8, device=q.device)
    same_device(q, workspace)
    ws_n = 0 if workspace is None else workspace.numel() * workspace.element_size()
    with on(q.device):
        done(moa_qk_norm_rope_bwd(q.data_ptr(), ptr(k), dq_out.data_ptr(), ptr(dk_out), ptr(q_weight),
                                  ptr(k_weight), ptr(positions), ptr(inv_freq), dq.data_ptr(), ptr(dk),
                                  ptr(dwq), ptr(dwk), B, Hq, Hk, N, d, rot, strides(q), strides(k),
                                  strides(dq_out), strides(dk_out), strides(dq), strides(dk), axes,
                                  array(sections), int(interleaved), float(eps), _DTYPE_CODES[q.dtype],
                                  wcode, ptr(workspace), ws_n, handle(stream, q)))
    return dq, dk, dwq, dwk
