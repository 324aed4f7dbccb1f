"""Norms of queries and keys for each head with the rotation by position (``include/moa_rope.h``)."""
from __future__ import annotations

import functools

from . import MOA_F32, _DTYPE_CODES, _stream_handle, _torch as torch
from ._call import (Function, Packed, check_list, check_rows, ci, f32, i64, is_list, new_like, on_stream, run, sz, vp,
                    workspace as _workspace)

_SIZES = [i64] * 6
moa_qk_norm_rope = Function(
    "moa_qk_norm_rope",
    [vp] * 8 + _SIZES + [vp] * 4 + [ci, vp, ci, f32, ci, ci, vp])
moa_qk_norm_rope_bwd = Function(
    "moa_qk_norm_rope_bwd",
    [vp] * 12 + _SIZES + [vp] * 6 + [ci, vp, ci, f32, ci, ci, vp, sz, vp])
moa_qk_norm_rope_bwd_workspace_bytes = Function("moa_qk_norm_rope_bwd_workspace_bytes", [i64] * 5, sz)

_HOW = "q 5q q d 2q"   # axes, sections with a flag before, interleaved, eps, types
_fwd = Packed("moa_packed_qk_norm_rope", "8q 6q 16q" + _HOW + "q")
_bwd = Packed("moa_packed_qk_norm_rope_bwd", "12q 6q 24q" + _HOW + "3q")
_bwd_ws_bytes = functools.lru_cache(maxsize=1024)(moa_qk_norm_rope_bwd_workspace_bytes)
_NONE4, _NONE5 = (0,) * 4, (0,) * 5   # strides and sections that are not there
if torch is not None:   # the C functions above need none
    _int64, _float32, _empty_like = torch.int64, torch.float32, torch.empty_like


def _like(name, t, x, shape, device):
    """t is a tensor like x: its strides."""
    s = t.stride()
    if t.shape != shape or t.dtype is not x.dtype or t.get_device() != device or s[-1] != 1:
        check_rows(name, t, shape, x.dtype, device)
    return s


def _weight(name, w, d, device):
    code = _DTYPE_CODES.get(w.dtype)
    if code is None:
        raise TypeError(f"{name}: unsupported dtype {w.dtype}; use torch.float32 or torch.bfloat16")
    if w.shape != (d,) or w.get_device() != device or not w.is_contiguous():
        check_list(name, w, (d,), w.dtype, device)
    return code


def _common(q, k, positions, inv_freq, q_weight, k_weight, sections):
    """Checks what forward and backward share.  (shape of q, of k, strides of q, of k, device,
    rot, axes, sections with a flag before, weight type, addresses)."""
    qn = q.shape
    device = q.get_device()
    qs = q.stride()
    if len(qn) != 4 or device < 0 or q.dtype not in _DTYPE_CODES or qs[3] != 1:
        check_rows("q", q)
    B, _, N, d = qn
    kn, ks, kp = (B, 0, N, d), _NONE4, 0
    if k is not None:
        kn = k.shape
        if len(kn) != 4 or kn[0] != B or kn[2] != N or kn[3] != d:
            raise ValueError(f"k must be [B, Hk, N, d] with q's B, N and d, got {tuple(kn)} for {tuple(qn)}")
        ks = _like("k", k, q, kn, device)
        kp = k.data_ptr()
    elif k_weight is not None:
        raise ValueError("k_weight without k")
    wcode, wq, wk = MOA_F32, 0, 0
    if q_weight is not None:
        wcode = _weight("q_weight", q_weight, d, device)
        wq = q_weight.data_ptr()
    if k_weight is not None:
        code = _weight("k_weight", k_weight, d, device)
        if q_weight is not None and code != wcode:
            raise TypeError("q_weight and k_weight must share one dtype")
        wcode, wk = code, k_weight.data_ptr()
    rot, freq = 0, 0
    if inv_freq is not None:
        n = inv_freq.shape[0] if inv_freq.dim() == 1 else -1
        if not is_list(inv_freq, (n,), _float32, device):
            check_list("inv_freq", inv_freq, (n,), _float32, device)
        rot, freq = 2 * n, inv_freq.data_ptr()
    axes, sec = 1, _NONE5
    if sections is not None:   # more than four are refused by their number
        axes, sec = len(sections), (1, *map(int, sections), 0, 0, 0, 0)[:5]
    pos = 0
    if positions is not None:
        shape = (B, N) if sections is None else (axes, B, N)
        if not is_list(positions, shape, _int64, device):
            check_list("positions", positions, shape, _int64, device)
        pos = positions.data_ptr()
    return qn, kn, qs, ks, device, rot, axes, sec, wcode, (q.data_ptr(), kp, wq, wk, pos, freq)


def qk_norm_rope(q, k=None, positions=None, inv_freq=None, q_weight=None, k_weight=None, eps=1e-6,
                 interleaved=False, sections=None, q_out=None, k_out=None, stream=None):
    """RMS norm of every head row of q [B, Hq, N, d] and k [B, Hk, N, d] with ``q_weight`` and
    ``k_weight`` [d] (None: no norm), then the rotation of its first ``2 * len(inv_freq)``
    elements by position (None: no rotation).

    q, k: bf16 or fp32 device tensors, any views with contiguous heads (slices of a packed
    projection output, ``[B, N, H, d]`` transposed); k may be None.  ``positions``: contiguous
    int64 [B, N], or [axes, B, N] with ``sections`` = rotated pairs of each axis (time, height, width, ...);
    None: 0 .. N-1.  ``inv_freq``: fp32 [rot/2], radians per position.  Pairs are (i, i + rot/2),
    or (2i, 2i + 1) when ``interleaved``.  ``q_out`` and ``k_out`` may be q and k (in place).
    Returns (q_out, k_out).  Raises ``MoaAttnError`` on a rejected call.
    """
    if stream is not None:
        with on_stream(stream, q):
            return qk_norm_rope(q, k, positions, inv_freq, q_weight, k_weight, eps, interleaved, sections, q_out, k_out)
    qn, kn, qs, ks, device, rot, axes, sec, wcode, (qp, kp, wq, wk, pos, freq) = _common(
        q, k, positions, inv_freq, q_weight, k_weight, sections)
    if q_out is None:
        q_out = new_like(q)
    qos = _like("q_out", q_out, q, qn, device)
    kos, kop = ks, 0
    if k is not None:
        if k_out is None:
            k_out = new_like(k)
        kos, kop = _like("k_out", k_out, k, kn, device), k_out.data_ptr()
    B, Hq, N, d = qn
    run(_fwd, device, qp, kp, q_out.data_ptr(), kop, wq, wk, pos, freq, B, Hq, kn[1], N, d, rot, *qs, *ks, *qos, *kos,
        axes, *sec, interleaved, eps, _DTYPE_CODES[q.dtype], wcode, _stream_handle(None, q))
    return q_out, (None if k is None else k_out)


def qk_norm_rope_bwd(q, k, dq_out, dk_out, positions=None, inv_freq=None, q_weight=None, k_weight=None,
                     eps=1e-6, interleaved=False, sections=None, dq=None, dk=None, workspace=None,
                     stream=None):
    """Gradients of ``qk_norm_rope``: (dq, dk, dq_weight, dk_weight) from its inputs q and k and
    the gradients of its outputs (k and dk_out may be None).  dq and dk have q's dtype and may be
    given (also dq_out and dk_out themselves); the weights' gradients are fp32 [d], None where
    there is no weight.  The other arguments must be the forward's."""
    if stream is not None:
        with on_stream(stream, q):
            return qk_norm_rope_bwd(q, k, dq_out, dk_out, positions, inv_freq, q_weight, k_weight, eps, interleaved,
                                    sections, dq, dk, workspace)
    qn, kn, qs, ks, device, rot, axes, sec, wcode, (qp, kp, wq, wk, pos, freq) = _common(
        q, k, positions, inv_freq, q_weight, k_weight, sections)
    if (k is None) != (dk_out is None):
        raise ValueError("k and dk_out go together")
    if dq is None:
        dq = new_like(q)
    gqs, dqs = _like("dq_out", dq_out, q, qn, device), _like("dq", dq, q, qn, device)
    gks, dks, gkp, dkp = ks, ks, 0, 0
    if k is not None:
        if dk is None:
            dk = new_like(k)
        gks, dks = _like("dk_out", dk_out, k, kn, device), _like("dk", dk, k, kn, device)
        gkp, dkp = dk_out.data_ptr(), dk.data_ptr()
    B, Hq, N, d = qn
    dwq = None if q_weight is None else _empty_like(q_weight, dtype=_float32)
    dwk = None if k_weight is None else _empty_like(k_weight, dtype=_float32)
    if workspace is None and (dwq is not None or dwk is not None):
        workspace = q.new_empty(_bwd_ws_bytes(B, Hq, kn[1], N, d), dtype=torch.uint8)
    ws, ws_n = _workspace(workspace, device)
    run(_bwd, device, qp, kp, dq_out.data_ptr(), gkp, wq, wk, pos, freq, dq.data_ptr(), dkp,
        0 if dwq is None else dwq.data_ptr(), 0 if dwk is None else dwk.data_ptr(), B, Hq, kn[1], N, d, rot, *qs, *ks,
        *gqs, *gks, *dqs, *dks, axes, *sec, interleaved, eps, _DTYPE_CODES[q.dtype], wcode, ws, ws_n,
        _stream_handle(None, q))
    return dq, (None if k is None else dk), dwq, dwk
