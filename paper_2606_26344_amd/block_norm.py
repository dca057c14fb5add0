"""Python binding of the norms between two blocks in libgmlp.so
(include/gmlp_block_norm.h).

Argument marshalling only.  Names mirror the C entry points:

    forward(y, res, ...)           -> gmlp_block_norm           (r, xn)
    backward(dxn, dr, y, r, ...)   -> gmlp_block_norm_backward  (dy, dres, dw_pre, dw_post, dgate)
    workspace_size(T, D)           -> gmlp_block_norm_workspace_size

    z = y, or with ``post`` y / rms(y) * w_post
    r = res_scale * res + gate * z
    xn = r / rms(r) * w_pre

y, xn [T, D], the gains w_pre and w_post [D] and the gate ([D], or [T, D]) are
``torch.bfloat16``; the residual stream res, r [T, D] is ``torch.bfloat16`` or
``torch.float32``.  All contiguous, on one HIP device.
"""
from __future__ import annotations

from typing import Optional

import torch

from .gmlp import _CALL_DEVICE, _check, _empty, _empty_like, _expect, _on_current, _ptr, _scratch, _stream, library

POST, RES_FP32, GATE_ROWS = 1, 2, 4


def workspace_size(T: int, D: int) -> int:
    return int(library().gmlp_block_norm_workspace_size(T, D))


class Workspace:
    """A caller-owned workspace for backward(); it needs no preparation.  (The
    calls of the other modules need theirs prepared, which backward() would undo:
    neither takes the other's.)"""

    def __init__(self, T: int, D: int, device=None, stream=None):
        n = workspace_size(T, D)
        if n == 0:
            raise ValueError("invalid shape T=%d D=%d" % (T, D))
        # Allocated on the stream the calls will run on, with slack to align it.
        self.storage = _empty((n + 256,), torch.uint8, device or "cuda", stream)
        off = (-self.storage.data_ptr()) % 256
        self.buffer = self.storage[off:off + n]
        self.nbytes = n


def make_workspace(T: int, D: int, device=None, stream=None) -> Workspace:
    """A workspace that fits backward() of up to T rows of D."""
    return Workspace(T, D, device=device, stream=stream)


def _stream_tensor(t, name, shape, device, dtype) -> None:
    """Expects a tensor of the residual stream."""
    if dtype is torch.bfloat16:
        _expect(t, name, shape, device)
    elif (not isinstance(t, torch.Tensor) or t.dtype is not torch.float32 or t.device != device
          or tuple(t.shape) != tuple(shape) or not t.is_contiguous()):
        raise ValueError("%s must be a contiguous float32 tensor of shape %s on %s" % (name, tuple(shape), device))


def _options(like, name, w_pre, w_post, gate, post):
    """(T, D, device, dtype of the residual stream, flags) of a call."""
    if not isinstance(like, torch.Tensor) or like.dim() != 2:
        raise ValueError("%s must be a 2-D tensor" % name)
    if like.dtype not in (torch.bfloat16, torch.float32):
        raise TypeError("%s must be torch.bfloat16 or torch.float32, got %s" % (name, like.dtype))
    T, D = like.shape
    dev = like.device
    if dev.type != "cuda":
        raise ValueError("%s must be on a HIP device, got %s" % (name, dev))
    _on_current(dev)
    _stream_tensor(like, name, (T, D), dev, like.dtype)
    flags = (POST if post else 0) | (RES_FP32 if like.dtype is torch.float32 else 0)
    for t, n in ((w_pre, "w_pre"), (w_post, "w_post")):
        if t is not None:
            _expect(t, n, (D,), dev)
    if gate is not None:
        if gate.dim() == 2:
            _expect(gate, "gate", (T, D), dev)
            flags |= GATE_ROWS
        else:
            _expect(gate, "gate", (D,), dev)
    return T, D, dev, like.dtype, flags


def forward(y: Optional[torch.Tensor], res: torch.Tensor, w_pre: Optional[torch.Tensor] = None,
            w_post: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None, post: bool = False,
            res_scale: float = 1.0, eps: float = 1e-6, r: Optional[torch.Tensor] = None,
            xn: Optional[torch.Tensor] = None, stream=None):
    """(r, xn).  ``y`` None: the norm before the first block (r = res_scale *
    res).  ``r`` (which may be ``res``) and ``xn`` (which may be ``y``) may be
    given to write into."""
    T, D, dev, dtype, flags = _options(res, "res", w_pre, w_post, gate, post)
    if y is not None:
        _expect(y, "y", (T, D), dev)
    if r is None:
        r = _empty_like(res, stream)
    else:
        _stream_tensor(r, "r", (T, D), dev, dtype)
    if xn is None:
        xn = _empty((T, D), torch.bfloat16, dev, stream) if y is None else _empty_like(y, stream)
    else:
        _expect(xn, "xn", (T, D), dev)
    _check(library().gmlp_block_norm(_ptr(y), res.data_ptr(), _ptr(w_pre), _ptr(w_post), _ptr(gate), r.data_ptr(),
                                     xn.data_ptr(), T, D, flags, res_scale, eps, _stream(stream)))
    return r, xn


def backward(dxn: torch.Tensor, dr: Optional[torch.Tensor], y: Optional[torch.Tensor], r: torch.Tensor,
             w_pre: Optional[torch.Tensor] = None, w_post: Optional[torch.Tensor] = None,
             gate: Optional[torch.Tensor] = None, post: bool = False, res_scale: float = 1.0, eps: float = 1e-6,
             dy: Optional[torch.Tensor] = None, dres: Optional[torch.Tensor] = None,
             workspace: Optional[Workspace] = None, stream=None):
    """(dy, dres, dw_pre, dw_post, dgate) from dxn and dr, the gradients of
    forward()'s xn and r (``dr`` None: zeros), its y and its r; None for an
    input that was None.  ``dy`` (which may be ``dxn``) and ``dres`` (which may
    be ``dr``) may be given to write into."""
    T, D, dev, dtype, flags = _options(r, "r", w_pre, w_post, gate, post)
    _expect(dxn, "dxn", (T, D), dev)
    if dr is not None:
        _stream_tensor(dr, "dr", (T, D), dev, dtype)
    if y is not None:
        _expect(y, "y", (T, D), dev)
        if dy is None:
            dy = _empty_like(y, stream)
        else:
            _expect(dy, "dy", (T, D), dev)
    elif dy is not None:
        raise ValueError("dy is given without y")
    if dres is None:
        dres = _empty_like(r, stream)
    else:
        _stream_tensor(dres, "dres", (T, D), dev, dtype)
    dw_pre, dw_post, dgate = (None if t is None else _empty_like(t, stream) for t in (w_pre, w_post, gate))
    if workspace is None:
        nbytes = workspace_size(T, D)
        keep, ws = _scratch(nbytes, 1, _CALL_DEVICE, stream, False, "invalid shape T=%d D=%d" % (T, D))
    elif not isinstance(workspace, Workspace):
        raise TypeError("workspace must be one of make_workspace(), got %s" % type(workspace).__name__)
    elif workspace.buffer.device != dev:
        raise ValueError("workspace must be on %s, got %s" % (dev, workspace.buffer.device))
    else:
        keep, ws, nbytes = None, workspace.buffer.data_ptr(), workspace.nbytes
    _check(library().gmlp_block_norm_backward(
        dxn.data_ptr(), _ptr(dr), _ptr(y), r.data_ptr(), _ptr(w_pre), _ptr(w_post), _ptr(gate), _ptr(dy),
        dres.data_ptr(), _ptr(dw_pre), _ptr(dw_post), _ptr(dgate), T, D, flags, res_scale, eps, ws, nbytes,
        _stream(stream)))
    return dy, dres, dw_pre, dw_post, dgate
