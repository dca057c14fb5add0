"""Python binding of the Gated MLP's training step in libgmlp.so
(include/gmlp_train.h).

Argument marshalling only.  Names mirror the C entry points:

    forward(x, wg, wu, wd)                -> gmlp_train_forward   (y, g, u)
    backward(dy, x, wg, wu, wd, g, u)     -> gmlp_train_backward  (dx, dwg, dwu, dwd)
    describe(T, D, F, backward)           -> gmlp_train_describe
    workspace_size(T, D, F)               -> gmlp_train_workspace_size

A step keeps g and u (``torch.bfloat16`` [T, F]) from the forward call for the
backward call; everything else is recomputed.  Tensors and the workspace are as
for :mod:`paper_2606_26344_amd.gmlp`; without a workspace the calls take memory
for one call from torch's caching allocator.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

import torch

from .gmlp import (_CALL_DEVICE, FRESH_WORKSPACE, PATH_AUTO, Workspace, _check, _empty, _empty_like, _expect,
                   _on_current, _parse_plan, _prepared, _ptr, _scratch, _stream, _variant, library)

GRADIENTS = ("dx", "dwg", "dwu", "dwd")


def workspace_size(T: int, D: int, F: int) -> int:
    return int(library().gmlp_train_workspace_size(T, D, F))


def make_workspace(T: int, D: int, F: int, device=None, stream=None) -> Workspace:
    """A zeroed workspace that fits forward() and backward() of up to T tokens."""
    return Workspace(T, D, F, device=device, stream=stream, size=workspace_size)


def describe(T: int, D: int, F: int, backward: bool = True) -> list:
    """The kernels backward() (or forward()) enqueues: (name, grid, block, k_splits)."""
    buf = ctypes.create_string_buffer(1024)
    _check(library().gmlp_train_describe(T, D, F, int(backward), buf, len(buf)))
    return _parse_plan(buf)


def _workspace(workspace, T, D, F, device, rows, stream):
    """(tensor to keep, address, bytes, path) of a call's workspace."""
    if workspace is not None:
        return None, *_prepared(workspace, device), PATH_AUTO
    n = workspace_size(T, D, F)
    keep, ws = _scratch(n, rows, _CALL_DEVICE, stream, False, "invalid shape T=%d D=%d F=%d" % (T, D, F))
    return keep, ws, n, PATH_AUTO | FRESH_WORKSPACE


def _output(t, name, like, stream):
    """The given output, or a new one, of the shape of a tensor already checked."""
    if t is None:
        return _empty_like(like, stream)
    _expect(t, name, like.shape, like.device)
    return t


def _weights(x, wg, wu, wd):
    if x.dim() != 2 or wg.dim() != 2:
        raise ValueError("x and wg must be 2-D")
    T, D = x.shape
    F = wg.shape[1]
    dev = x.device
    _expect(x, "x", (T, D), dev)
    _expect(wg, "wg", (D, F), dev)
    _expect(wu, "wu", (D, F), dev)
    _expect(wd, "wd", (F, D), dev)
    _on_current(dev)
    return T, D, F, dev


def forward(x: torch.Tensor, wg: torch.Tensor, wu: torch.Tensor, wd: torch.Tensor,
            out: Optional[torch.Tensor] = None, g: Optional[torch.Tensor] = None, u: Optional[torch.Tensor] = None,
            activation: str = "silu", beta: float = 1.0, workspace: Optional[Workspace] = None, stream=None):
    """(y, g, u): y = (act(g) * u) wd with g = x wg, u = x wu, all bf16; g and u
    are for backward().  ``out``, ``g`` and ``u`` may be given to write into."""
    T, D, F, dev = _weights(x, wg, wu, wd)
    act, beta, _, _ = _variant(activation, beta, False, 0.0)
    out = _output(out, "out", x, stream)
    g = _empty((T, F), torch.bfloat16, dev, stream) if g is None else g
    u = _empty_like(g, stream) if u is None else u
    _expect(g, "g", (T, F), dev)
    _expect(u, "u", (T, F), dev)
    keep, ws, nbytes, path = _workspace(workspace, T, D, F, dev, T, stream)
    _check(library().gmlp_train_forward(x.data_ptr(), wg.data_ptr(), wu.data_ptr(), wd.data_ptr(), out.data_ptr(),
                                        g.data_ptr(), u.data_ptr(), T, D, F, act, beta, path, ws, nbytes,
                                        _stream(stream)))
    return out, g, u


def backward(dy: torch.Tensor, x: torch.Tensor, wg: torch.Tensor, wu: torch.Tensor, wd: torch.Tensor,
             g: torch.Tensor, u: torch.Tensor, activation: str = "silu", beta: float = 1.0,
             dx: Optional[torch.Tensor] = None, dwg: Optional[torch.Tensor] = None,
             dwu: Optional[torch.Tensor] = None, dwd: Optional[torch.Tensor] = None,
             want: Sequence[str] = GRADIENTS, workspace: Optional[Workspace] = None, stream=None):
    """(dx, dwg, dwu, dwd): the gradients of x and the weights from dy, that of
    forward()'s y, with the activation and beta of that call.  ``want`` names
    those to compute (the others are None); ``dx`` .. ``dwd`` may be given to
    write into."""
    T, D, F, dev = _weights(x, wg, wu, wd)
    _expect(dy, "dy", (T, D), dev)
    _expect(g, "g", (T, F), dev)
    _expect(u, "u", (T, F), dev)
    if want is not GRADIENTS and set(want) - set(GRADIENTS):
        raise ValueError("want names %s, the gradients are %s" % (sorted(set(want) - set(GRADIENTS)), GRADIENTS))
    act, beta, _, _ = _variant(activation, beta, False, 0.0)
    outs = []
    for name, t, like in (("dx", dx, x), ("dwg", dwg, wg), ("dwu", dwu, wu), ("dwd", dwd, wd)):
        if name in want:
            outs.append(_output(t, name, like, stream))
        elif t is not None:
            raise ValueError("%s is given but not wanted" % name)
        else:
            outs.append(None)
    # The weight gradients of no tokens are zeros, which a kernel writes.
    keep, ws, nbytes, path = _workspace(workspace, T, D, F, dev, 1, stream)
    _check(library().gmlp_train_backward(dy.data_ptr(), x.data_ptr(), wg.data_ptr(), wu.data_ptr(), wd.data_ptr(),
                                         g.data_ptr(), u.data_ptr(), *[_ptr(t) for t in outs], T, D, F, act, beta,
                                         path, ws, nbytes, _stream(stream)))
    return tuple(outs)
