"""Python binding of the experts' Gated MLPs in libgmlp.so (include/gmlp_experts.h),
over rows sorted by expert (:mod:`paper_2606_26344_amd.route`).

Argument marshalling only.  Names mirror the C entry points:

    forward(xs, offsets, wg, wu, wd)                    -> gmlp_experts_forward   ys
    train_forward(xs, offsets, wg, wu, wd)              -> gmlp_experts_forward   (ys, g, u)
    backward(dys, xs, offsets, wg, wu, wd, g, u)        -> gmlp_experts_backward  (dxs, dwg, dwu, dwd)
    describe(N, E, D, F, backward)                      -> gmlp_experts_describe
    workspace_size(N, E, D, F)                          -> gmlp_experts_workspace_size

xs, ys, dxs, dys [N, D] and g, u [N, F] are ``torch.bfloat16``, as are the weights wg, wu
[E, D, F] and wd [E, F, D]; offsets [E + 1] is int32: expert e has the rows offsets[e] ..
offsets[e + 1] - 1 (offsets that fall count as their running maximum).  Rows that no expert
has are not written.  All contiguous, on one HIP device.  Without a workspace the calls
take memory for one call from torch's caching allocator.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

import torch

from . import gmlp
from .gmlp import (_CALL_DEVICE, FRESH_WORKSPACE, PATH_AUTO, _check, _empty, _empty_like, _expect, _on_current,
                   _parse_plan, _prepared, _ptr, _scratch, _stream, _variant, library)
from .route import _numbers

GRADIENTS = ("dxs", "dwg", "dwu", "dwd")


def workspace_size(N: int, E: int, D: int, F: int) -> int:
    return int(library().gmlp_experts_workspace_size(N, E, D, F))


class Workspace(gmlp.Workspace):
    """A caller-owned workspace for the calls of this module, prepared at creation."""

    def __init__(self, N: int, E: int, D: int, F: int, device=None, stream=None):
        n = workspace_size(N, E, D, F)
        if n == 0:
            raise ValueError("invalid shape N=%d E=%d D=%d F=%d" % (N, E, D, F))
        super().__init__(N, D, F, device=device, stream=stream, nbytes=n)

    def fits(self, N: int, E: int, D: int, F: int) -> bool:
        """Whether it is large enough for calls of this (valid) shape."""
        return 0 < workspace_size(N, E, D, F) <= self.nbytes


def make_workspace(N: int, E: int, D: int, F: int, device=None, stream=None) -> Workspace:
    """A prepared workspace that fits the calls of up to N rows."""
    return Workspace(N, E, D, F, device=device, stream=stream)


def describe(N: int, E: int, D: int, F: int, backward: bool = False) -> list:
    """The kernels forward() (or backward()) enqueues: (name, grid, block, most k_splits)."""
    buf = ctypes.create_string_buffer(1024)
    _check(library().gmlp_experts_describe(N, E, D, F, int(backward), buf, len(buf)))
    return _parse_plan(buf)


def _workspace(workspace, N, E, D, F, device, rows, stream):
    """(tensor to keep, address, bytes, path) of a call's workspace."""
    if workspace is not None:
        return None, *_prepared(workspace, device), PATH_AUTO
    n = workspace_size(N, E, D, F)
    keep, ws = _scratch(n, rows, _CALL_DEVICE, stream, False, "invalid shape N=%d E=%d D=%d F=%d" % (N, E, D, F))
    return keep, ws, n, PATH_AUTO | FRESH_WORKSPACE


def _output(t, name, shape, device, stream):
    """The given output, or a new one."""
    if t is None:
        return _empty(shape, torch.bfloat16, device, stream)
    _expect(t, name, shape, device)
    return t


def _arguments(xs, offsets, wg, wu, wd):
    """(N, E, D, F, device) of checked inputs."""
    for t, name, dims in ((xs, "xs", 2), (wg, "wg", 3)):
        if not isinstance(t, torch.Tensor) or t.dim() != dims:
            raise ValueError("%s must be a %d-D tensor" % (name, dims))
    N, D = xs.shape
    E, _, F = wg.shape
    dev = xs.device
    _expect(xs, "xs", (N, D), dev)
    _expect(wg, "wg", (E, D, F), dev)
    _expect(wu, "wu", (E, D, F), dev)
    _expect(wd, "wd", (E, F, D), dev)
    _numbers(offsets, "offsets", (E + 1,), dev, (torch.int32,))
    _on_current(dev)
    return N, E, D, F, dev


def _forward(xs, offsets, wg, wu, wd, out, g, u, keep_gates, activation, beta, workspace, stream):
    N, E, D, F, dev = _arguments(xs, offsets, wg, wu, wd)
    act, beta, _, _ = _variant(activation, beta, False, 0.0)
    out = _output(out, "out", (N, D), dev, stream)
    if keep_gates:
        g, u = _output(g, "g", (N, F), dev, stream), _output(u, "u", (N, F), dev, stream)
    keep, ws, nbytes, path = _workspace(workspace, N, E, D, F, dev, N, stream)
    _check(library().gmlp_experts_forward(_ptr(xs), offsets.data_ptr(), wg.data_ptr(), wu.data_ptr(), wd.data_ptr(),
                                          _ptr(out), _ptr(g), _ptr(u), N, E, D, F, act, beta, path, ws, nbytes,
                                          _stream(stream)))
    return out, g, u


def forward(xs: torch.Tensor, offsets: torch.Tensor, wg: torch.Tensor, wu: torch.Tensor, wd: torch.Tensor,
            out: Optional[torch.Tensor] = None, activation: str = "silu", beta: float = 1.0,
            workspace: Optional[Workspace] = None, stream=None) -> torch.Tensor:
    """ys [N, D]: each expert's Gated MLP of its rows.  ``out`` may be given to write
    into."""
    return _forward(xs, offsets, wg, wu, wd, out, None, None, False, activation, beta, workspace, stream)[0]


def train_forward(xs: torch.Tensor, offsets: torch.Tensor, wg: torch.Tensor, wu: torch.Tensor, wd: torch.Tensor,
                  out: Optional[torch.Tensor] = None, g: Optional[torch.Tensor] = None,
                  u: Optional[torch.Tensor] = None, activation: str = "silu", beta: float = 1.0,
                  workspace: Optional[Workspace] = None, stream=None):
    """(ys, g, u): forward(), and g = xs wg, u = xs wu [N, F] for backward().  All may be
    given to write into."""
    return _forward(xs, offsets, wg, wu, wd, out, g, u, True, activation, beta, workspace, stream)


def backward(dys: torch.Tensor, xs: torch.Tensor, offsets: torch.Tensor, wg: torch.Tensor, wu: torch.Tensor,
             wd: torch.Tensor, g: torch.Tensor, u: torch.Tensor, activation: str = "silu", beta: float = 1.0,
             dxs: Optional[torch.Tensor] = None, dwg: Optional[torch.Tensor] = None,
             dwu: Optional[torch.Tensor] = None, dwd: Optional[torch.Tensor] = None,
             want: Sequence[str] = GRADIENTS, workspace: Optional[Workspace] = None, stream=None):
    """(dxs, dwg, dwu, dwd): the gradients of xs and the weights from dys, that of
    train_forward()'s ys, with the activation and beta of that call.  An expert without
    rows has zeros for weight gradients.  ``want`` names those to compute (the others are
    None); they may be given to write into."""
    N, E, D, F, dev = _arguments(xs, offsets, wg, wu, wd)
    _expect(dys, "dys", (N, D), dev)
    _expect(g, "g", (N, F), dev)
    _expect(u, "u", (N, F), dev)
    if want is not GRADIENTS and set(want) - set(GRADIENTS):
        raise ValueError("want names %s, the gradients are %s" % (sorted(set(want) - set(GRADIENTS)), GRADIENTS))
    act, beta, _, _ = _variant(activation, beta, False, 0.0)
    outs = []
    for name, t, like in (("dxs", dxs, xs), ("dwg", dwg, wg), ("dwu", dwu, wu), ("dwd", dwd, wd)):
        if name in want:
            if t is None:
                t = _empty_like(like, stream)
            else:
                _expect(t, name, like.shape, dev)
        elif t is not None:
            raise ValueError("%s is given but not wanted" % name)
        outs.append(t)
    # The weight gradients of no rows are zeros, which a kernel writes.
    keep, ws, nbytes, path = _workspace(workspace, N, E, D, F, dev, 1, stream)
    _check(library().gmlp_experts_backward(_ptr(dys), _ptr(xs), offsets.data_ptr(), wg.data_ptr(), wu.data_ptr(),
                                           wd.data_ptr(), _ptr(g), _ptr(u), *[_ptr(t) for t in outs], N, E, D, F, act,
                                           beta, path, ws, nbytes, _stream(stream)))
    return tuple(outs)
