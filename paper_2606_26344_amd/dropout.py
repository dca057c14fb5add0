"""Python binding of dropout in libgmlp.so (include/gmlp_dropout.h).

Argument marshalling only.  Names mirror the C entry points:

    forward(x, p, seed, ...)       -> gmlp_dropout           out = res + kept x / (1 - p)
    backward(dout, p, seed, ...)   -> gmlp_dropout_backward  dx = kept dout / (1 - p)
    counters(T, D)                 counters that a call takes

x and dx [T, D] are ``torch.bfloat16``; the residual stream, res and out (or dout),
``torch.bfloat16`` or ``torch.float32``.  All contiguous, on one HIP device.  The mask is
a function of (seed, offset + position) and an element's place, made again by
backward(); ``position`` is an int64 tensor of one element on the device, which a
program that replays captured calls moves on between replays.
"""
from __future__ import annotations

from typing import Optional

import torch

from .block_norm import _stream_tensor
from .gmlp import _check, _empty, _empty_like, _expect, _on_current, _ptr, _stream, library

FP32 = 1


def counters(T: int, D: int) -> int:
    """How far a call on [T, D] moves the offset for the next."""
    return T * D // 8


def _number(value, name) -> int:
    if not isinstance(value, int) or not 0 <= value < 1 << 64:
        raise ValueError("%s must be an int in 0 .. 2^64 - 1, got %r" % (name, value))
    return value


def _mask(p, seed, offset, position, device):
    """The arguments that name a mask."""
    if position is not None and (not isinstance(position, torch.Tensor) or position.dtype is not torch.int64
                                 or position.numel() != 1 or position.device != device):
        raise ValueError("position must be an int64 tensor of one element on %s" % device)
    return float(p), _number(seed, "seed"), _number(offset, "offset"), _ptr(position)


def _like(t, name):
    """(T, D, device) of the tensor that a call is about."""
    if not isinstance(t, torch.Tensor) or t.dim() != 2:
        raise ValueError("%s must be a 2-D tensor" % name)
    if t.device.type != "cuda":
        raise ValueError("%s must be on a HIP device, got %s" % (name, t.device))
    _on_current(t.device)
    return (*t.shape, t.device)


def forward(x: torch.Tensor, p: float, seed: int, offset: int = 0, res: Optional[torch.Tensor] = None,
            position: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """out, of res's type (without one bfloat16).  ``out`` may be given to write into
    and may be ``res``, or ``x`` where it is bfloat16."""
    T, D, dev = _like(x, "x")
    _expect(x, "x", (T, D), dev)
    if res is not None:
        if not isinstance(res, torch.Tensor) or res.dtype not in (torch.bfloat16, torch.float32):
            raise TypeError("res must be a torch.bfloat16 or torch.float32 tensor")
        _stream_tensor(res, "res", (T, D), dev, res.dtype)
    like = x if res is None else res
    if out is None:
        out = _empty_like(like, stream)
    else:
        _stream_tensor(out, "out", (T, D), dev, like.dtype)
    mask = _mask(p, seed, offset, position, dev)
    _check(library().gmlp_dropout(x.data_ptr(), _ptr(res), out.data_ptr(), T, D, *mask,
                                  FP32 if like.dtype is torch.float32 else 0, _stream(stream)))
    return out


def backward(dout: torch.Tensor, p: float, seed: int, offset: int = 0, position: Optional[torch.Tensor] = None,
             dx: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """dx (bfloat16) from dout, the gradient of forward()'s out, with the numbers of that
    call; res's gradient is dout.  ``dx`` may be given to write into and may be a
    bfloat16 ``dout``."""
    T, D, dev = _like(dout, "dout")
    if dout.dtype not in (torch.bfloat16, torch.float32):
        raise TypeError("dout must be torch.bfloat16 or torch.float32, got %s" % dout.dtype)
    _stream_tensor(dout, "dout", (T, D), dev, dout.dtype)
    if dx is not None:
        _expect(dx, "dx", (T, D), dev)
    else:
        dx = _empty((T, D), torch.bfloat16, dev, stream)
    mask = _mask(p, seed, offset, position, dev)
    _check(library().gmlp_dropout_backward(dout.data_ptr(), dx.data_ptr(), T, D, *mask,
                                           FP32 if dout.dtype is torch.float32 else 0, _stream(stream)))
    return dx
