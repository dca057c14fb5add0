"""Python binding of routing in libgmlp.so (include/gmlp_route.h): tokens sorted by
expert and back, around :mod:`paper_2606_26344_amd.experts`.

Argument marshalling only.  Names mirror the C entry points:

    sort(ids, E)                               -> gmlp_route_sort     (offsets, slots)
    dispatch(x, slots)                         -> gmlp_route_dispatch         xs
    combine(ys, slots, weights)                -> gmlp_route_combine          y
    combine_backward(dy, ys, slots, weights)   -> gmlp_route_combine_backward (dys, dweights)
    dispatch_backward(dxs, slots)              -> gmlp_route_combine          dx

ids [T, k] are int32 or int64 (one that is not in 0 .. E - 1 is no expert), offsets
[E + 1] and slots [T, k] int32; expert e has rows offsets[e] .. offsets[e + 1] - 1 of the
sorted rows xs, ys [T k, D].  Rows x, y, xs, ys are ``torch.bfloat16``, weights [T, k]
``torch.float32`` or ``torch.bfloat16``.  All contiguous, on one HIP device.
"""
from __future__ import annotations

from typing import Optional, Sequence

import torch

from .gmlp import _check, _empty, _empty_like, _expect, _on_current, _ptr, _stream, library

BF16, IDS64 = 1, 2
GRADIENTS = ("dys", "dweights")

_INT32 = (torch.int32,)
_IDS = (torch.int32, torch.int64)
_WEIGHTS = (torch.float32, torch.bfloat16)


def _numbers(t, name, shape, device, dtypes) -> None:
    """Expects a tensor of one of the types."""
    if isinstance(t, torch.Tensor) and t.dtype in dtypes and t.device == device and t.shape == shape and t.is_contiguous():
        return
    if not isinstance(t, torch.Tensor) or t.dtype not in dtypes:
        raise TypeError("%s must be a tensor of %s" % (name, " or ".join(map(str, dtypes))))
    raise ValueError("%s must be contiguous, of shape %s, on the HIP device %s" % (name, tuple(shape), device))


def _choices(t, name, dtypes):
    """(T, k, device) of ids or slots."""
    if not isinstance(t, torch.Tensor) or t.dim() != 2:
        raise ValueError("%s must be a 2-D tensor" % name)
    if not t.is_cuda:
        raise ValueError("%s must be on a HIP device, got %s" % (name, t.device))
    dev = t.device
    _on_current(dev)
    _numbers(t, name, t.shape, dev, dtypes)
    return (*t.shape, dev)


def _new(like, shape, stream):
    """A new tensor of `like`'s type and device (_empty where a stream is given)."""
    return like.new_empty(shape) if stream is None else _empty(shape, like.dtype, like.device, stream)


def _slots(slots):
    return _choices(slots, "slots", _INT32)


def _width(t, name) -> int:
    if not isinstance(t, torch.Tensor) or t.dim() != 2:
        raise ValueError("%s must be a 2-D tensor" % name)
    return t.shape[1]


def sort(ids: torch.Tensor, experts: int, offsets: Optional[torch.Tensor] = None,
         slots: Optional[torch.Tensor] = None, stream=None):
    """(offsets, slots): where each expert's rows begin, and the row of every
    assignment, -1 for one without an expert.  Both may be given to write into."""
    T, k, dev = _choices(ids, "ids", _IDS)
    if offsets is None:
        offsets = _empty((max(int(experts), 0) + 1,), torch.int32, dev, stream)
    else:
        _numbers(offsets, "offsets", (experts + 1,), dev, _INT32)
    if slots is None:
        slots = _empty((T, k), torch.int32, dev, stream)
    else:
        _numbers(slots, "slots", (T, k), dev, _INT32)
    _check(library().gmlp_route_sort(_ptr(ids), offsets.data_ptr(), _ptr(slots), T, k, experts,
                                     IDS64 if ids.dtype is torch.int64 else 0, _stream(stream)))
    return offsets, slots


def dispatch(x: torch.Tensor, slots: torch.Tensor, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """xs [T k, D]: x's rows in their slots.  Rows behind the last expert's are not
    written.  ``out`` may be given to write into."""
    T, k, dev = _slots(slots)
    D = _width(x, "x")
    _expect(x, "x", (T, D), dev)
    if out is None:
        out = _new(x, (T * k, D), stream)
    else:
        _expect(out, "out", (T * k, D), dev)
    _check(library().gmlp_route_dispatch(_ptr(x), _ptr(slots), _ptr(out), T, k, D, _stream(stream)))
    return out


def combine(ys: torch.Tensor, slots: torch.Tensor, weights: Optional[torch.Tensor] = None,
            out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """y [T, D]: the sum of a token's rows of ys, times ``weights`` if given.  ``out``
    may be given to write into."""
    T, k, dev = _slots(slots)
    D = _width(ys, "ys")
    _expect(ys, "ys", (T * k, D), dev)
    if weights is not None:
        _numbers(weights, "weights", (T, k), dev, _WEIGHTS)
    if out is None:
        out = _new(ys, (T, D), stream)
    else:
        _expect(out, "out", (T, D), dev)
    flags = BF16 if weights is not None and weights.dtype is torch.bfloat16 else 0
    _check(library().gmlp_route_combine(_ptr(ys), _ptr(slots), _ptr(weights), _ptr(out), T, k, D, flags,
                                        _stream(stream)))
    return out


def dispatch_backward(dxs: torch.Tensor, slots: torch.Tensor, dx: Optional[torch.Tensor] = None,
                      stream=None) -> torch.Tensor:
    """dx [T, D] from dxs, the gradient of dispatch()'s xs."""
    return combine(dxs, slots, None, dx, stream)


def combine_backward(dy: torch.Tensor, ys: torch.Tensor, slots: torch.Tensor, weights: torch.Tensor,
                     dys: Optional[torch.Tensor] = None, dweights: Optional[torch.Tensor] = None,
                     want: Sequence[str] = GRADIENTS, stream=None):
    """(dys, dweights) from dy, the gradient of combine()'s y.  Rows of dys behind the
    last expert's are not written.  ``want`` names those to compute (the other is None);
    both may be given to write into, and ``dys`` may be ``ys``."""
    T, k, dev = _slots(slots)
    D = _width(dy, "dy")
    _expect(dy, "dy", (T, D), dev)
    _expect(ys, "ys", (T * k, D), dev)
    _numbers(weights, "weights", (T, k), dev, _WEIGHTS)
    if want is not GRADIENTS and set(want) - set(GRADIENTS):
        raise ValueError("want names %s, the gradients are %s" % (sorted(set(want) - set(GRADIENTS)), GRADIENTS))
    for name, t in (("dys", dys), ("dweights", dweights)):
        if t is not None and name not in want:
            raise ValueError("%s is given but not wanted" % name)
    if dys is not None:
        _expect(dys, "dys", (T * k, D), dev)
    elif "dys" in want:
        dys = _empty_like(ys, stream)
    if dweights is not None:
        _numbers(dweights, "dweights", (T, k), dev, (weights.dtype,))
    elif "dweights" in want:
        dweights = _empty_like(weights, stream)
    _check(library().gmlp_route_combine_backward(_ptr(dy), _ptr(ys), _ptr(slots), _ptr(weights), _ptr(dys),
                                                 _ptr(dweights), T, k, D,
                                                 BF16 if weights.dtype is torch.bfloat16 else 0, _stream(stream)))
    return dys, dweights
