"""Python binding of the products with 4-bit weights in libgmlp.so
(include/gmlp_w4.h).

Argument marshalling only.  Names mirror the C entry points:

    quantize(w, group, zeros)   -> gmlp_w4_quantize    (q, scales, zero points)
    pack(q, scales, zeros)      -> gmlp_w4_pack        a Weight for the products
    from_weight(w, group)       quantize, then pack
    dequantize(weight)          -> gmlp_w4_dequantize
    matmul(x, weight)           -> gmlp_w4_matmul      y = x w
    gate_up(x, wg, wu)          -> gmlp_w4_gate_up     h = act(x wg) * (x wu)
    forward(x, wg, wu, wd)      -> gmlp_w4_forward     the whole MLP

w[k, n] = (q[k, n] - zeros[k // group, n]) * scales[k // group, n], zeros 8 if not
given.  Activations, scales and results are ``torch.bfloat16``, q and zeros
``torch.uint8`` of 0..15; at most MAX_TOKENS rows of x.
"""
from __future__ import annotations

from typing import Optional

import torch

from .gmlp import (_CALL_DEVICE, FRESH_WORKSPACE, PATH_AUTO, Workspace, _check, _empty, _expect, _on_current, _prepared,
                   _ptr, _scratch, _stream, _variant, library)

MAX_TOKENS = 64


class Weight:
    """A packed 4-bit weight [K, N]; ``buffer`` holds it, 256-byte aligned."""

    def __init__(self, K: int, N: int, group: int, zeros: bool, device, stream=None):
        n = int(library().gmlp_w4_packed_size(K, N, group, int(zeros)))
        if n == 0:
            raise ValueError("invalid 4-bit weight K=%d N=%d group=%d" % (K, N, group))
        self.K, self.N, self.group, self.zeros = K, N, group, bool(zeros)
        self.storage = _empty((n + 256,), torch.uint8, device, stream)
        off = (-self.storage.data_ptr()) % 256
        self.buffer = self.storage[off:off + n]
        self.device = self.buffer.device


def workspace_size(T: int, D: int, F: int) -> int:
    return int(library().gmlp_w4_workspace_size(T, D, F))


def make_workspace(T: int, D: int, F: int, device=None, stream=None) -> Workspace:
    """A prepared workspace for forward() and gate_up() with weights [D, F] and
    for matmul() with weights [D, F] or [F, D]."""
    return Workspace(T, D, F, device=device, stream=stream, size=workspace_size)


def _expect_bytes(t, name, shape, device) -> None:
    if (not isinstance(t, torch.Tensor) or t.dtype is not torch.uint8 or t.device != device
            or tuple(t.shape) != tuple(shape) or not t.is_contiguous()):
        raise ValueError("%s must be a contiguous uint8 tensor of shape %s on %s" % (name, tuple(shape), device))


def quantize(w: torch.Tensor, group: int = 128, zeros: bool = False, stream=None):
    """(q, scales, zeros) of a bf16 weight [K, N], rounded to nearest group by
    group; zeros is None unless asked for."""
    if w.dim() != 2:
        raise ValueError("w must be 2-D")
    K, N = w.shape
    dev = w.device
    _expect(w, "w", (K, N), dev)
    _on_current(dev)
    groups = -(-K // max(group, 1))
    q = _empty((K, N), torch.uint8, dev, stream)
    s = _empty((groups, N), torch.bfloat16, dev, stream)
    z = _empty((groups, N), torch.uint8, dev, stream) if zeros else None
    _check(library().gmlp_w4_quantize(w.data_ptr(), q.data_ptr(), s.data_ptr(), _ptr(z), K, N, group, _stream(stream)))
    return q, s, z


def pack(q: torch.Tensor, scales: torch.Tensor, zeros: Optional[torch.Tensor] = None, group: int = 128,
         stream=None) -> Weight:
    """Lay a weight out for the products, once."""
    if q.dim() != 2:
        raise ValueError("q must be 2-D")
    K, N = q.shape
    dev = q.device
    if dev.type != "cuda":
        raise ValueError("q must be on a HIP device, got %s" % dev)
    _on_current(dev)
    shape = (-(-K // max(group, 1)), N)
    _expect_bytes(q, "q", (K, N), dev)
    _expect(scales, "scales", shape, dev)
    if zeros is not None:
        _expect_bytes(zeros, "zeros", shape, dev)
    w = Weight(K, N, group, zeros is not None, dev, stream)
    _check(library().gmlp_w4_pack(q.data_ptr(), scales.data_ptr(), _ptr(zeros), w.buffer.data_ptr(), K, N, group,
                                  _stream(stream)))
    return w


def from_weight(w: torch.Tensor, group: int = 128, zeros: bool = False, stream=None) -> Weight:
    """quantize(), then pack()."""
    return pack(*quantize(w, group, zeros, stream), group=group, stream=stream)


def dequantize(w: Weight, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """bf16((q - zeros) * scales) [K, N], for example for the entry points of
    :mod:`paper_2606_26344_amd.gmlp` with many tokens."""
    _on_current(w.device)
    if out is None:
        out = _empty((w.K, w.N), torch.bfloat16, w.device, stream)
    else:
        _expect(out, "out", (w.K, w.N), w.device)
    _check(library().gmlp_w4_dequantize(w.buffer.data_ptr(), out.data_ptr(), w.K, w.N, w.group, int(w.zeros),
                                        _stream(stream)))
    return out


def _workspace(workspace, T, D, F, device, stream):
    """(tensor to keep, address, bytes, path) of a call's workspace."""
    if workspace is not None:
        return None, *_prepared(workspace, device), PATH_AUTO
    n = workspace_size(T, D, F)
    if n == 0 and T > MAX_TOKENS:  # refused by the library, with its reason
        return None, None, 0, PATH_AUTO
    keep, ws = _scratch(n, T, _CALL_DEVICE, stream, False, "invalid shape T=%d D=%d F=%d" % (T, D, F))
    return keep, ws, n, PATH_AUTO | FRESH_WORKSPACE


def _expect_weight(w, name, K, N, like, device) -> None:
    if not isinstance(w, Weight):
        raise TypeError("%s must be a packed 4-bit Weight" % name)
    if (w.K, w.N) != (K, N):
        raise ValueError("%s is [%d, %d], expected [%d, %d]" % (name, w.K, w.N, K, N))
    if (w.group, w.zeros) != (like.group, like.zeros):
        raise ValueError("%s has another group size or kind than the first weight" % name)
    if w.device != device:
        raise ValueError("%s must be on %s, got %s" % (name, device, w.device))


def _first(x, w, name):
    """(T, K, device) of a call's x and its first weight."""
    if not isinstance(w, Weight):
        raise TypeError("%s must be a packed 4-bit Weight" % name)
    if x.dim() != 2:
        raise ValueError("x must be 2-D")
    T, dev = x.shape[0], x.device
    _expect(x, "x", (T, w.K), dev)
    _expect_weight(w, name, w.K, w.N, w, dev)
    _on_current(dev)
    return T, dev


def _output(out, T, N, dev, stream):
    if out is None:
        return _empty((T, N), torch.bfloat16, dev, stream)
    _expect(out, "out", (T, N), dev)
    return out


def matmul(x: torch.Tensor, w: Weight, out: Optional[torch.Tensor] = None, workspace: Optional[Workspace] = None,
           stream=None) -> torch.Tensor:
    """y = x w, x [T, K]."""
    T, dev = _first(x, w, "w")
    out = _output(out, T, w.N, dev, stream)
    keep, ws, nbytes, path = _workspace(workspace, T, w.K, w.N, dev, stream)
    _check(library().gmlp_w4_matmul(x.data_ptr(), w.buffer.data_ptr(), out.data_ptr(), T, w.K, w.N, w.group,
                                    int(w.zeros), path, ws, nbytes, _stream(stream)))
    return out


def gate_up(x: torch.Tensor, wg: Weight, wu: Weight, out: Optional[torch.Tensor] = None, activation: str = "silu",
            beta: float = 1.0, workspace: Optional[Workspace] = None, stream=None) -> torch.Tensor:
    """h = bf16(act(x wg) * (x wu)); wg and wu of one group size and kind."""
    T, dev = _first(x, wg, "wg")
    _expect_weight(wu, "wu", wg.K, wg.N, wg, dev)
    act, beta, _, _ = _variant(activation, beta, False, 0.0)
    out = _output(out, T, wg.N, dev, stream)
    keep, ws, nbytes, path = _workspace(workspace, T, wg.K, wg.N, dev, stream)
    _check(library().gmlp_w4_gate_up(x.data_ptr(), wg.buffer.data_ptr(), wu.buffer.data_ptr(), out.data_ptr(), T, wg.K,
                                     wg.N, wg.group, int(wg.zeros), act, beta, path, ws, nbytes, _stream(stream)))
    return out


def forward(x: torch.Tensor, wg: Weight, wu: Weight, wd: Weight, out: Optional[torch.Tensor] = None,
            activation: str = "silu", beta: float = 1.0, workspace: Optional[Workspace] = None,
            stream=None) -> torch.Tensor:
    """y = (act(x wg) * (x wu)) wd; the three weights of one group size and kind."""
    T, dev = _first(x, wg, "wg")
    D, F = wg.K, wg.N
    _expect_weight(wu, "wu", D, F, wg, dev)
    _expect_weight(wd, "wd", F, D, wg, dev)
    act, beta, _, _ = _variant(activation, beta, False, 0.0)
    out = _output(out, T, D, dev, stream)
    keep, ws, nbytes, path = _workspace(workspace, T, D, F, dev, stream)
    _check(library().gmlp_w4_forward(x.data_ptr(), wg.buffer.data_ptr(), wu.buffer.data_ptr(), wd.buffer.data_ptr(),
                                     out.data_ptr(), T, D, F, wg.group, int(wg.zeros), act, beta, path, ws, nbytes,
                                     _stream(stream)))
    return out
