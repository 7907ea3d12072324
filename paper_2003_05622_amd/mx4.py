"""Operators on frozen rows (include/hps_mx4.h): rows in microscaled 4-bit floating point, their scores against
queries of the same form, log probabilities over the scores, and the gradient of these.

    rows, found = table.get_mx4(keys)                   # a catalogue is frozen
    queries, rounded = mx4_quantize(pooled, values=True)
    got = mx4_logprobs(queries, rows, given=chosen, top=10, scale=8.0)
    d = mx4_logprobs_backward(queries, rows, chosen, d_logp, got.lse, scale=8.0)
    table.push(d)

Tensors are torch CUDA tensors on one GPU; work goes to that GPU's current stream.  Argument marshalling only; nothing is
kept between calls.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional

from .binding import EINVAL, HpsError, Mx4Operand, _check, _ptr, lib

MX4_MAX_TOP = 64


def _row_shape(dim: int):
    """(bytes of codes, bytes of scales) of a row."""
    if dim < 4 or dim > 1024 or dim % 4:
        raise HpsError(EINVAL, "dim %d" % dim)
    return (4 if dim <= 8 else 8 if dim <= 16 else (dim + 31) // 32 * 16), (dim + 31) // 32


class Mx4Rows:
    """Rows in the 4-bit form: codes uint8 [n, hps_mx4_row_bytes(dim)], scales uint8 [n, hps_mx4_row_scales(dim)]."""
    __slots__ = ("codes", "scales", "dim", "n")

    def __init__(self, codes, scales, dim: int):
        import torch
        n, shape = codes.shape[0], _row_shape(dim)
        if codes.dtype != torch.uint8 or scales.dtype != torch.uint8 or codes.shape != (n, shape[0]) or scales.shape != (n, shape[1]):
            raise ValueError("rows of dim %d: codes must be uint8 [n, %d] and scales uint8 [n, %d]" % ((dim,) + shape))
        if not (codes.is_contiguous() and scales.is_contiguous()):
            raise ValueError("codes and scales must be contiguous")
        if not codes.is_cuda or codes.device != scales.device:
            raise ValueError("codes and scales must be on one GPU")
        self.codes, self.scales, self.dim, self.n = codes, scales, dim, n

    @classmethod
    def empty(cls, n: int, dim: int, device) -> "Mx4Rows":
        import torch
        shape = _row_shape(dim)
        return cls(torch.empty((n, shape[0]), dtype=torch.uint8, device=device),
                   torch.empty((n, shape[1]), dtype=torch.uint8, device=device), dim)

    @property
    def device(self):
        return self.codes.device

    def __getitem__(self, part: slice) -> "Mx4Rows":
        """A range of the rows, in place."""
        if not isinstance(part, slice):
            raise TypeError("rows are taken by ranges")
        return Mx4Rows(self.codes[part], self.scales[part], self.dim)

    def _operand(self) -> Mx4Operand:
        return Mx4Operand(self.codes.data_ptr(), self.scales.data_ptr(), self.n)

    def dequantize(self):
        """The values that the rows stand for, float32 [n, dim]."""
        import torch
        out = torch.empty((self.n, self.dim), dtype=torch.float32, device=self.device)
        with _On(self.device) as stream:
            _check(lib().hps_mx4_dequantize(ctypes.byref(self._operand()), self.dim, _ptr(out), stream), "hps_mx4_dequantize")
        return out


class _On:
    """Makes a tensor's GPU the current one for a call; gives the current stream there."""
    __slots__ = ("device", "before")

    def __init__(self, device):
        self.device = device.index

    def __enter__(self):
        from torch._C import _cuda_getCurrentRawStream, _cuda_getDevice
        self.before = _cuda_getDevice()
        if self.before != self.device:
            import torch
            torch.cuda.set_device(self.device)
        return _cuda_getCurrentRawStream(self.device)

    def __exit__(self, *_):
        if self.before != self.device:
            import torch
            torch.cuda.set_device(self.before)


class LogProbs(NamedTuple):
    """What mx4_logprobs gives; logp / top_* are None where nothing of the kind was asked for."""
    lse: "torch.Tensor"                      # noqa: F821
    entropy: "torch.Tensor"                  # noqa: F821
    logp: Optional["torch.Tensor"]           # noqa: F821
    top_index: Optional["torch.Tensor"]      # noqa: F821
    top_logp: Optional["torch.Tensor"]       # noqa: F821


def _array(t, name: str, dtype, shape, device):
    """A contiguous tensor of this type, shape and GPU (None stays None)."""
    if t is None:
        return
    if t.dtype != dtype or tuple(t.shape) != shape or not t.is_contiguous() or t.device != device:
        raise ValueError("%s must be a contiguous %s tensor of shape %s on %s" % (name, dtype, shape, device))


def _pair(queries: Mx4Rows, rows: Mx4Rows, bias):
    if queries.dim != rows.dim:
        raise ValueError("queries of dim %d and rows of dim %d" % (queries.dim, rows.dim))
    if queries.device != rows.device:
        raise ValueError("queries and rows must be on one GPU")
    if bias is not None:
        import torch
        _array(bias, "bias", torch.float32, (rows.n,), rows.device)


def mx4_quantize(x, values: bool = False):
    """Mx4Rows of x [n, dim] (float32 or bfloat16; its rows may lie apart); with values=True also the values they stand
    for, float32 [n, dim]."""
    import torch
    if x.dim() != 2 or x.dtype not in (torch.float32, torch.bfloat16) or not x.is_cuda:
        raise ValueError("x must be a float32 or bfloat16 CUDA tensor [n, dim]")
    n, dim = x.shape
    if x.stride(1) != 1 and n and dim > 1:
        raise ValueError("the values of a row must lie next to each other")
    stride = x.stride(0) if n > 1 else dim
    rows = Mx4Rows.empty(n, dim, x.device)
    rounded = torch.empty((n, dim), dtype=torch.float32, device=x.device) if values else None
    with _On(x.device) as stream:
        _check(lib().hps_mx4_quantize(_ptr(x), 1 if x.dtype == torch.bfloat16 else 0, n, dim, stride, _ptr(rows.codes),
                                      _ptr(rows.scales), _ptr(rounded), stream), "hps_mx4_quantize")
    return (rows, rounded) if values else rows


def mx4_scores(queries: Mx4Rows, rows: Mx4Rows, scale: float = 1.0, bias=None, dtype=None, out=None):
    """scale * <query, row> + bias of every query and row: [queries, rows], float32 or bfloat16 (`out`: written there)."""
    import torch
    _pair(queries, rows, bias)
    if out is None:
        out = torch.empty((queries.n, rows.n), dtype=dtype or torch.float32, device=rows.device)
    elif dtype is not None and dtype != out.dtype:
        raise ValueError("out is not of the type asked for")
    if out.dtype not in (torch.float32, torch.bfloat16) or tuple(out.shape) != (queries.n, rows.n) or out.device != rows.device:
        raise ValueError("the scores are float32 or bfloat16 [queries, rows], on the rows' GPU")
    if out.stride(1) != 1 and rows.n > 1 and queries.n:
        raise ValueError("the scores of a query must lie next to each other")
    stride = out.stride(0) if queries.n > 1 else rows.n
    with _On(rows.device) as stream:
        _check(lib().hps_mx4_scores(ctypes.byref(queries._operand()), ctypes.byref(rows._operand()), rows.dim, scale, _ptr(bias),
                                    _ptr(out), 1 if out.dtype == torch.bfloat16 else 0, stride, stream), "hps_mx4_scores")
    return out


def mx4_logprobs(queries: Mx4Rows, rows: Mx4Rows, given=None, top: int = 0, scale: float = 1.0, bias=None) -> LogProbs:
    """Log-sum-exp and entropy of each query's scores; log probabilities of the given rows (int32 [queries, g]); the `top`
    best rows (int32 numbers and log probabilities, best first)."""
    import torch
    _pair(queries, rows, bias)
    m, device, g = queries.n, rows.device, 0
    if top < 0 or top > MX4_MAX_TOP:
        raise HpsError(EINVAL, "top %d" % top)
    if given is not None:
        if given.dim() != 2:
            raise ValueError("given must be [queries, g]")
        g = given.shape[1]
        _array(given, "given", torch.int32, (m, g), device)
    lse, entropy = torch.empty((2, m), dtype=torch.float32, device=device)
    logp = torch.empty((m, g), dtype=torch.float32, device=device) if given is not None else None
    index = torch.empty((m, top), dtype=torch.int32, device=device) if top else None
    best = torch.empty((m, top), dtype=torch.float32, device=device) if top else None
    size = lib().hps_mx4_logprobs_bytes(m, rows.n, rows.dim, top)
    space = torch.empty(size, dtype=torch.uint8, device=device)
    with _On(device) as stream:
        _check(lib().hps_mx4_logprobs(ctypes.byref(queries._operand()), ctypes.byref(rows._operand()), rows.dim, scale, _ptr(bias),
                                      _ptr(given), g, top, _ptr(lse), _ptr(entropy), _ptr(logp), _ptr(index), _ptr(best), _ptr(space),
                                      size, stream), "hps_mx4_logprobs")
    return LogProbs(lse, entropy, logp, index, best)


def mx4_logprobs_backward(queries: Mx4Rows, rows: Mx4Rows, given, d_logp, lse, entropy=None, d_entropy=None, scale: float = 1.0,
                          bias=None):
    """The gradient of sum(d_logp * logp) + sum(d_entropy * entropy) with respect to the values that the queries stand
    for, float32 [queries, dim].  lse, entropy: of mx4_logprobs, for the same arguments."""
    import torch
    _pair(queries, rows, bias)
    m, device, g = queries.n, rows.device, 0
    if (given is None) != (d_logp is None):
        raise ValueError("given rows and their gradients come together")
    if given is not None:
        if given.dim() != 2:
            raise ValueError("given must be [queries, g]")
        g = given.shape[1]
        _array(given, "given", torch.int32, (m, g), device)
        _array(d_logp, "d_logp", torch.float32, (m, g), device)
    if d_entropy is not None and entropy is None:
        raise ValueError("a gradient of the entropy needs the entropy")
    for name, t in (("lse", lse), ("entropy", entropy), ("d_entropy", d_entropy)):
        _array(t, name, torch.float32, (m,), device)
    out = torch.empty((m, rows.dim), dtype=torch.float32, device=device)
    size = lib().hps_mx4_logprobs_backward_bytes(m, rows.n, rows.dim)
    space = torch.empty(size, dtype=torch.uint8, device=device)
    with _On(device) as stream:
        _check(lib().hps_mx4_logprobs_backward(ctypes.byref(queries._operand()), ctypes.byref(rows._operand()), rows.dim, scale,
                                               _ptr(bias), _ptr(lse), _ptr(entropy), _ptr(given), _ptr(d_logp), g, _ptr(d_entropy),
                                               _ptr(out), _ptr(space), size, stream), "hps_mx4_logprobs_backward")
    return out
