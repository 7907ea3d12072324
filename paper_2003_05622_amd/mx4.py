"""Operators on frozen rows (include/hps_mx4.h): rows in microscaled 4-bit floating point, their scores against
queries of the same form, log probabilities over the scores, and the gradient of these.

    rows, found = table.get_mx4(keys)                   # a catalogue is frozen
    queries, rounded = mx4_quantize(pooled, values=True)
    got = mx4_logprobs(queries, rows, given=chosen, top=10, scale=8.0)
    d = mx4_logprobs_backward(queries, rows, chosen, d_logp, got.lse, scale=8.0)
    table.push(d)

Tensors are torch CUDA tensors on one GPU; work goes to that GPU's current stream.  Argument marshalling only; nothing is
kept between calls.  Results are no part of autograd's graph, whatever the arguments are: gradients are asked for by
mx4_logprobs_backward, and go on into push() as above (quantising counts as the identity).
"""
from __future__ import annotations

import ctypes
import functools
from typing import NamedTuple, Optional

from .binding import EINVAL, OK, HpsError, Mx4Operand, _ptr, lib

MX4_MAX_TOP = 64


@functools.lru_cache(maxsize=None)
def _row_shape(dim: int):
    """(bytes of codes, bytes of scales) of a row."""
    if dim < 4 or dim > 1024 or dim % 4:
        raise HpsError(EINVAL, "dim %d" % dim)
    return (4 if dim <= 8 else 8 if dim <= 16 else (dim + 31) // 32 * 16), (dim + 31) // 32


class Mx4Rows:
    """Rows in the 4-bit form: codes uint8 [n, hps_mx4_row_bytes(dim)], scales uint8 [n, hps_mx4_row_scales(dim)]."""
    __slots__ = ("codes", "scales", "dim", "n", "device")

    def __init__(self, codes, scales, dim: int):
        import torch
        n, shape = codes.shape[0], _row_shape(dim)
        if codes.dtype is not torch.uint8 or scales.dtype is not torch.uint8 or codes.shape != (n, shape[0]) or scales.shape != (n, shape[1]):
            raise ValueError("rows of dim %d: codes must be uint8 [n, %d] and scales uint8 [n, %d]" % ((dim,) + shape))
        if not (codes.is_contiguous() and scales.is_contiguous()):
            raise ValueError("codes and scales must be contiguous")
        if codes.get_device() < 0 or scales.get_device() != codes.get_device():
            raise ValueError("codes and scales must be on one GPU")
        self.codes, self.scales, self.dim, self.n, self.device = codes, scales, dim, n, codes.device

    @classmethod
    def empty(cls, n: int, dim: int, device) -> "Mx4Rows":
        """Rows to be written."""
        import torch
        shape = _row_shape(dim)
        rows = cls.__new__(cls)
        rows.codes = torch.empty((n, shape[0]), dtype=torch.uint8, device=device)
        rows.scales = torch.empty((n, shape[1]), dtype=torch.uint8, device=device)
        rows.dim, rows.n, rows.device = dim, n, rows.codes.device
        return rows

    def __getitem__(self, part: slice) -> "Mx4Rows":
        """A range of the rows, in place."""
        if not isinstance(part, slice):
            raise TypeError("rows are taken by ranges")
        return Mx4Rows(self.codes[part], self.scales[part], self.dim)

    def _operand(self):
        return ctypes.byref(Mx4Operand(self.codes.data_ptr(), self.scales.data_ptr(), self.n))

    def dequantize(self):
        """The values that the rows stand for, float32 [n, dim]."""
        import torch
        out = torch.empty((self.n, self.dim), dtype=torch.float32, device=self.device)
        _call("hps_mx4_dequantize", self.device, self._operand(), self.dim, out.data_ptr())
        return out


@functools.lru_cache(maxsize=256)
def _space(name: str, *sizes) -> int:
    """Bytes of workspace a call of these sizes needs."""
    return getattr(lib(), name)(*sizes)


def _call(name: str, device, *args) -> None:
    """Calls an entry point with `device` the current GPU, on its current stream."""
    import torch
    fn, index = getattr(lib(), name), device.index
    if torch._C._cuda_getDevice() == index:
        status = fn(*args, torch._C._cuda_getCurrentRawStream(index))
    else:
        with torch.cuda.device(index):
            status = fn(*args, torch._C._cuda_getCurrentRawStream(index))
    if status != OK:
        raise HpsError(status, name)


class LogProbs(NamedTuple):
    """What mx4_logprobs gives; logp / top_* are None where nothing of the kind was asked for."""
    lse: "torch.Tensor"                      # noqa: F821
    entropy: "torch.Tensor"                  # noqa: F821
    logp: Optional["torch.Tensor"]           # noqa: F821
    top_index: Optional["torch.Tensor"]      # noqa: F821
    top_logp: Optional["torch.Tensor"]       # noqa: F821


def _array(t, name: str, dtype, shape, device):
    """Address of a contiguous tensor of this type, shape and GPU (None stays None)."""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous() or t.get_device() != device.index:
        raise ValueError("%s must be a contiguous %s tensor of shape %s on %s" % (name, dtype, tuple(shape), device))
    return t.data_ptr()


def _pair(queries: Mx4Rows, rows: Mx4Rows):
    if queries.dim != rows.dim:
        raise ValueError("queries of dim %d and rows of dim %d" % (queries.dim, rows.dim))
    if queries.device != rows.device:
        raise ValueError("queries and rows must be on one GPU")


def _given(given, m: int, device):
    """(address, how many a query)"""
    if given is None:
        return None, 0
    import torch
    if given.dim() != 2:
        raise ValueError("given must be [queries, g]")
    g = given.shape[1]
    return _array(given, "given", torch.int32, (m, g), device), g


def mx4_quantize(x, values: bool = False):
    """Mx4Rows of x [n, dim] (float32 or bfloat16; its rows may lie apart); with values=True also the values they stand
    for, float32 [n, dim]."""
    import torch
    dtype = x.dtype
    if x.dim() != 2 or (dtype is not torch.float32 and dtype is not torch.bfloat16) or not x.is_cuda:
        raise ValueError("x must be a float32 or bfloat16 CUDA tensor [n, dim]")
    n, dim = x.shape
    apart, step = x.stride()
    if step != 1 and n and dim > 1:
        raise ValueError("the values of a row must lie next to each other")
    rows = Mx4Rows.empty(n, dim, x.device)
    rounded = torch.empty((n, dim), dtype=torch.float32, device=rows.device) if values else None
    _call("hps_mx4_quantize", rows.device, x.data_ptr(), 0 if dtype is torch.float32 else 1, n, dim, apart if n > 1 else dim,
          rows.codes.data_ptr(), rows.scales.data_ptr(), rounded.data_ptr() if values else None)
    return (rows, rounded) if values else rows


def mx4_scores(queries: Mx4Rows, rows: Mx4Rows, scale: float = 1.0, bias=None, dtype=None, out=None):
    """scale * <query, row> + bias of every query and row: [queries, rows], float32 or bfloat16 (`out`: written there)."""
    import torch
    _pair(queries, rows)
    m, n, device = queries.n, rows.n, rows.device
    if out is None:
        out = torch.empty((m, n), dtype=dtype or torch.float32, device=device)
    elif dtype is not None and dtype != out.dtype:
        raise ValueError("out is not of the type asked for")
    if (out.dtype is not torch.float32 and out.dtype is not torch.bfloat16) or out.shape != (m, n) or out.device != device:
        raise ValueError("the scores are float32 or bfloat16 [queries, rows], on the rows' GPU")
    apart, step = out.stride()
    if step != 1 and n > 1 and m:
        raise ValueError("the scores of a query must lie next to each other")
    _call("hps_mx4_scores", device, queries._operand(), rows._operand(), rows.dim, scale, _array(bias, "bias", torch.float32, (n,), device),
          out.data_ptr(), 0 if out.dtype is torch.float32 else 1, apart if m > 1 else n)
    return out


def mx4_logprobs(queries: Mx4Rows, rows: Mx4Rows, given=None, top: int = 0, scale: float = 1.0, bias=None) -> LogProbs:
    """Log-sum-exp and entropy of each query's scores; log probabilities of the given rows (int32 [queries, g]); the `top`
    best rows (int32 numbers and log probabilities, best first)."""
    import torch
    _pair(queries, rows)
    m, n, dim, device = queries.n, rows.n, rows.dim, rows.device
    if top < 0 or top > MX4_MAX_TOP:
        raise HpsError(EINVAL, "top %d" % top)
    asked, g = _given(given, m, device)
    lse, entropy = torch.empty(m, dtype=torch.float32, device=device), torch.empty(m, dtype=torch.float32, device=device)
    logp = torch.empty((m, g), dtype=torch.float32, device=device) if given is not None else None
    index = torch.empty((m, top), dtype=torch.int32, device=device) if top else None
    best = torch.empty((m, top), dtype=torch.float32, device=device) if top else None
    size = _space("hps_mx4_logprobs_bytes", m, n, dim, top)
    space = torch.empty(size, dtype=torch.uint8, device=device)
    _call("hps_mx4_logprobs", device, queries._operand(), rows._operand(), dim, scale, _array(bias, "bias", torch.float32, (n,), device), asked,
          g, top, lse.data_ptr(), entropy.data_ptr(), _ptr(logp), _ptr(index), _ptr(best), space.data_ptr(), size)
    return LogProbs(lse, entropy, logp, index, best)


def mx4_logprobs_backward(queries: Mx4Rows, rows: Mx4Rows, given, d_logp, lse, entropy=None, d_entropy=None, scale: float = 1.0,
                          bias=None):
    """The gradient of sum(d_logp * logp) + sum(d_entropy * entropy) with respect to the values that the queries stand
    for, float32 [queries, dim].  lse, entropy: of mx4_logprobs, for the same arguments."""
    import torch
    _pair(queries, rows)
    m, n, dim, device = queries.n, rows.n, rows.dim, rows.device
    if (given is None) != (d_logp is None):
        raise ValueError("given rows and their gradients come together")
    asked, g = _given(given, m, device)
    if d_entropy is not None and entropy is None:
        raise ValueError("a gradient of the entropy needs the entropy")
    if lse is None:
        raise ValueError("lse of mx4_logprobs is needed")
    args = (_array(bias, "bias", torch.float32, (n,), device), _array(lse, "lse", torch.float32, (m,), device),
            _array(entropy, "entropy", torch.float32, (m,), device), asked, _array(d_logp, "d_logp", torch.float32, (m, g), device), g,
            _array(d_entropy, "d_entropy", torch.float32, (m,), device))
    out = torch.empty((m, dim), dtype=torch.float32, device=device)
    size = _space("hps_mx4_logprobs_backward_bytes", m, n, dim)
    space = torch.empty(size, dtype=torch.uint8, device=device)
    _call("hps_mx4_logprobs_backward", device, queries._operand(), rows._operand(), dim, scale, *args, out.data_ptr(), space.data_ptr(),
          size)
    return out
