"""Operators of a path's inner phase on torch CUDA tensors (declared in ``include/dipaco.h``).

Layer norm with its gradient, matrices packed in 8 bits (activation checkpoints and the operands of
the products), the GELU that writes and reads such checkpoints, and the product of packed matrices
on the tensor cores.  Each function allocates its results (and workspace) with torch, launches on the
current stream of the tensors' device, and raises ``ValueError`` for shapes and dtypes that do not
fit together or ``binding.DipacoError`` with the library's status.  There is no CPU path.

Autograd records nothing of these calls: the gradients are calls of their own.  A tensor that requires a
gradient is refused while gradients are being recorded; inside ``torch.no_grad()`` or a
``torch.autograd.Function``, or detached, it is taken.
"""
from __future__ import annotations

from typing import Optional, Tuple, Union

import torch

from . import binding as B

BLOCK = 128  # one scale per BLOCK x BLOCK values
_F32, _E4M3, _E8M0 = torch.float32, torch.float8_e4m3fn, torch.float8_e8m0fnu
_CODES = {torch.float32: B.DIPACO_F32, torch.bfloat16: B.DIPACO_BF16}
_stream = torch._C._cuda_getCurrentRawStream  # of a device index


class Packed:
    """A matrix in 8 bits: ``codes`` [rows, cols] float8_e4m3fn, row stride a multiple of 16, and
    ``scales`` [ceil(rows/128), ceil(cols/128)] float8_e8m0fnu, contiguous; value = code * scale.

    The tensors cannot be exchanged for others: ``struct`` holds the addresses of their data, which has to
    stay where it is.  Copies (``copy``, ``pickle``) are built anew from their own tensors."""

    __slots__ = ("_codes", "_scales", "_struct")

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor):
        rows, cols = codes.shape
        stride, unit = codes.stride()
        if codes.dtype != _E4M3 or scales.dtype != _E8M0:
            raise ValueError("codes must be float8_e4m3fn and scales float8_e8m0fnu")
        if scales.shape != ((rows + 127) >> 7, (cols + 127) >> 7) or not scales.is_contiguous():
            raise ValueError("scales must be contiguous with one entry per block of 128 x 128")
        if unit != 1 and cols > 1:
            raise ValueError("codes must be row-major")
        if rows == 1:
            stride = (cols + 15) & ~15
        if not codes.is_cuda or scales.get_device() != codes.get_device():
            raise ValueError("codes and scales must be on one CUDA device")
        if codes.requires_grad or scales.requires_grad:
            _refuse_gradient("codes or scales")
        self._codes, self._scales = codes, scales
        self._struct = B.PackedStruct(codes.data_ptr(), scales.data_ptr(), rows, cols, stride)

    def __reduce__(self):  # as bytes: torch does not pickle e8m0
        return _packed_of_bytes, (self._codes.view(torch.uint8), self._scales.view(torch.uint8))

    @property
    def codes(self) -> torch.Tensor:
        return self._codes

    @property
    def scales(self) -> torch.Tensor:
        return self._scales

    @property
    def struct(self) -> B.PackedStruct:
        return self._struct

    @classmethod
    def empty(cls, rows: int, cols: int, device) -> "Packed":
        """A packed matrix with nothing in it yet."""
        return _packed_beside(torch.empty(0, device=device), rows, cols)

    @property
    def shape(self) -> Tuple[int, int]:
        return self._struct.rows, self._struct.cols

    @property
    def device(self) -> torch.device:
        return self._codes.device


def _packed_of_bytes(codes: torch.Tensor, scales: torch.Tensor) -> Packed:
    return Packed(codes.view(_E4M3), scales.view(_E8M0))


def _packed_beside(x: torch.Tensor, rows: int, cols: int) -> Packed:
    """An empty packed matrix on x's device."""
    stride = (cols + 15) & ~15
    codes = x.new_empty((rows, stride), dtype=_E4M3)
    scales = x.new_empty(((rows + 127) >> 7, (cols + 127) >> 7), dtype=_E8M0)
    p = object.__new__(Packed)
    p._codes = codes if stride == cols else codes[:, :cols]
    p._scales = scales
    p._struct = B.PackedStruct(codes.data_ptr(), scales.data_ptr(), rows, cols, stride)
    return p


def _refuse_gradient(name: str) -> None:
    if torch.is_grad_enabled():
        raise ValueError("%s requires a gradient, which these operators do not record: detach it, or call under "
                         "torch.no_grad()" % name)


def _dense(name: str, x: torch.Tensor) -> Tuple[int, int, int, int]:
    """(rows, cols, row stride, dtype code) of a row-major matrix on a CUDA device."""
    if x.requires_grad:
        _refuse_gradient(name)
    code = _CODES.get(x.dtype)
    if code is None or x.dim() != 2 or not x.is_cuda:
        raise ValueError("%s must be a float32 or bfloat16 matrix on a CUDA device" % name)
    rows, cols = x.shape
    stride, unit = x.stride()
    if unit != 1 and cols > 1:
        raise ValueError("%s must be row-major" % name)
    return rows, cols, stride, code


def _param(cols: int, dev: int, t: torch.Tensor) -> Tuple[int, int]:
    """(pointer, dtype code) of gamma or beta."""
    if t.requires_grad:
        _refuse_gradient("gamma or beta")
    code = _CODES.get(t.dtype)
    if code is None or t.shape != (cols,) or t.get_device() != dev or (cols > 1 and t.stride(0) != 1):
        raise ValueError("gamma and beta must be contiguous float32 or bfloat16 vectors of the row's length")
    return t.data_ptr(), code


def _params(cols: int, dev: int, gamma, beta) -> Tuple[Optional[int], Optional[int], int]:
    """Pointers of gamma and beta and their common dtype code."""
    g, code = (None, B.DIPACO_F32) if gamma is None else _param(cols, dev, gamma)
    if beta is None:
        return g, None, code
    b, beta_code = _param(cols, dev, beta)
    if gamma is not None and beta_code != code:
        raise ValueError("gamma and beta must have one dtype")
    return g, b, beta_code


def pack(x: torch.Tensor) -> Packed:
    """The packed form of a dense matrix."""
    rows, cols, stride, code = _dense("x", x)
    dev = x.get_device()
    out = _packed_beside(x, rows, cols)
    B.dipaco_pack(x.data_ptr(), stride, code, out.struct, dev, _stream(dev))
    return out


def unpack(x: Packed, dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
    """The values that a packed matrix stands for."""
    if dtype not in _CODES:
        raise ValueError("dtype must be float32 or bfloat16")
    dev = x.codes.get_device()
    y = x.codes.new_empty(x.shape, dtype=dtype)
    B.dipaco_unpack(x.struct, y.data_ptr(), y.stride(0), _CODES[dtype], dev, _stream(dev))
    return y


def layer_norm(x: torch.Tensor, gamma: Optional[torch.Tensor] = None, beta: Optional[torch.Tensor] = None,
               eps: float = 1e-5, stats: bool = False):
    """The norm of every row of x, in x's dtype; with ``stats`` (y, mean, rstd) for the backward pass."""
    rows, cols, stride, code = _dense("x", x)
    dev = x.get_device()
    g, b, pcode = _params(cols, dev, gamma, beta)
    y = x.new_empty((rows, cols))
    if not stats:
        B.dipaco_layer_norm(x.data_ptr(), stride, g, b, y.data_ptr(), cols, None, None, rows, cols, eps, code, pcode,
                            dev, _stream(dev))
        return y
    mean, rstd = x.new_empty((2, rows), dtype=_F32).unbind(0)
    B.dipaco_layer_norm(x.data_ptr(), stride, g, b, y.data_ptr(), cols, mean.data_ptr(), rstd.data_ptr(), rows, cols,
                        eps, code, pcode, dev, _stream(dev))
    return y, mean, rstd


def layer_norm_pack(x: torch.Tensor, gamma: Optional[torch.Tensor] = None, beta: Optional[torch.Tensor] = None,
                    eps: float = 1e-5, keep: bool = True):
    """(y, x, mean, rstd): the norm of every row of x, packed, and x itself packed as the checkpoint
    that ``layer_norm_backward`` reads (None without ``keep``)."""
    rows, cols, stride, code = _dense("x", x)
    dev = x.get_device()
    g, b, pcode = _params(cols, dev, gamma, beta)
    y = _packed_beside(x, rows, cols)
    kept = _packed_beside(x, rows, cols) if keep else None
    mean, rstd = x.new_empty((2, rows), dtype=_F32).unbind(0)
    B.dipaco_layer_norm_pack(x.data_ptr(), stride, g, b, y.struct, kept.struct if keep else None, mean.data_ptr(),
                             rstd.data_ptr(), eps, code, pcode, dev, _stream(dev))
    return y, kept, mean, rstd


def layer_norm_backward(dy: torch.Tensor, x: Union[torch.Tensor, Packed], mean: torch.Tensor, rstd: torch.Tensor,
                        gamma: Optional[torch.Tensor] = None):
    """(dx, dgamma, dbeta) from the norm's input or its packed checkpoint; dgamma and dbeta are fp32."""
    rows, cols, stride, code = _dense("dy", dy)
    dev = dy.get_device()
    g, _, pcode = _params(cols, dev, gamma, None)
    for t in (mean, rstd):
        if t.shape != (rows,) or t.dtype != _F32 or t.get_device() != dev or not t.is_contiguous():
            raise ValueError("mean and rstd must be contiguous float32 vectors with one entry per row")
        if t.requires_grad:
            _refuse_gradient("mean or rstd")
    if isinstance(x, Packed):
        x_ptr, x_stride, packed = None, 0, x.struct
        x_shape, x_dev = x.shape, x.codes.get_device()
    else:
        *x_shape, x_stride, x_code = _dense("x", x)
        if x_code != code:
            raise ValueError("x and dy must have one dtype")
        x_ptr, packed, x_dev = x.data_ptr(), None, x.get_device()
    if tuple(x_shape) != (rows, cols) or x_dev != dev:
        raise ValueError("x and dy must have one shape and device")
    dx = dy.new_empty((rows, cols))
    dgamma, dbeta = dy.new_empty((2, cols), dtype=_F32).unbind(0)
    need = B.dipaco_layer_norm_workspace(rows, cols)
    work = dy.new_empty(need, dtype=torch.uint8) if need else None
    B.dipaco_layer_norm_backward(dy.data_ptr(), stride, x_ptr, x_stride, packed, mean.data_ptr(), rstd.data_ptr(), g,
                                 dx.data_ptr(), cols, dgamma.data_ptr(), dbeta.data_ptr(), rows, cols, code, pcode,
                                 work.data_ptr() if need else None, need, dev, _stream(dev))
    return dx, dgamma, dbeta


def gelu_pack(x: torch.Tensor, keep: bool = True):
    """(y, x): the GELU of x, packed, and x itself packed as the checkpoint that
    ``gelu_pack_backward`` reads (None without ``keep``)."""
    rows, cols, stride, code = _dense("x", x)
    dev = x.get_device()
    y = _packed_beside(x, rows, cols)
    kept = _packed_beside(x, rows, cols) if keep else None
    B.dipaco_gelu_pack(x.data_ptr(), stride, code, y.struct, kept.struct if keep else None, dev, _stream(dev))
    return y, kept


def gelu_pack_backward(dy: torch.Tensor, x: Packed) -> Packed:
    """dy * gelu'(x), packed, from the GELU's packed input."""
    rows, cols, stride, code = _dense("dy", dy)
    dev = dy.get_device()
    if x.shape != (rows, cols) or x.codes.get_device() != dev:
        raise ValueError("x and dy must have one shape and device")
    dx = _packed_beside(dy, rows, cols)
    B.dipaco_gelu_pack_backward(dy.data_ptr(), stride, code, x.struct, dx.struct, dev, _stream(dev))
    return dx


def packed_matmul(a: Packed, b: Packed, transpose_a: bool = False, transpose_b: bool = False,
                  out_dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None,
                  accumulate: bool = False) -> torch.Tensor:
    """op(a) op(b) with fp32 sums, op transposing where asked.  ``out`` is written (its dtype is the
    result's), or added to with ``accumulate``."""
    m, k = a.shape
    k2, n = b.shape
    if transpose_a:
        m, k = k, m
    if transpose_b:
        k2, n = n, k2
    dev = a.codes.get_device()
    if k != k2 or b.codes.get_device() != dev:
        raise ValueError("the operands' contracted extents (%d and %d) and devices must agree" % (k, k2))
    if out is None:
        code = _CODES.get(out_dtype)
        if accumulate or code is None:
            raise ValueError("accumulate needs out, and out_dtype is float32 or bfloat16")
        out, stride = a.codes.new_empty((m, n), dtype=out_dtype), n
    else:
        rows, cols, stride, code = _dense("out", out)
        if (rows, cols) != (m, n) or out.get_device() != dev:
            raise ValueError("out must be [%d, %d] on the operands' device" % (m, n))
    need = B.dipaco_packed_matmul_workspace(m, n, k)
    work = a.codes.new_empty(need, dtype=torch.uint8) if need else None
    B.dipaco_packed_matmul(a.struct, b.struct, transpose_a, transpose_b, out.data_ptr(), stride, code, accumulate,
                           work.data_ptr() if need else None, need, dev, _stream(dev))
    return out


def inner_status(device=None) -> int:
    """Waits for the current stream and reports DIPACO_OK, or DIPACO_ETIMEOUT once (to each stream that
    asks) after a bounded wait inside one of these operators ran out on the device."""
    dev = None if device is None else torch.device(device).index
    dev = torch.cuda.current_device() if dev is None else dev
    return B.dipaco_inner_status(dev, _stream(dev))
