"""Operators of a path's inner phase on torch CUDA tensors (declared in ``include/dipaco.h``).

Layer norm with its gradient, matrices packed in 8 bits (activation checkpoints and the operands of
the products), the GELU that writes and reads such checkpoints, the product of packed matrices on the
tensor cores, linear layers with bias, activation and residual, the norms around a block with its gate
and residual, and the clipping of gradients.  Each function allocates its results (and workspace) with
torch, launches on the current stream of the tensors' device, and raises ``ValueError`` for shapes and dtypes that do not
fit together or ``binding.DipacoError`` with the library's status.  There is no CPU path.

Autograd records nothing of these calls: the gradients are calls of their own.  A tensor that requires a
gradient is refused while gradients are being recorded; inside ``torch.no_grad()`` or a
``torch.autograd.Function``, or detached, it is taken.
"""
from __future__ import annotations

import ctypes
import math
from typing import NamedTuple, Optional, Sequence, Tuple, Union

import torch

from . import binding as B

BLOCK = 128  # one scale per BLOCK x BLOCK values
_F32, _E4M3, _E8M0 = torch.float32, torch.float8_e4m3fn, torch.float8_e8m0fnu
_CODES = {torch.float32: B.DIPACO_F32, torch.bfloat16: B.DIPACO_BF16}
_ACTIVATIONS = {None: B.DIPACO_ACTIVATION_NONE, "relu": B.DIPACO_ACTIVATION_RELU,
                "silu": B.DIPACO_ACTIVATION_SILU, "gelu": B.DIPACO_ACTIVATION_GELU}
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


def _activation(name: Optional[str]) -> int:
    code = _ACTIVATIONS.get(name)
    if code is None:
        raise ValueError("activation must be None, 'relu', 'silu' or 'gelu'")
    return code


def _layer(x: Packed, w: Packed, bias: Optional[torch.Tensor]) -> Tuple[int, int, int, int, Optional[int], int]:
    """(tokens, out, in, device, pointer of the bias, its dtype code) of x [tokens, in] through w [out, in]."""
    m, k = x.shape
    n, k2 = w.shape
    dev = x.codes.get_device()
    if k != k2 or w.codes.get_device() != dev:
        raise ValueError("x and w must have one inner extent (%d and %d) and device" % (k, k2))
    if bias is None:
        return m, n, k, dev, None, B.DIPACO_F32
    if bias.requires_grad:
        _refuse_gradient("bias")
    code = _CODES.get(bias.dtype)
    if code is None or bias.shape != (n,) or bias.get_device() != dev or (n > 1 and bias.stride(0) != 1):
        raise ValueError("bias must be a contiguous float32 or bfloat16 vector with one entry per output")
    return m, n, k, dev, bias.data_ptr(), code


def packed_linear(x: Packed, w: Packed, bias: Optional[torch.Tensor] = None, activation: Optional[str] = None,
                  residual: Optional[torch.Tensor] = None, out_dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """act(x w^T + bias) + residual for x [tokens, in] and w [out, in], with fp32 sums, rounded once to ``out_dtype``
    (the residual's, or bfloat16).  ``activation`` is None, "relu", "silu" or "gelu"."""
    m, n, k, dev, bias_ptr, bias_code = _layer(x, w, bias)
    act = _activation(activation)
    if out_dtype is None:
        out_dtype = torch.bfloat16 if residual is None else residual.dtype
    code = _CODES.get(out_dtype)
    if code is None:
        raise ValueError("out_dtype must be float32 or bfloat16")
    r_ptr, r_stride = (None, 0) if residual is None else _like("residual", residual, (m, n), dev, code)
    y = x.codes.new_empty((m, n), dtype=out_dtype)
    need = B.dipaco_packed_matmul_workspace(m, n, k)
    work = y.new_empty(need, dtype=torch.uint8) if need else None
    B.dipaco_packed_linear(x.struct, w.struct, bias_ptr, bias_code, act, r_ptr, r_stride, y.data_ptr(), n, code,
                           work.data_ptr() if need else None, need, dev, _stream(dev))
    return y


def packed_linear_pack(x: Packed, w: Packed, bias: Optional[torch.Tensor] = None, activation: Optional[str] = None,
                       keep: bool = True):
    """(y, a): y = act(a) of a = x w^T + bias, packed, and a itself packed as the checkpoint that
    ``packed_linear_pack_backward`` reads (None without ``keep``, and without an activation, where y is a)."""
    m, n, k, dev, bias_ptr, bias_code = _layer(x, w, bias)
    act = _activation(activation)
    y = _packed_beside(x.codes, m, n)
    a = _packed_beside(x.codes, m, n) if keep and act else None
    need = B.dipaco_packed_linear_pack_workspace(m, n, k)
    work = x.codes.new_empty(need, dtype=torch.uint8) if need else None
    B.dipaco_packed_linear_pack(x.struct, w.struct, bias_ptr, bias_code, act, y.struct, a.struct if a else None,
                                work.data_ptr() if need else None, need, dev, _stream(dev))
    return y, a


def packed_linear_pack_backward(dy: Packed, w: Packed, a: Optional[Packed] = None, activation: Optional[str] = None,
                                bias: bool = True):
    """(da, dbias) from the gradient dy [tokens, out] of a layer w [out, in]: da = (dy w) act'(a), packed, for the
    checkpoint a [tokens, in] of the layer before, whose bias has the gradient dbias, the sum of da over the tokens in
    float32 (None without ``bias``)."""
    act = _activation(activation)
    m, k = dy.shape
    k2, n = w.shape
    dev = dy.codes.get_device()
    if k != k2 or w.codes.get_device() != dev:
        raise ValueError("dy and w must have one outer extent (%d and %d) and device" % (k, k2))
    if act:
        if a is None or a.shape != (m, n) or a.codes.get_device() != dev:
            raise ValueError("a must be the packed input [%d, %d] of the activation, on dy's device" % (m, n))
    elif a is not None:
        raise ValueError("a is only read for an activation")
    da = _packed_beside(dy.codes, m, n)
    dbias = dy.codes.new_empty(n, dtype=_F32) if bias else None
    need = B.dipaco_packed_linear_pack_backward_workspace(m, n, k) if bias else 0
    work = da.codes.new_empty(need, dtype=torch.uint8) if need else None
    B.dipaco_packed_linear_pack_backward(dy.struct, w.struct, a.struct if act else None, act, da.struct,
                                         dbias.data_ptr() if bias else None, work.data_ptr() if need else None, need, dev,
                                         _stream(dev))
    return da, dbias


class ResidualNormGradients(NamedTuple):
    """Gradients of ``residual_norm``; None for what the call does not have."""
    x: torch.Tensor
    f: torch.Tensor
    gate: Optional[torch.Tensor]        # of the gate's shape: fp32, or in dn's dtype for a gate of every value
    gamma: Optional[torch.Tensor]       # fp32, as the following
    beta: Optional[torch.Tensor]
    post_gamma: Optional[torch.Tensor]
    post_beta: Optional[torch.Tensor]


def _gate(gate: Optional[torch.Tensor], rows: int, cols: int, dev: int, code: int) -> Tuple[int, Optional[int], int, int]:
    """(kind, pointer, row stride, dtype code) of a gate [cols], [rows, 1] or [rows, cols]."""
    if gate is None:
        return B.DIPACO_GATE_NONE, None, 0, B.DIPACO_F32
    if gate.requires_grad:
        _refuse_gradient("gate")
    own = _CODES.get(gate.dtype)
    if own is None or gate.get_device() != dev:
        raise ValueError("gate must be float32 or bfloat16, on the rows' device")
    if gate.shape == (cols,):
        if cols > 1 and gate.stride(0) != 1:
            raise ValueError("a gate of columns must be contiguous")
        return B.DIPACO_GATE_COLS, gate.data_ptr(), 0, own
    in_steps = rows > 1 and gate.dim() == 2 and gate.stride(0) != 1
    if gate.shape == (rows, 1) and not (in_steps and cols == 1):  # of one column: every value's, if rows are apart
        if in_steps:
            raise ValueError("a gate of rows must be contiguous")
        return B.DIPACO_GATE_ROWS, gate.data_ptr(), 0, own
    if gate.shape == (rows, cols):
        if own != code or (cols > 1 and gate.stride(1) != 1):
            raise ValueError("a gate of all values must be row-major and have the rows' dtype")
        return B.DIPACO_GATE_FULL, gate.data_ptr(), gate.stride(0), own
    raise ValueError("gate must be [cols], [rows, 1] or [rows, cols]")


def _residual_norm_args(rows, cols, dev, code, gamma, beta, post_gamma, post_beta, gate, residual_scale, post_norm, norm,
                        eps) -> B.ResidualNormStruct:
    if not norm and (gamma is not None or beta is not None):
        raise ValueError("gamma and beta belong to the norm that is left out")
    if not post_norm and (post_gamma is not None or post_beta is not None):
        raise ValueError("post_gamma and post_beta belong to the norm that is left out")
    given, pcode = [None] * 4, None
    for i, p in enumerate((gamma, beta, post_gamma, post_beta)):
        if p is not None:
            given[i], p_code = _param(cols, dev, p)
            if pcode is None:
                pcode = p_code
            elif p_code != pcode:
                raise ValueError("the norms' parameters must have one dtype")
    kind, gate_ptr, gate_stride, gate_code = _gate(gate, rows, cols, dev, code)
    return B.ResidualNormStruct(rows, cols, *given, gate_ptr, gate_stride, kind, gate_code, code,
                                B.DIPACO_F32 if pcode is None else pcode, post_norm, norm, residual_scale, eps)


def _like(name: str, x: torch.Tensor, shape: Tuple[int, int], dev: int, code: int) -> Tuple[int, int]:
    """(pointer, row stride) of a dense matrix that has to go with others."""
    rows, cols, stride, own = _dense(name, x)
    if (rows, cols) != shape or own != code or x.get_device() != dev:
        raise ValueError("%s must have the other matrices' shape, dtype and device" % name)
    return x.data_ptr(), stride


def residual_norm(x: torch.Tensor, f: torch.Tensor, gamma: Optional[torch.Tensor] = None,
                  beta: Optional[torch.Tensor] = None, post_gamma: Optional[torch.Tensor] = None,
                  post_beta: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                  residual_scale: float = 1.0, post_norm: bool = True, norm: bool = True, eps: float = 1e-5):
    """(z, n, stats) of a residual stream x and a block's result f:

        z = residual_scale * x + gate * (LN(f) * post_gamma + post_beta),   n = LN(z) * gamma + beta,

    the norm after the block, its gate and residual, and the norm before the next one, of z as it is held in x's
    dtype.  ``gate`` is [cols], [rows, 1] or [rows, cols].  Without ``post_norm`` f goes in as it is; without ``norm``
    n is None.  stats [4, rows] is for ``residual_norm_backward``."""
    rows, cols, x_stride, code = _dense("x", x)
    dev = x.get_device()
    f_ptr, f_stride = _like("f", f, (rows, cols), dev, code)
    args = _residual_norm_args(rows, cols, dev, code, gamma, beta, post_gamma, post_beta, gate, residual_scale,
                               post_norm, norm, eps)
    z = x.new_empty((rows, cols))
    n = x.new_empty((rows, cols)) if norm else None
    stats = x.new_empty((4, rows), dtype=_F32)
    B.dipaco_residual_norm(args, x.data_ptr(), x_stride, f_ptr, f_stride, z.data_ptr(), cols,
                           n.data_ptr() if norm else None, cols, None, None, stats.data_ptr(), dev, _stream(dev))
    return z, n, stats


def residual_norm_pack(x: torch.Tensor, f: torch.Tensor, gamma: Optional[torch.Tensor] = None,
                       beta: Optional[torch.Tensor] = None, post_gamma: Optional[torch.Tensor] = None,
                       post_beta: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                       residual_scale: float = 1.0, post_norm: bool = True, eps: float = 1e-5, keep: bool = True):
    """(z, n, kept, stats): ``residual_norm`` with n packed, and z packed too as the checkpoint that
    ``residual_norm_backward`` reads (None without ``keep``)."""
    rows, cols, x_stride, code = _dense("x", x)
    dev = x.get_device()
    f_ptr, f_stride = _like("f", f, (rows, cols), dev, code)
    args = _residual_norm_args(rows, cols, dev, code, gamma, beta, post_gamma, post_beta, gate, residual_scale,
                               post_norm, True, eps)
    z = x.new_empty((rows, cols))
    n = _packed_beside(x, rows, cols)
    kept = _packed_beside(x, rows, cols) if keep else None
    stats = x.new_empty((4, rows), dtype=_F32)
    B.dipaco_residual_norm(args, x.data_ptr(), x_stride, f_ptr, f_stride, z.data_ptr(), cols, None, 0, n.struct,
                           kept.struct if keep else None, stats.data_ptr(), dev, _stream(dev))
    return z, n, kept, stats


def residual_norm_backward(dn: Optional[torch.Tensor], dz: Optional[torch.Tensor], f: Union[torch.Tensor, Packed],
                           z: Union[torch.Tensor, Packed, None], stats: torch.Tensor,
                           gamma: Optional[torch.Tensor] = None, post_gamma: Optional[torch.Tensor] = None,
                           post_beta: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                           residual_scale: float = 1.0, post_norm: bool = True) -> ResidualNormGradients:
    """Gradients of ``residual_norm`` from those of n (dn; None without ``norm``, and then z may be None) and of z
    (dz; None where z goes nowhere else).  f and z are the forward pass's, or packed checkpoints of them."""
    like = dn if dn is not None else dz
    if like is None:
        raise ValueError("dn or dz must be given")
    rows, cols, stride, code = _dense("dn" if dn is not None else "dz", like)
    dev = like.get_device()
    norm = dn is not None
    dz_ptr, dz_stride = (None, 0) if dz is None else _like("dz", dz, (rows, cols), dev, code)
    if stats.shape != (4, rows) or stats.dtype != _F32 or stats.get_device() != dev or not stats.is_contiguous():
        raise ValueError("stats must be the contiguous float32 [4, rows] of the forward call")
    if stats.requires_grad:
        _refuse_gradient("stats")
    read = []
    for name, t in (("f", f), ("z", z if norm else None)):
        if isinstance(t, Packed):
            if t.shape != (rows, cols) or t.codes.get_device() != dev:
                raise ValueError("%s must have the other matrices' shape and device" % name)
            read += [None, 0, t.struct]
        elif t is not None:
            read += [*_like(name, t, (rows, cols), dev, code), None]
        elif name == "z" and not norm:
            read += [None, 0, None]
        else:
            raise ValueError("%s must be given" % name)
    args = _residual_norm_args(rows, cols, dev, code, gamma, None, post_gamma, post_beta, gate, residual_scale,
                               post_norm, norm, 0.0)
    dx, df = like.new_empty((rows, cols)), like.new_empty((rows, cols))
    dgate = None if gate is None else gate.new_empty(
        gate.shape, dtype=gate.dtype if args.gate_kind == B.DIPACO_GATE_FULL else _F32)
    sums = like.new_empty((4, cols), dtype=_F32).unbind(0)
    dgamma, dbeta = sums[:2] if norm else (None, None)
    dpost_gamma, dpost_beta = sums[2:] if post_norm else (None, None)
    need = B.dipaco_residual_norm_workspace(rows, cols)
    work = like.new_empty(need, dtype=torch.uint8) if need else None
    ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    B.dipaco_residual_norm_backward(args, ptr(dn), stride, dz_ptr, dz_stride, *read, stats.data_ptr(), dx.data_ptr(), cols,
                                    df.data_ptr(), cols, ptr(dgate), cols, ptr(dgamma), ptr(dbeta), ptr(dpost_gamma),
                                    ptr(dpost_beta), ptr(work), need, dev, _stream(dev))
    return ResidualNormGradients(dx, df, dgate, dgamma, dbeta, dpost_gamma, dpost_beta)


def _dense_in_some_order(t: torch.Tensor) -> bool:
    """Whether t's values fill the memory from its first to its last without gaps."""
    if t.is_contiguous():
        return True
    step = 1
    for stride, size in sorted(zip(t.stride(), t.shape)):
        if size != 1:
            if stride != step:
                return False
            step *= size
    return True


def _gradients(grads: Sequence[torch.Tensor], any_order: bool):
    """(tensors, device, numels, pointers, dtype codes) of gradients that are taken as they lie in memory."""
    grads = list(grads)
    if not grads:
        raise ValueError("there must be a gradient")
    dev = grads[0].get_device()
    codes = [_CODES.get(t.dtype) for t in grads]
    for t, code in zip(grads, codes):
        if code is None or dev < 0 or t.get_device() != dev:
            raise ValueError("gradients must be float32 or bfloat16 tensors on one CUDA device")
        if not t.is_contiguous() and not (any_order and _dense_in_some_order(t)):
            raise ValueError("gradients must be contiguous")
        if t.requires_grad:
            _refuse_gradient("a gradient")
    return grads, dev, [t.numel() for t in grads], [t.data_ptr() for t in grads], codes


def _clip(like: torch.Tensor, dev, numels, ptrs, codes, out_ptrs, out_codes, max_norm: float,
          keep: bool = True) -> Optional[torch.Tensor]:
    count = len(numels)
    words, longs = ctypes.c_int32 * count, ctypes.c_int64 * count
    numel, dtypes, grads = longs(*numels), words(*codes), longs(*ptrs)
    out = out_dtypes = None
    if out_ptrs is not None:
        out = grads if out_ptrs is ptrs else longs(*out_ptrs)
        out_dtypes = dtypes if out_codes is codes else words(*out_codes)
    norm = like.new_empty((), dtype=_F32) if keep else None
    need = B.dipaco_clip_gradients_workspace(numel, count) if keep or max_norm < math.inf else 0
    work = like.new_empty(need, dtype=torch.uint8) if need else None
    B.dipaco_clip_gradients(grads, out, numel, dtypes, out_dtypes, count, max_norm, norm.data_ptr() if keep else None,
                            work.data_ptr() if need else None, need, dev, _stream(dev))
    return norm


def _most(max_norm: float) -> float:
    max_norm = float(max_norm)
    if not max_norm >= 0.0:
        raise ValueError("max_norm must not be negative")
    return max_norm


def gradient_norm(grads: Sequence[torch.Tensor]) -> torch.Tensor:
    """The norm of all gradients together, a float32 scalar on their device."""
    grads, dev, numels, ptrs, codes = _gradients(grads, True)
    return _clip(grads[0], dev, numels, ptrs, codes, None, None, math.inf)


def clip_gradients(grads: Sequence[torch.Tensor], max_norm: float) -> torch.Tensor:
    """Multiplies the gradients by min(1, max_norm / norm) in place and returns their norm before that.  No two may
    share memory."""
    grads, dev, numels, ptrs, codes = _gradients(grads, True)
    return _clip(grads[0], dev, numels, ptrs, codes, ptrs, codes, _most(max_norm))


def gather_gradients(grads: Sequence[torch.Tensor], max_norm: Optional[float] = None, dtype: torch.dtype = torch.float32,
                     norm: bool = True) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """(flat, norm): the gradients one after another in a vector, as the modules lie in a path's copy, clipped to
    ``max_norm`` unless it is None, and their norm before that (None without ``norm``)."""
    if dtype not in _CODES:
        raise ValueError("dtype must be float32 or bfloat16")
    most = math.inf if max_norm is None else _most(max_norm)
    grads, dev, numels, ptrs, codes = _gradients(grads, False)
    flat = grads[0].new_empty(sum(numels), dtype=dtype)
    at, size, out = flat.data_ptr(), flat.element_size(), []
    for n in numels:
        out.append(at)
        at += n * size
    return flat, _clip(flat, dev, numels, ptrs, codes, out, [_CODES[dtype]] * len(out), most, norm)


def inner_status(device=None) -> int:
    """Waits for the current stream and reports DIPACO_OK, or DIPACO_ETIMEOUT once (to each stream that
    asks) after a bounded wait inside one of these operators ran out on the device."""
    dev = None if device is None else torch.device(device).index
    dev = torch.cuda.current_device() if dev is None else dev
    return B.dipaco_inner_status(dev, _stream(dev))
