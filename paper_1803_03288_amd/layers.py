"""Operators of a worker's layers, by the kernels of ``libtictac.so`` (C ABI and formulas: ``include/tictac.h``).

What a worker's iteration does between the transfers that the rest of the package orders: layers whose parameters are
transferred in 8 bits, a quarter of the bytes of float32, and whose activations are kept in 8 bits for the backward pass.

    y8, mean, rstd, x8 = layers.layer_norm_q8(x, gamma, beta, save=True)      # forward
    y = layers.linear_q8(y8, w8, bias, dtype=x.dtype)
    dn, dw, db = layers.linear_q8_backward(dy, y8, w8)                        # backward, from y8 and x8 alone
    dx, dgamma, dbeta = layers.layer_norm_backward(dn, x8, gamma, mean, rstd)

``python -m paper_1803_03288_amd.measured`` runs a stack of such layers, measures their ops and orders their transfers.

Tensors are CUDA tensors of float32, float16 or bfloat16; the last dimension is the row, and outputs have the shape of
the input in the others.  Rows may lie at any stride; elements of a row that are not next to each other are copied first.
Everything runs on the current stream; there is no CPU fallback.  A wrong argument raises ``ValueError`` or ``TypeError``, what the library
refuses ``TicTacError``.
"""

from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional, Union

import torch

from .binding import _check, _stream, lib

GROUP = 128                     # columns per scale of kept activations
_DTYPE = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
_I32, _I64, _PTR, _SIZE = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t

_SIGNATURES = {
    "tictac_quantize_rows": (_I32, _I64, _I64, _PTR, _I64, _I32, _PTR, _I64, _PTR, _PTR),
    "tictac_dequantize_rows": (_I32, _I64, _I64, _PTR, _I64, _PTR, _I32, _PTR, _I64, _PTR),
    "tictac_layer_norm": (_I32, _I64, _I64, _PTR, _I64, _I32, _PTR, _PTR, ctypes.c_float, _PTR, _I64, _PTR, _PTR, _PTR, _I64, _PTR,
                          _PTR, _I64, _PTR, _PTR),
    "tictac_layer_norm_backward_workspace": (_I64, _I64, _PTR),
    "tictac_layer_norm_backward": (_I32, _I64, _I64, _PTR, _I64, _PTR, _I64, _PTR, _I64, _PTR, _I32, _PTR, _PTR, _PTR, _PTR, _I64,
                                   _PTR, _PTR, _PTR, _SIZE, _PTR),
    "tictac_linear_q8_workspace": (_I32, _I64, _I64, _I64, _PTR),
    "tictac_linear_q8": (_I32, _I64, _I64, _I64, _PTR, _I64, _PTR, _I64, _PTR, _PTR, _I64, _PTR, _I32, _PTR, _PTR, _I64, _PTR, _SIZE,
                         _PTR),
    "tictac_linear_q8_backward_workspace": (_I32, _I64, _I64, _I64, _PTR),
    "tictac_linear_q8_backward": (_I32, _I64, _I64, _I64, _PTR, _I64, _PTR, _I64, _PTR, _PTR, _I64, _PTR, _PTR, _I64, _PTR, _I64, _PTR,
                                  _PTR, _SIZE, _PTR),
}
_calls: dict = {}


def _call(name: str, *args) -> None:
    fn = _calls.get(name)
    if fn is None:
        # (an object of its own: its argument types are not those of other callers of the library)
        fn = ctypes.CFUNCTYPE(_I32, *_SIGNATURES[name])((name, lib()))
        _calls[name] = fn
    rc = fn(*args)
    if rc:
        _check(rc)


class Rows8(NamedTuple):
    """8-bit rows: the values ``q * scale`` of ``[rows][cols]``.  ``q`` is int8 ``[rows][ld]``, ``ld`` a multiple of 128, zeros behind column
    ``cols``; ``scale`` is float32 ``[rows][1]`` (``group`` 0) or ``[rows][ceil(cols / 128)]`` (``group`` 128)."""
    q: torch.Tensor
    scale: torch.Tensor
    cols: int
    group: int = 0

    @property
    def shape(self):
        return (self.q.shape[0], self.cols)


def _padded(cols: int) -> int:
    return (cols + 127) // 128 * 128


def _float_rows(name: str, x: torch.Tensor) -> torch.Tensor:
    """``x`` as ``[rows][cols]`` with the elements of a row next to each other."""
    if not x.is_cuda:
        raise ValueError(f"{name} is on {x.device}: the operators take CUDA tensors")
    if x.dtype not in _DTYPE:
        raise TypeError(f"{name} is {x.dtype}: expected float32, float16 or bfloat16")
    if x.dim() != 2:
        if x.dim() == 0:
            raise ValueError(f"{name} has no dimension")
        x = x.reshape(-1, x.shape[-1]) if x.shape[-1] else x.reshape(0, 0)
    if x.shape[1] == 0:
        raise ValueError(f"{name} has rows of no columns")
    if x.stride(1) != 1 and x.shape[1] > 1 or x.stride(0) < 0:
        x = x.contiguous()
    return x


def _vector(name: str, v: Optional[torch.Tensor], n: int, dtype: torch.dtype, like: torch.Tensor) -> Optional[torch.Tensor]:
    """A parameter of ``n`` values in float32 or ``dtype``."""
    if v is None:
        return None
    if v.dim() != 1 or v.shape[0] != n:
        raise ValueError(f"{name} has the shape {tuple(v.shape)}, expected ({n},)")
    if v.dtype != torch.float32 and v.dtype != dtype:
        raise TypeError(f"{name} is {v.dtype}: expected float32 or {dtype}")
    if v.device != like.device:
        raise ValueError(f"{name} is on {v.device}, expected {like.device}")
    return v if v.is_contiguous() else v.contiguous()


def _statistic(name: str, v: torch.Tensor, rows: int, like: torch.Tensor) -> torch.Tensor:
    if v.dtype != torch.float32 or v.numel() != rows or v.device != like.device:
        raise ValueError(f"{name}: expected {rows} float32 values on {like.device}")
    return v if v.is_contiguous() else v.contiguous()


def _rows8(name: str, r: Rows8, group: int, device: torch.device) -> Rows8:
    q, scale, cols, has = r
    if has != group:
        raise ValueError(f"{name} has a scale per {has or 'row'}: expected one per {group or 'row'}")
    if q.dtype != torch.int8 or q.dim() != 2 or scale.dtype != torch.float32:
        raise TypeError(f"{name}: expected int8 rows and float32 scales")
    if q.device != device or scale.device != device:
        raise ValueError(f"{name} is on {q.device} and {scale.device}, expected {device}")
    if cols < 1 or q.shape[1] < _padded(cols) or (q.stride(1) != 1) or not scale.is_contiguous():
        raise ValueError(f"{name}: rows of {cols} columns are padded to {_padded(cols)}, contiguous, and so are their scales")
    if scale.numel() != q.shape[0] * ((cols + GROUP - 1) // GROUP if group else 1):
        raise ValueError(f"{name}: {scale.numel()} scales for {q.shape[0]} rows of {cols} columns")
    return r


def _row_stride(q: torch.Tensor) -> int:
    return q.stride(0) if q.shape[0] > 1 else _padded(q.shape[1])


def _ld(x: torch.Tensor) -> int:
    return x.stride(0) if x.shape[0] > 1 else x.shape[1]


def _same_device(x: torch.Tensor) -> None:
    if x.device.index != torch.cuda.current_device():
        raise ValueError(f"tensors are on {x.device}, the current device is cuda:{torch.cuda.current_device()}")


def _workspace(name: str, *sizes, device) -> Optional[torch.Tensor]:
    n = ctypes.c_size_t()
    _call(name, *sizes, ctypes.addressof(n))
    return torch.empty(n.value, dtype=torch.uint8, device=device) if n.value else None


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _new_rows8(rows: int, cols: int, group: int, device) -> Rows8:
    return Rows8(torch.empty((rows, _padded(cols)), dtype=torch.int8, device=device),
                 torch.empty((rows, (cols + GROUP - 1) // GROUP if group else 1), dtype=torch.float32, device=device), cols, group)


def quantize_rows(x: torch.Tensor, group: int = 0) -> Rows8:
    """``x`` in 8 bits.  ``group`` 0: a scale per row (weights by output channel, operands of products); 128: one per 128 columns
    (activations kept for the backward pass).  A row (group) with a NaN or an infinity reads as NaN throughout."""
    if group not in (0, GROUP):
        raise ValueError(f"group = {group}: expected 0 or {GROUP}")
    x = _float_rows("x", x)
    _same_device(x)
    rows, cols = x.shape
    r = _new_rows8(rows, cols, group, x.device)
    _call("tictac_quantize_rows", _DTYPE[x.dtype], rows, cols, x.data_ptr(), _ld(x), group, r.q.data_ptr(), r.q.shape[1], r.scale.data_ptr(),
          _stream())
    return r


def dequantize_rows(r: Rows8, dtype: torch.dtype = torch.float32) -> torch.Tensor:
    """The values of 8-bit rows, ``[rows][cols]``, rounded to ``dtype``."""
    if dtype not in _DTYPE:
        raise TypeError(f"{dtype}: expected float32, float16 or bfloat16")
    _rows8("r", r, r.group, r.q.device)
    if r.group not in (0, GROUP) or not r.q.is_cuda:
        raise ValueError("r: expected CUDA tensors and a group of 0 or 128")
    _same_device(r.q)
    x = torch.empty(r.shape, dtype=dtype, device=r.q.device)
    _call("tictac_dequantize_rows", _DTYPE[dtype], x.shape[0], x.shape[1], r.q.data_ptr(), _row_stride(r.q), r.scale.data_ptr(), r.group, x.data_ptr(),
          x.shape[1], _stream())
    return x


def _layer_norm(x, weight, bias, eps, want_y, want_y8, save):
    shape = x.shape
    x = _float_rows("x", x)
    _same_device(x)
    rows, cols = x.shape
    weight = _vector("weight", weight, cols, x.dtype, x)
    bias = _vector("bias", bias, cols, x.dtype, x)
    if weight is not None and bias is not None and weight.dtype != bias.dtype:
        raise TypeError(f"weight is {weight.dtype} and bias {bias.dtype}: expected one type")
    some = weight if weight is not None else bias
    y = torch.empty((rows, cols), dtype=x.dtype, device=x.device) if want_y else None
    mean, rstd = torch.empty((2, rows), dtype=torch.float32, device=x.device).unbind(0)
    y8 = _new_rows8(rows, cols, 0, x.device) if want_y8 else None
    x8 = _new_rows8(rows, cols, GROUP, x.device) if save else None
    ld = _padded(cols)
    _call("tictac_layer_norm", _DTYPE[x.dtype], rows, cols, x.data_ptr(), _ld(x), 0 if some is None else _DTYPE[some.dtype], _ptr(weight), _ptr(bias), eps,
          _ptr(y), cols, mean.data_ptr(), rstd.data_ptr(), y8 and y8.q.data_ptr(), ld, y8 and y8.scale.data_ptr(), x8 and x8.q.data_ptr(), ld,
          x8 and x8.scale.data_ptr(), _stream())
    return (y.view(shape) if want_y and len(shape) != 2 else y), y8, mean, rstd, x8


def layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, eps: float = 1e-5, save: bool = False):
    """``(y, mean, rstd)`` of layer norm over the last dimension; with ``save`` also ``x`` as 8-bit rows of group 128 for the backward
    pass, from the same read of ``x``.  ``weight`` and ``bias`` in float32 or the type of ``x``; ``mean`` and ``rstd`` float32 ``[rows]``."""
    y, _, mean, rstd, x8 = _layer_norm(x, weight, bias, eps, True, False, save)
    return (y, mean, rstd, x8) if save else (y, mean, rstd)


def layer_norm_q8(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, eps: float = 1e-5, save: bool = False):
    """``(y8, mean, rstd)``: layer norm whose output is 8-bit rows, the operand of ``linear_q8``; ``save`` as in ``layer_norm``."""
    _, y8, mean, rstd, x8 = _layer_norm(x, weight, bias, eps, False, True, save)
    return (y8, mean, rstd, x8) if save else (y8, mean, rstd)


def layer_norm_backward(dy: torch.Tensor, x: Union[torch.Tensor, Rows8], weight: Optional[torch.Tensor], mean: torch.Tensor, rstd: torch.Tensor):
    """``(dx, dweight, dbias)`` of layer norm from its input, or from the 8-bit rows (group 128) that the forward pass saved.
    ``dweight`` and ``dbias`` have the type of ``weight`` (float32 without one)."""
    shape = dy.shape
    dy = _float_rows("dy", dy)
    _same_device(dy)
    rows, cols = dy.shape
    saved = isinstance(x, Rows8)
    if saved:
        _rows8("x", x, GROUP, dy.device)
    else:
        x = _float_rows("x", x)
        if x.dtype != dy.dtype or x.device != dy.device:
            raise TypeError(f"x is {x.dtype} on {x.device}, dy {dy.dtype} on {dy.device}")
    if tuple(x.shape) != (rows, cols):
        raise ValueError(f"x is {tuple(x.shape)}, dy {(rows, cols)}")
    weight = _vector("weight", weight, cols, dy.dtype, dy)
    mean, rstd = _statistic("mean", mean, rows, dy), _statistic("rstd", rstd, rows, dy)
    of = torch.float32 if weight is None else weight.dtype
    dx = torch.empty((rows, cols), dtype=dy.dtype, device=dy.device)
    dweight, dbias = torch.empty(cols, dtype=of, device=dy.device), torch.empty(cols, dtype=of, device=dy.device)
    room = _workspace("tictac_layer_norm_backward_workspace", rows, cols, device=dy.device)
    _call("tictac_layer_norm_backward", _DTYPE[dy.dtype], rows, cols, dy.data_ptr(), _ld(dy), None if saved else x.data_ptr(), 0 if saved else _ld(x),
          x.q.data_ptr() if saved else None, _row_stride(x.q) if saved else 0, x.scale.data_ptr() if saved else None, _DTYPE[of], _ptr(weight), mean.data_ptr(),
          rstd.data_ptr(), dx.data_ptr(), cols, dweight.data_ptr(), dbias.data_ptr(), _ptr(room), 0 if room is None else room.numel(), _stream())
    return (dx.view(shape) if len(shape) != 2 else dx), dweight, dbias


def linear_q8(x: Union[torch.Tensor, Rows8], w: Rows8, bias: Optional[torch.Tensor] = None, dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """``x @ w.T + bias`` with both operands in 8 bits, ``w`` ``[outs][cols]`` with a scale per output, sums exact.  ``x`` is rounded to 8 bits, a scale
    per row, in the call, unless it is given as ``Rows8``; then ``dtype`` is the output's type (float32 unless given)."""
    saved = isinstance(x, Rows8)
    if saved:
        shape, dtype = x.shape, dtype or torch.float32
        if dtype not in _DTYPE:
            raise TypeError(f"{dtype}: expected float32, float16 or bfloat16")
        device = x.q.device
        if not x.q.is_cuda:
            raise ValueError(f"x is on {device}: the operators take CUDA tensors")
        _rows8("x", x, 0, device)
        rows, cols = x.shape
        _same_device(x.q)
    else:
        shape = x.shape
        if dtype is not None and dtype != x.dtype:
            raise TypeError(f"dtype = {dtype} with x of {x.dtype}: expected the same")
        x = _float_rows("x", x)
        _same_device(x)
        (rows, cols), dtype, device = x.shape, x.dtype, x.device
    _rows8("w", w, 0, device)
    outs = w.q.shape[0]
    if w.cols != cols:
        raise ValueError(f"x has {cols} columns, w {w.cols}")
    bias = _vector("bias", bias, outs, dtype, w.q)
    y = torch.empty((rows, outs), dtype=dtype, device=device)
    room = _workspace("tictac_linear_q8_workspace", 0 if saved else 1, rows, cols, outs, device=device)
    _call("tictac_linear_q8", _DTYPE[dtype], rows, cols, outs, None if saved else x.data_ptr(), 0 if saved else _ld(x), x.q.data_ptr() if saved else None,
          _row_stride(x.q) if saved else 0, x.scale.data_ptr() if saved else None, w.q.data_ptr(), _row_stride(w.q), w.scale.data_ptr(),
          0 if bias is None else _DTYPE[bias.dtype], _ptr(bias), y.data_ptr(), outs, _ptr(room), 0 if room is None else room.numel(), _stream())
    return y if len(shape) == 2 else y.view(*shape[:-1], outs)


def linear_q8_backward(dy: torch.Tensor, x: Rows8, w: Rows8):
    """``(dx, dw, db)`` of ``linear_q8`` from the 8-bit rows that the forward pass took, all of the type of ``dy``; the rounding of the
    input counts as the identity."""
    shape = dy.shape
    dy = _float_rows("dy", dy)
    _same_device(dy)
    rows, outs = dy.shape
    _rows8("x", x, 0, dy.device)
    _rows8("w", w, 0, dy.device)
    cols = x.cols
    if x.q.shape[0] != rows or w.q.shape[0] != outs or w.cols != cols:
        raise ValueError(f"dy is {(rows, outs)}, x {tuple(x.shape)}, w {tuple(w.shape)}")
    dx = torch.empty((rows, cols), dtype=dy.dtype, device=dy.device)
    dw = torch.empty((outs, cols), dtype=dy.dtype, device=dy.device)
    db = torch.empty(outs, dtype=dy.dtype, device=dy.device)
    dt = _DTYPE[dy.dtype]
    room = _workspace("tictac_linear_q8_backward_workspace", dt, rows, cols, outs, device=dy.device)
    _call("tictac_linear_q8_backward", dt, rows, cols, outs, dy.data_ptr(), _ld(dy), x.q.data_ptr(), _row_stride(x.q), x.scale.data_ptr(), w.q.data_ptr(),
          _row_stride(w.q), w.scale.data_ptr(), dx.data_ptr(), cols, dw.data_ptr(), cols, db.data_ptr(), _ptr(room), 0 if room is None else room.numel(), _stream())
    return (dx.view(*shape[:-1], cols) if len(shape) != 2 else dx), dw, db
