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
Everything runs on the current stream; there is no CPU fallback.  There is no autograd either: outputs carry no graph, also where an input requires a
gradient, and the backward passes are calls of their own, to be made by hand or from a ``torch.autograd.Function``.  A wrong argument raises ``ValueError`` or ``TypeError``, what the library
refuses ``TicTacError``.
"""

from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional, Union

import torch

from .binding import _check, lib

GROUP = 128                     # columns per scale of kept activations
_CALLS = ("quantize_rows", "dequantize_rows", "layer_norm", "layer_norm_backward_workspace", "layer_norm_backward", "linear_q8_workspace", "linear_q8",
          "linear_q8_backward_workspace", "linear_q8_backward")
_module = None


def _native():
    """The compiled half of this module (``csrc/layers_binding.cpp``): it checks tensors, allocates outputs and workspaces and makes the C calls."""
    global _module
    if _module is None:
        library = lib()                             # (raises where the library has not been built)
        from . import _layers
        _layers.init(tuple(ctypes.cast(getattr(library, "tictac_" + name), ctypes.c_void_p).value for name in _CALLS), _check, torch.OutOfMemoryError)
        _module = _layers
    return _module


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


def quantize_rows(x: torch.Tensor, group: int = 0) -> Rows8:
    """``x`` in 8 bits.  ``group`` 0: a scale per row (weights by output channel, operands of products); 128: one per 128 columns
    (activations kept for the backward pass).  A row (group) with a NaN or an infinity reads as NaN throughout."""
    q, scale = (_module or _native()).quantize_rows(x, group)
    return Rows8(q, scale, x.shape[-1], group)


def dequantize_rows(r: Rows8, dtype: torch.dtype = torch.float32) -> torch.Tensor:
    """The values of 8-bit rows, ``[rows][cols]``, rounded to ``dtype``."""
    return (_module or _native()).dequantize_rows(r, dtype)


def layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, eps: float = 1e-5, save: bool = False):
    """``(y, mean, rstd)`` of layer norm over the last dimension; with ``save`` also ``x`` as 8-bit rows of group 128 for the backward
    pass, from the same read of ``x``.  ``weight`` and ``bias`` in float32 or the type of ``x``; ``mean`` and ``rstd`` float32 ``[rows]``."""
    if not save:
        return (_module or _native()).layer_norm(x, weight, bias, eps, False, False)
    y, mean, rstd, q, scale = (_module or _native()).layer_norm(x, weight, bias, eps, False, True)
    return y, mean, rstd, Rows8(q, scale, x.shape[-1], GROUP)


def layer_norm_q8(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, eps: float = 1e-5, save: bool = False):
    """``(y8, mean, rstd)``: layer norm whose output is 8-bit rows, formed from its float32 values, the operand of ``linear_q8``; ``save`` as in ``layer_norm``."""
    if not save:
        q, scale, mean, rstd = (_module or _native()).layer_norm(x, weight, bias, eps, True, False)
        return Rows8(q, scale, x.shape[-1]), mean, rstd
    q, scale, mean, rstd, xq, xs = (_module or _native()).layer_norm(x, weight, bias, eps, True, True)
    return Rows8(q, scale, x.shape[-1]), mean, rstd, Rows8(xq, xs, x.shape[-1], GROUP)


def layer_norm_backward(dy: torch.Tensor, x: Union[torch.Tensor, Rows8], weight: Optional[torch.Tensor], mean: torch.Tensor, rstd: torch.Tensor):
    """``(dx, dweight, dbias)`` of layer norm from its input, or from the 8-bit rows (group 128) that the forward pass saved.
    ``dweight`` and ``dbias`` have the type of ``weight`` (float32 without one)."""
    return (_module or _native()).layer_norm_backward(dy, x, weight, mean, rstd)


def linear_q8(x: Union[torch.Tensor, Rows8], w: Rows8, bias: Optional[torch.Tensor] = None, dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """``x @ w.T + bias`` with both operands in 8 bits, ``w`` ``[outs][cols]`` with a scale per output, sums exact.  ``x`` is rounded to 8 bits, a scale
    per row, in the call, unless it is given as ``Rows8``; then ``dtype`` is the output's type (float32 unless given)."""
    return (_module or _native()).linear_q8(x, w, bias, dtype)


def linear_q8_backward(dy: torch.Tensor, x: Rows8, w: Rows8):
    """``(dx, dw, db)`` of ``linear_q8`` from the 8-bit rows that the forward pass took, all of the type of ``dy``; the rounding of the
    input counts as the identity.  The products are of bfloat16 values with sums in float32: ``dy`` times a scale takes three of them for float32 (exact) and
    two for float16, but for bfloat16 one factor of each term is rounded to 8 bits (up to 2^-8 of it, beside the rounding of the outputs); ``dy`` in
    float32 avoids that."""
    return (_module or _native()).linear_q8_backward(dy, x, w)
