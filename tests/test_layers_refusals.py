"""CPU-only checks of the layers' operators: what the C calls refuse before anything is launched, and what the Python entry
points refuse before the library is called."""

import ctypes

import pytest
import torch

from layer_calls import call
from paper_1803_03288_amd import binding, build as build_mod, layers

P = 4096            # a pointer that is aligned and never followed: the call is refused first, or has nothing to do


@pytest.fixture(scope="module", autouse=True)
def built():
    import os
    if not (os.path.exists(binding.LIB_PATH) and os.path.exists(build_mod.LAYERS)):
        build_mod.build()


def code(name, *args):
    try:
        call(name, *args)
    except binding.TicTacError as e:
        assert str(e).split(": ", 1)[1]                     # with a message
        return e.code
    return 0


QUANTIZE = ("tictac_quantize_rows", [2, 4, 200, P, 200, 0, P, 256, P, None])
DEQUANTIZE = ("tictac_dequantize_rows", [2, 4, 200, P, 256, P, 0, P, 200, None])
NORM = ("tictac_layer_norm", [2, 4, 200, P, 200, 0, P, P, 1e-5, P, 200, P, P, P, 256, P, P, 256, P, None])
NORM_BACK = ("tictac_layer_norm_backward", [2, 5000, 200, P, 200, P, 200, None, 0, None, 0, P, P, P, P, 200, P, P, P, 1 << 22, None])
LINEAR = ("tictac_linear_q8", [2, 100, 200, 50, P, 200, None, 0, None, P, 256, P, 0, P, P, 50, P, 1 << 30, None])
LINEAR_BACK = ("tictac_linear_q8_backward", [2, 100, 200, 50, P, 50, P, 256, P, P, 256, P, P, 200, P, 200, P, P, 1 << 30, None])


@pytest.mark.parametrize("call,at,value,want", [
    (QUANTIZE, 0, 3, -9), (QUANTIZE, 1, -1, -9), (QUANTIZE, 2, 0, -9), (QUANTIZE, 3, None, -1), (QUANTIZE, 3, P + 1, -9), (QUANTIZE, 4, -200, -9),
    (QUANTIZE, 5, 64, -9), (QUANTIZE, 6, None, -1), (QUANTIZE, 6, P + 8, -9), (QUANTIZE, 7, 200, -9), (QUANTIZE, 7, 128, -9), (QUANTIZE, 8, None, -1),
    (DEQUANTIZE, 0, -1, -9), (DEQUANTIZE, 3, None, -1), (DEQUANTIZE, 4, 255, -9), (DEQUANTIZE, 5, P + 2, -9), (DEQUANTIZE, 6, 1, -9), (DEQUANTIZE, 7, None, -1),
    (DEQUANTIZE, 8, 199, -9),
    (NORM, 0, 9, -9), (NORM, 5, 4, -9), (NORM, 2, 0, -9), (NORM, 3, None, -1), (NORM, 8, -1.0, -9), (NORM, 8, float("nan"), -9), (NORM, 10, 100, -9),
    (NORM, 11, None, -1), (NORM, 12, None, -1), (NORM, 13, None, -1), (NORM, 14, 200, -9), (NORM, 18, None, -1), (NORM, 6, P + 2, -9),
    (NORM_BACK, 3, None, -1), (NORM_BACK, 5, None, -1), (NORM_BACK, 7, P, -9), (NORM_BACK, 12, None, -1), (NORM_BACK, 13, None, -1), (NORM_BACK, 15, 3, -9),
    (NORM_BACK, 18, None, -1), (NORM_BACK, 18, P + 16, -9), (NORM_BACK, 19, 1, -8),
    (LINEAR, 2, 131073, -9), (LINEAR, 1, (1 << 21) + 1, -9), (LINEAR, 3, -1, -9), (LINEAR, 4, None, -1), (LINEAR, 6, P, -9), (LINEAR, 9, None, -1),
    (LINEAR, 10, 1 << 25, -9), (LINEAR, 10, 130, -9), (LINEAR, 12, 5, -9), (LINEAR, 14, None, -1), (LINEAR, 15, 49, -9), (LINEAR, 16, None, -1), (LINEAR, 17, 10, -8),
    (LINEAR_BACK, 0, 3, -9), (LINEAR_BACK, 4, None, -1), (LINEAR_BACK, 6, None, -1), (LINEAR_BACK, 7, 100, -9), (LINEAR_BACK, 9, None, -1), (LINEAR_BACK, 13, 5, -9),
    (LINEAR_BACK, 15, 5, -9), (LINEAR_BACK, 16, P + 1, -9), (LINEAR_BACK, 17, None, -1), (LINEAR_BACK, 18, 100, -8),
])
def test_arguments_that_are_refused(call, at, value, want):
    name, args = call
    args = list(args)
    args[at] = value
    assert code(name, *args) == want


def test_nothing_to_do():
    for (name, args), rows in ((QUANTIZE, 1), (DEQUANTIZE, 1), (NORM, 1), (LINEAR, 1)):
        args = [None if a == P else a for a in args]
        args[rows] = 0
        assert code(name, *args) == 0
    assert code("tictac_linear_q8", *[0 if i == 3 else a for i, a in enumerate(LINEAR[1])]) == 0
    assert code("tictac_layer_norm_backward", *[None if i in (14, 16, 17) else a for i, a in enumerate(NORM_BACK[1])]) == 0
    assert code("tictac_linear_q8_backward", *[None if i in (12, 14, 16) else a for i, a in enumerate(LINEAR_BACK[1])]) == 0


def test_workspaces():
    n = ctypes.c_size_t(7)
    at = ctypes.addressof(n)
    call("tictac_layer_norm_backward_workspace", 0, 100, at)
    assert n.value == 0
    call("tictac_layer_norm_backward_workspace", 5000, 100, at)
    assert n.value >= 2 * 100 * 4
    call("tictac_linear_q8_workspace", 0, 1, 4096, 4096, at)
    few = n.value
    call("tictac_linear_q8_workspace", 1, 1000, 4096, 4096, at)
    assert n.value >= 1000 * (4096 + 4) > few
    assert code("tictac_linear_q8_workspace", 1, 1000, 0, 4096, at) == -9
    assert code("tictac_linear_q8_workspace", 1, 1000, 10, 4096, None) == -1
    assert code("tictac_linear_q8_backward_workspace", 7, 1000, 10, 4096, at) == -9
    assert code("tictac_layer_norm_backward_workspace", -1, 10, at) == -9


def test_tensors_that_are_refused():
    x = torch.ones(4, 256)
    r = layers.Rows8(torch.zeros(4, 256, dtype=torch.int8), torch.ones(4, 1), 256)
    for call in (lambda: layers.quantize_rows(x), lambda: layers.layer_norm(x), lambda: layers.layer_norm_q8(x), lambda: layers.linear_q8(x, r), lambda: layers.linear_q8(r, r),
                 lambda: layers.layer_norm_backward(x, x, None, x[:, 0], x[:, 0]), lambda: layers.linear_q8_backward(x, r, r), lambda: layers.dequantize_rows(r),
                 lambda: layers.quantize_rows(x, 32)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        layers.dequantize_rows(r, torch.float64)
    assert r.shape == (4, 256)
