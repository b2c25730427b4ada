"""CPU-only checks of products in 8-bit floats and of the update: what the C calls refuse before anything is launched, what the Python entry points refuse, the definition of
the hash by which moments are rounded."""

import ctypes

import pytest
import torch

from f8_reference import at_random, random_bits
from paper_1803_03288_amd import binding, build as build_mod, layers

P = 4096            # a pointer that is aligned and never followed: the call is refused first, or has nothing to do
I32, I64, PTR, SIZE, F32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_float


class Float8(ctypes.Structure):
    _fields_ = [("q", PTR), ("ld", I64), ("scale", PTR), ("ld_scale", I64), ("format", I32), ("block", I32)]


class Gradient(ctypes.Structure):
    _fields_ = [("g", PTR), ("numel", I64), ("dtype", I32)]


class Tensor(ctypes.Structure):
    _fields_ = [("p", PTR), ("g", PTR), ("m", PTR), ("v", PTR), ("m_scale", PTR), ("v_scale", PTR), ("copy", PTR), ("numel", I64), ("dtype", I32), ("grad_dtype", I32), ("copy_dtype", I32)]


class Options(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in ("lr", "beta1", "beta2", "eps", "weight_decay")] + [("step", I64), ("seed", ctypes.c_uint64), ("grad_scale", F32), ("max_norm", F32),
                                                                                                ("norm", PTR), ("lr_at", PTR), ("step_at", PTR)]


SIGNATURES = {
    "tictac_quantize_f8": (I32, I64, I64, PTR, I64, PTR, PTR), "tictac_dequantize_f8": (I32, I64, I64, PTR, PTR, I64, PTR),
    "tictac_linear_f8_workspace": (I32, I32, I64, I64, I64, PTR), "tictac_linear_f8": (I32, I64, I64, I64, PTR, I64, PTR, PTR, I32, PTR, PTR, I64, PTR, SIZE, PTR),
    "tictac_linear_f8_backward_workspace": (I32, I64, I64, I64, PTR),
    "tictac_linear_f8_backward": (I32, I64, I64, I64, PTR, I64, I32, PTR, PTR, PTR, I64, PTR, I64, PTR, PTR, SIZE, PTR),
    "tictac_gradient_norm_workspace": (I32, PTR), "tictac_gradient_norm": (I32, PTR, F32, PTR, PTR, SIZE, PTR), "tictac_adamw_step": (I32, PTR, PTR, PTR),
}


@pytest.fixture(scope="module", autouse=True)
def built():
    import os
    if not (os.path.exists(binding.LIB_PATH) and os.path.exists(build_mod.LAYERS)):
        build_mod.build()


def code(name, *args):
    rc = ctypes.CFUNCTYPE(I32, *SIGNATURES[name])((name, binding.lib()))(*args)
    if rc:
        assert binding.lib().tictac_last_error()            # with a message
    return rc


def f8(q=P, ld=256, scale=P, ld_scale=4, format=0, block=1):
    return Float8(q, ld, scale, ld_scale, format, block)


BAD_F8 = [({"q": None}, -1), ({"scale": None}, -1), ({"ld": 200}, -9), ({"ld": 128}, -9), ({"ld_scale": 2}, -9), ({"ld_scale": 6}, -9), ({"format": 2}, -9), ({"format": -1}, -9), ({"block": 0}, -9),
          ({"block": 64}, -9), ({"q": P + 8}, -9), ({"scale": P + 2}, -9)]


def quantize(to=None, **changed):
    a = dict(dtype=2, rows=4, cols=200, x=P, ld_x=200, stream=None)
    a.update(changed)
    to = ctypes.addressof(to) if to is not None else None
    return code("tictac_quantize_f8", a["dtype"], a["rows"], a["cols"], a["x"], a["ld_x"], to, a["stream"])


def dequantize(r=None, **changed):
    a = dict(dtype=2, rows=4, cols=200, x=P, ld_x=200)
    a.update(changed)
    return code("tictac_dequantize_f8", a["dtype"], a["rows"], a["cols"], ctypes.addressof(r) if r is not None else None, a["x"], a["ld_x"], None)


def linear(x8=None, w=None, **changed):
    a = dict(dtype=2, rows=100, cols=200, outs=50, x=P, ld_x=200, bias_dtype=0, bias=P, y=P, ld_y=50, workspace=P, bytes=1 << 30)
    a.update(changed)
    return code("tictac_linear_f8", a["dtype"], a["rows"], a["cols"], a["outs"], a["x"], a["ld_x"], ctypes.addressof(x8) if x8 is not None else None, ctypes.addressof(w) if w is not None else None,
                a["bias_dtype"], a["bias"], a["y"], a["ld_y"], a["workspace"], a["bytes"], None)


def backward(x8=None, w=None, **changed):
    a = dict(dtype=2, rows=100, cols=200, outs=50, dy=P, ld_dy=50, format=0, dx=P, ld_dx=200, dw=P, ld_dw=200, db=P, workspace=P, bytes=1 << 30)
    a.update(changed)
    return code("tictac_linear_f8_backward", a["dtype"], a["rows"], a["cols"], a["outs"], a["dy"], a["ld_dy"], a["format"], ctypes.addressof(x8) if x8 is not None else None,
                ctypes.addressof(w) if w is not None else None, a["dx"], a["ld_dx"], a["dw"], a["ld_dw"], a["db"], a["workspace"], a["bytes"], None)


@pytest.mark.parametrize("changed,want", BAD_F8)
def test_operands_that_are_refused(changed, want):
    bad = f8(**changed)
    assert quantize(bad) == want
    assert dequantize(bad) == want
    assert linear(None, bad) == want
    assert linear(bad, f8(), x=None) == want
    assert backward(bad, f8()) == want
    assert backward(f8(), bad) == want


@pytest.mark.parametrize("changed,want", [({"dtype": 3}, -9), ({"rows": -1}, -9), ({"cols": 0}, -9), ({"x": None}, -1), ({"x": P + 1}, -9), ({"ld_x": -1}, -9)])
def test_blocks_that_are_refused(changed, want):
    assert quantize(f8(), **changed) == want
    assert dequantize(f8(), **changed) == want
    assert quantize(None) == dequantize(None) == -1
    assert quantize(f8(ld=1 << 30, ld_scale=1 << 23, block=128), rows=1 << 20, cols=1 << 30) == -9
    assert dequantize(f8(), ld_x=199) == -9


@pytest.mark.parametrize("changed,want", [({"dtype": 5}, -9), ({"cols": 131073}, -9), ({"rows": (1 << 21) + 1}, -9), ({"outs": -1}, -9), ({"x": None}, -1), ({"bias_dtype": 7}, -9), ({"y": None}, -1),
                                          ({"ld_y": 49}, -9), ({"workspace": None}, -1), ({"workspace": P + 8}, -9), ({"bytes": 10}, -8), ({"bias": P + 1}, -9)])
def test_products_that_are_refused(changed, want):
    assert linear(None, f8(), **changed) == want


@pytest.mark.parametrize("changed,want", [({"dtype": 5}, -9), ({"dy": None}, -1), ({"format": 3}, -9), ({"ld_dx": 199}, -9), ({"ld_dw": 100}, -9), ({"db": P + 1}, -9), ({"workspace": None}, -1), ({"bytes": 99}, -8),
                                          ({"rows": 1 << 21, "outs": 1 << 20}, -9)])
def test_gradients_that_are_refused(changed, want):
    assert backward(f8(), f8(), **changed) == want


def test_more_refusals_and_nothing_to_do():
    assert linear(f8(), f8()) == -9                         # both x and x8
    assert linear(None, f8(format=1)) == -9 and backward(f8(), f8(format=1)) == -9           # weights are e4m3
    assert linear(None, f8(ld=1 << 25)) == -9
    assert linear(None, None) == backward(None, f8()) == backward(f8(), None) == -1
    assert quantize(None, rows=0, x=None) == dequantize(None, rows=0, x=None) == linear(None, None, rows=0, x=None) == linear(None, None, outs=0) == 0
    assert backward(None, None, dx=None, dw=None, db=None) == 0
    n = ctypes.c_size_t(7)
    at = ctypes.addressof(n)
    assert code("tictac_linear_f8_workspace", 2, 1, 1000, 4096, 4096, at) == 0 and n.value >= 1000 * (4096 + 32)
    assert code("tictac_linear_f8_workspace", 0, 0, 1000, 4096, 4096, at) == 0 and n.value >= 2 * 4096 * (1000 + 4096)
    assert code("tictac_linear_f8_workspace", 2, 1, 1000, 0, 4096, at) == -9
    assert code("tictac_linear_f8_workspace", 2, 1, 1000, 10, 4096, None) == -1
    assert code("tictac_linear_f8_backward_workspace", 1, 0, 10, 10, at) == 0 and n.value == 0
    assert code("tictac_linear_f8_backward_workspace", 1, 100, 10, 10, None) == -1
    assert code("tictac_gradient_norm_workspace", 3, at) == 0 and n.value >= 8
    assert code("tictac_gradient_norm_workspace", -1, at) == code("tictac_gradient_norm_workspace", 1 << 24, at) == -9 and code("tictac_gradient_norm_workspace", 1, None) == -1


@pytest.mark.parametrize("changed,want", [({"n": -1}, -9), ({"n": 1 << 24}, -9), ({"numel": (1 << 37) + 1}, -9), ({"list": None}, -1), ({"norm": None}, -1), ({"norm": P + 2}, -9), ({"scale": float("nan")}, -9), ({"scale": float("inf")}, -9), ({"g": None}, -1),
                                          ({"g": P + 2}, -9), ({"numel": -1}, -9), ({"dtype": 4}, -9), ({"workspace": None}, -1), ({"bytes": 7}, -8)])
def test_norms_that_are_refused(changed, want):
    a = dict(n=1, list=P, scale=1.0, norm=P, workspace=P, bytes=1 << 20, g=P, numel=100, dtype=0)
    a.update(changed)
    one = Gradient(a["g"], a["numel"], a["dtype"])
    assert code("tictac_gradient_norm", a["n"], a["list"] and ctypes.addressof(one), a["scale"], a["norm"], a["workspace"], a["bytes"], None) == want


def adamw(tensors=None, **changed):
    tensor = dict(p=0x10000, g=0x20000, m=0x30000, v=0x40000, m_scale=None, v_scale=None, copy=None, numel=1000, dtype=0, grad_dtype=0, copy_dtype=0)
    options = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, step=1, seed=0, grad_scale=1.0, max_norm=1.0, norm=None, lr_at=None, step_at=None)
    for k, v in changed.items():
        (tensor if k in tensor else options)[k] = v
    tensors = [tensor] if tensors is None else [dict(tensor, **t) for t in tensors]
    all_ = (Tensor * max(1, len(tensors)))(*[Tensor(**t) for t in tensors])
    o = Options(**options)
    return code("tictac_adamw_step", len(tensors), ctypes.addressof(all_), ctypes.addressof(o), None)


NAN = float("nan")


@pytest.mark.parametrize("changed,want", [
    ({"lr": NAN}, -9), ({"beta1": 1.0}, -9), ({"beta1": -0.1}, -9), ({"beta2": 1.5}, -9), ({"beta2": NAN}, -9), ({"eps": -1e-8}, -9), ({"eps": NAN}, -9), ({"weight_decay": float("inf")}, -9),
    ({"grad_scale": NAN}, -9), ({"step": 0}, -9), ({"norm": P, "max_norm": 0.0}, -9), ({"norm": P, "max_norm": NAN}, -9), ({"norm": P + 1}, -9), ({"lr_at": P + 1}, -9), ({"step_at": P + 4}, -9),
    ({"p": None}, -1), ({"g": None}, -1), ({"m": None}, -1), ({"v": None}, -1), ({"p": 0x10002}, -9), ({"dtype": 3}, -9), ({"grad_dtype": -1}, -9), ({"copy": 0x50000, "copy_dtype": 9}, -9),
    ({"numel": -5}, -9), ({"numel": (1 << 32) + 1}, -9), ({"m_scale": 0x50000}, -9), ({"m_scale": 0x50000, "v_scale": 0x50002}, -9), ({"m_scale": 0x50000, "v_scale": 0x60000, "m": 0x30008}, -9),
    ({"copy": 0x10000}, -9), ({"copy": 0x10f9c}, -9), ({"m": 0x20000}, -9), ({"v": 0x30000}, -9), ({"g": 0x10000}, -9),
])
def test_updates_that_are_refused(changed, want):
    assert adamw(**changed) == want


def test_tensors_that_overlap():
    apart = dict(p=0x110000, g=0x120000, m=0x130000, v=0x140000)
    assert adamw([{}, {}]) == -9                            # the same tensor twice
    assert adamw([{}, dict(apart, m=0x10000 + 3996)]) == -9
    assert adamw([{}, dict(apart, g=0x10000)]) == -9
    # 8 bits: rows are written up to the next multiple of 128
    assert adamw([{}, dict(apart, m_scale=0x150000, v_scale=0x160000, m=0x10000 - 1008)]) == -9
    assert adamw([]) == 0 and adamw([{"numel": 0, "p": None}]) == 0
    assert code("tictac_adamw_step", 1, None, P, None) == -1 and code("tictac_adamw_step", 0, None, None, None) == -1


def test_tensors_that_are_refused():
    x = torch.ones(4, 256)
    q = torch.zeros(4, 256, dtype=torch.uint8).view(torch.float8_e4m3fn)
    r = layers.Float8(q, torch.ones(4, 4, dtype=torch.uint8).view(torch.float8_e8m0fnu), 256)
    m = layers.adamw_moments([x], 32)
    for call in (lambda: layers.quantize_f8(x), lambda: layers.dequantize_f8(r), lambda: layers.linear_f8(x, r), lambda: layers.linear_f8(r, r), lambda: layers.linear_f8_backward(x, r, r),
                 lambda: layers.gradient_norm([x]), lambda: layers.gradient_norm([]), lambda: layers.adamw_step([x], [x], m, 1), lambda: layers.adamw_step([x], [], m, 1),
                 lambda: layers.adamw_moments([x], 16)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: layers.dequantize_f8(r, torch.float64), lambda: layers.gradient_norm(x), lambda: layers.adamw_step(x, [x], m, 1), lambda: layers.adamw_step([x], [x], m, "1")):
        with pytest.raises(TypeError):
            call()
    assert r.shape == (4, 256)


def test_moments_of_zeros():
    p = [torch.ones(3, 700), torch.ones(0), torch.ones(())]
    for bits in (8, 32):
        m = layers.adamw_moments(p, bits)
        assert len(m) == 3
        if bits == 32:
            assert [t.m.shape for t in m] == [(2100,), (0,), (1,)] and not m[0].v.any()
        else:
            assert m[0].m.shape == (1, 2100) and m[0].m.q.shape == (1, 2176) and m[0].m.scale.shape == (1, 20) and not m[0].v.q.view(torch.uint8).any()
            assert m[2].m.scale.shape == (1, 4)


def test_hash_has_no_preference():
    """The random halves of neighbours, of tensors and of steps: means within five standard deviations, no correlation beyond it."""
    n = 1 << 16
    halves = [h.double() / 65536 for seed, step, index in ((0, 1, 0), (0, 1, 1), (0, 2, 0), (1 << 40, 1, 0)) for b in (random_bits(seed, step, index, n),) for h in (b & 0xFFFF, b >> 16)]
    for i, a in enumerate(halves):
        assert abs(float(a.mean()) - 0.5) < 5 / (12 * n) ** 0.5
        for b in halves[:i] + [a.roll(1), a.roll(2), a.roll(128)]:
            assert abs(float(((a - 0.5) * (b - 0.5)).mean())) < 5 / 12 / n ** 0.5


def test_rounding_at_random_is_fair():
    """Values between two of e4m3 are rounded to either, by their distance; those of the type stay."""
    n = 1 << 14
    for x in (3.3, -0.7, 1.0, 447.9, 2.0 ** -8 * 1.3):
        row = torch.full((n,), x)
        row[::128] = 448.0                                  # a scale of one
        q, byte = at_random(row, random_bits(3, 7, 0, n) & 0xFFFF)
        q, found = q[1::128], set(q[1::128].tolist())
        assert len(found) <= 2 and set(byte.tolist()) == {127}
        low, high = min(found), max(found)
        assert low <= x + 1e-6 and high >= x - 1e-6
        assert abs(float(q.mean()) - x) <= 5 * (high - low) * 0.5 / len(q) ** 0.5 + 1e-6
