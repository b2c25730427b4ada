"""Every kernel of the products in 8-bit floats and of the update, by the sizes at which it is chosen, against the definition in 64 bits.

Each case names the kernels that it stands for, and the profiler says which ones ran.  Bounds are those of ``test_gpu_f8``; the definition is computed on the GPU in float64 from the
8-bit operands (their rounding is compared bit by bit there)."""

import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import f8_reference as ref
from test_gpu_f8 import BF16, E4, E5, F16, F32, HALF, L  # noqa: F401
from test_gpu_layer_paths import JOIN, kernels, ran

ONCE, DX, DW = "linear_f8_once_kernel<{dt}, {wide}>", "linear_f8_dx_few_kernel", "linear_f8_dw_few_kernel"
S64, S128X64, S128, S128DEEP, S256 = "product_f8_kernel<{f}, {dt}, 1, 1, 4>", "product_f8_kernel<{f}, {dt}, 2, 1, 3>", "product_f8_kernel<{f}, {dt}, 2, 2, 2>", "product_f8_kernel<{f}, {dt}, 2, 2, 4>", "product_f8_kernel_256<{f}, {dt}>"
WIDEN, EXACT64, EXACT128X64, EXACT256 = "widen_f8_kernel", "product_kernel<OpBf16Biased, 0, 2, 2, 4>", "product_kernel<OpBf16Biased, 0, 4, 2, 3>", "product_kernel_256<OpBf16Biased, 0>"
BACK64, BACK128X64, BACK128, BACK256 = "product_kernel<OpBf16, 0, 2, 2, 4>", "product_kernel<OpBf16, 0, 4, 2, 3>", "product_kernel<OpBf16, 0, 4, 4, 2>", "product_kernel_256<OpBf16, 0>"
DT = {F32: 0, F16: 1, BF16: 2}


def named(want, dtype, f8=E4, wide=True):
    return [w.format(dt=DT[dtype], f=int(f8 == E5), wide=str(wide).lower()) for w in want]


def operand(r):
    """(q, scale, least exponent) of a Float8 on the GPU in float64."""
    rows = r.q.shape[0]
    scale = torch.ldexp(torch.ones((), dtype=torch.float64, device="cuda"), r.scale.view(torch.uint8)[:, :-(-r.cols // 128)].to(torch.int32) - 127)
    return r.q[:, :r.cols].double(), scale.repeat_interleave(r.block, 0)[:rows].repeat_interleave(128, 1)[:, :r.cols], ref.F8[r.q.dtype][1]


def turned(L, r):  # noqa: F811
    """The same values in blocks along the rows: the operand of a gradient."""
    q, s, _ = operand(r)
    return operand(L.quantize_f8((q * s).float().t().contiguous()))


def close(got, want, bound, dtype):
    rel, least = HALF[dtype]
    assert got.shape == want.shape and bool(torch.isfinite(got).all())
    off = (got.double() - want).abs() - (bound + rel * (want.abs() + bound) + least)
    assert float(off.max()) <= 0, float(off.max())


def random(g, rows, cols, dtype, scale=1.0):
    return (torch.randn(rows, cols, generator=g, device="cuda") * torch.exp(0.5 * torch.randn(rows, 1, generator=g, device="cuda")) * scale).to(dtype)


# rows, columns, outputs, type of input and output, kernels (from floats)
FORWARD = [
    (4, 4096, 8000, BF16, [ONCE]), (4, 4096, 4000, F32, [ONCE]), (16, 2040, 4000, F16, [ONCE]), (4, 4097, 300, F32, [ONCE]), (2, 520, 100, F16, [ONCE]), (16, 2048, 1000, BF16, [ONCE]), (1, 32768, 30, BF16, [ONCE]),
    (16, 2050, 2100, BF16, ["few_kernel<false, 0, 1, 1>"]), (8, 8192, 2100, F16, ["few_kernel<false, 0, 1, 1>", JOIN]), (12, 4096, 4096, BF16, ["few_kernel<false, 0, 1, 1>"]),
    (16, 2048, 17000, BF16, ["few_kernel<false, 0, 1, 2>", JOIN]), (9, 20000, 3001, F16, ["few_kernel<false, 0, 1, 2>", JOIN]), (20, 500, 1030, BF16, ["few_kernel<false, 0, 2, 1>"]),
    (27, 4096, 1001, F16, ["few_kernel<false, 0, 2, 1>", JOIN]), (50, 3000, 1001, BF16, ["few_kernel<false, 0, 4, 1>", JOIN]), (61, 520, 8000, F16, ["few_kernel<false, 0, 4, 1>"]),
    (16, 2050, 2100, F32, ["few_kernel<true, 0, 1, 1>"]), (5, 8192, 60, F32, ["few_kernel<true, 0, 1, 1>", JOIN]), (16, 2048, 17000, F32, ["few_kernel<true, 0, 1, 2>", JOIN]), (20, 500, 1030, F32, ["few_kernel<true, 0, 2, 1>"]),
    (27, 8192, 4101, F32, ["few_kernel<true, 0, 2, 4>", JOIN]), (50, 3000, 1999, F32, ["few_kernel<true, 0, 4, 1>", JOIN]), (64, 8192, 4100, F32, ["few_kernel<true, 0, 4, 4>", JOIN]),
    (20, 20000, 1030, F16, [S64, JOIN]), (32, 2048, 9000, F16, [S64]), (64, 4096, 4096, F16, [S64, JOIN]), (17, 4096, 1999, BF16, [S64, JOIN]), (16, 4096, 17000, BF16, [S64]),
    (100, 777, 1001, F16, [S64]), (130, 4096, 2000, BF16, [S128X64, JOIN]), (130, 4100, 2001, F16, [S128X64, JOIN]), (1000, 520, 2000, BF16, [S128X64]), (1024, 8192, 2048, F16, [S128X64]), (1024, 512, 4096, F16, [S128X64]),
    (2048, 4096, 2048, F16, [S128DEEP]), (1000, 2000, 5000, BF16, [S128]), (1800, 600, 2301, BF16, [S128]), (2100, 100, 2060, F16, [S128]),
    # more tiles than compute units, of which the last ones are not whole; one step, few, an odd number of them
    (8192, 512, 16384, F16, [S256]), (8192, 128, 16384, BF16, [S256]), (16000, 300, 16104, BF16, [S256]), (16000, 300, 16101, BF16, [S256]), (16000, 200, 16101, F16, [S256]),
    (100, 777, 1001, F32, [WIDEN, EXACT64]), (1500, 300, 1501, F32, [WIDEN, EXACT128X64]), (8192, 512, 16384, F32, [WIDEN, EXACT256]),
]


@pytest.mark.parametrize("rows,cols,outs,dtype,want", FORWARD)
def test_products(L, rows, cols, outs, dtype, want):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(rows + cols + outs)
    x, w = random(g, rows, cols, dtype), L.quantize_f8(random(g, outs, cols, F32, cols ** -0.5), 128 if outs % 4 == 0 else 1)
    bias = torch.randn(outs, generator=g, device="cuda")
    print(rows, cols, outs, dtype, flush=True)
    names, got = kernels(lambda: L.linear_f8(x, w, bias))
    ran(names, named(want, dtype, wide=cols % 8 == 0))
    part, bound = ref.product(operand(L.quantize_f8(x)), operand(w), dtype != F32)
    close(got, part + bias.double(), bound + 2 * ref.U * (part.abs() + bias.double().abs()), dtype)
    del part, bound
    other = random(g, rows, cols, dtype)
    for _ in range(4):                                      # (nothing waits between them)
        L.linear_f8(other, w, bias)
        assert torch.equal(L.linear_f8(x, w, bias), got)


@pytest.mark.parametrize("rows,cols,outs,dtype,want", [(9, 3000, 1001, BF16, ["few_kernel<false, 1, 1, 1>"]), (12, 8192, 4101, BF16, ["few_kernel<false, 1, 1, 2>"]), (30, 3000, 1001, F16, ["few_kernel<false, 1, 2, 1>"]),
                                                       (64, 500, 2100, F16, ["few_kernel<false, 1, 4, 1>"]), (12, 8192, 4101, F32, ["few_kernel<true, 1, 1, 2>"]), (30, 3000, 2100, F32, ["few_kernel<true, 1, 2, 1>"]),
                                                       (30, 8192, 4101, F32, ["few_kernel<true, 1, 2, 4>"]), (60, 8192, 4101, F32, ["few_kernel<true, 1, 4, 4>"]), (50, 2000, 1999, F32, ["few_kernel<true, 1, 4, 1>"]),
                                                       (100, 777, 1001, F16, [S64]), (2100, 100, 2060, BF16, [S128]), (2048, 4096, 2048, BF16, [S128DEEP]), (1024, 8192, 2048, F16, [S128X64]), (8192, 300, 16104, F16, [S256]), (100, 777, 1001, F32, [WIDEN, EXACT64])])
def test_products_of_the_wider_range(L, rows, cols, outs, dtype, want):  # noqa: F811
    """Inputs in float8_e5m2, rounded before."""
    g = torch.Generator(device="cuda").manual_seed(rows + cols + outs)
    x, w = L.quantize_f8(random(g, rows, cols, F32), 1, E5), L.quantize_f8(random(g, outs, cols, F32, cols ** -0.5), 128)
    print(rows, cols, outs, dtype, flush=True)
    names, got = kernels(lambda: L.linear_f8(x, w, None, dtype))
    if JOIN not in want and any(JOIN in n for n in names):
        want = want + [JOIN]                                # (cuts along k are tested above)
    ran(names, named(want, dtype, E5))
    close(got, *ref.product(operand(x), operand(w), dtype != F32), dtype)


# rows, columns, outputs, type, rows per block of the weights, type of 8 bits of dy, kernels
BACKWARD = [
    (5, 4096, 9000, F16, 128, E4, [DX + "<0, 1>", JOIN, DW + "<0, 1, true>"]), (20, 2000, 9001, BF16, 128, E4, [DX + "<0, 2>", JOIN, DW + "<0, 2, true>"]), (30, 3001, 2801, BF16, 128, E5, [DX + "<1, 2>", JOIN, DW + "<1, 2, false>"]),
    (16, 4100, 2050, F16, 128, E5, [DX + "<1, 1>", JOIN, DW + "<1, 1, false>"]), (1, 8192, 1024, BF16, 128, E4, [DX + "<0, 1>", DW + "<0, 2, true>"]), (32, 8197, 1030, F16, 128, E4, [DX + "<0, 2>", DW + "<0, 1, false>"]),
    (5, 4096, 9000, F16, 1, E4, [S128X64, JOIN, DW]), (30, 3001, 2801, BF16, 1, E4, [S64, JOIN, DW]), (64, 5800, 5801, BF16, 128, E5, [S64, JOIN, DW + "<1, 2, true>"]), (100, 4100, 8195, F16, 128, E4, [S128X64, JOIN, DW + "<0, 1, false>"]),
    (128, 8192, 4096, BF16, 1, E5, [S64, DW + "<1, 2, true>"]), (64, 2104, 9000, F16, 128, E4, [S128, JOIN]), (30, 500, 300, BF16, 128, E5, [S64]), (1, 500, 300, F16, 128, E4, [S64]), (120, 3000, 4100, F16, 128, E4, [S128, JOIN]),
    (130, 264, 640, F16, 128, E4, [S64]), (1030, 190, 2070, BF16, 1, E5, [S64]), (300, 1000, 1024, BF16, 128, E4, [S64]), (1500, 1100, 2051, F16, 128, E5, [S128]), (700, 2000, 900, F16, 128, E4, [S128X64]),
    (700, 2000, 896, BF16, 1, E5, [S128X64]), (1500, 2048, 2048, BF16, 128, E4, [S128]), (1500, 2048, 2048, F16, 128, E5, [S128]), (3000, 2500, 1100, F16, 128, E4, [S256]), (4096, 4096, 4096, BF16, 128, E4, [S256]),
    (3000, 4104, 3008, F16, 1, E5, [S256]), (3000, 4100, 3000, F16, 128, E4, [S256]),
    (5, 1100, 1031, F32, 128, E4, [BACK128X64, JOIN]), (65, 200, 100, F32, 1, E5, [BACK64]), (1500, 2048, 2048, F32, 128, E4, [BACK128]), (4096, 4096, 4096, F32, 128, E5, [BACK256]),
]


@pytest.mark.parametrize("rows,cols,outs,dtype,block,f8,want", BACKWARD)
def test_gradients(L, rows, cols, outs, dtype, block, f8, want):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(rows + cols + outs)
    x, w = L.quantize_f8(random(g, rows, cols, F32)), L.quantize_f8(random(g, outs, cols, F32, cols ** -0.5), block)
    dy = random(g, rows, outs, dtype, 0.01)
    print(rows, cols, outs, dtype, flush=True)
    names, got = kernels(lambda: L.linear_f8_backward(dy, x, w, f8))
    up = lambda n: -(-n // 128)  # noqa: E731
    tiles = up(rows) * (up(outs) + up(cols)) + (0 if any(DX in w for w in want) else up(outs) * up(cols))
    turns = next(n for n in names if "turn_f8_kernel" in n)
    assert turns.endswith(", 4>" if tiles <= 256 else ", 8>"), (turns, tiles)
    ran(names, ["turn_f8_kernel"] + named(want, dtype, f8))
    close(got[0], *ref.product(operand(L.quantize_f8(dy, 1, f8)), turned(L, w), dtype != F32), dtype)
    close(got[1], *ref.product(operand(L.quantize_f8(dy.t().contiguous(), 1, f8)), turned(L, x), dtype != F32), dtype)
    close(got[2], dy.double().sum(0), ref.U * (rows + 16) * dy.double().abs().sum(0), dtype)
    other = dy.flip(0).contiguous()
    for _ in range(3):
        L.linear_f8_backward(other, x, w, f8)
        assert all(torch.equal(a, b) for a, b in zip(L.linear_f8_backward(dy, x, w, f8), got))


@pytest.mark.parametrize("tensors", [1, 2, 3, 58, 59, 76, 77, 176, 177])
@pytest.mark.parametrize("bits", [8, 32])
def test_updates(L, tensors, bits):  # noqa: F811
    """Launches by the number of tensors that one describes: the norm's 176, and another for their sums from three chunks on, the step's 58 with moments in 8 bits and 76 with moments in 32; the values are those of each tensor by itself."""
    g = torch.Generator(device="cuda").manual_seed(tensors)
    d = [torch.randn(1 + 300 * i % 977, generator=g, device="cuda") for i in range(tensors)]
    p, q = ([torch.ones_like(t) for t in d] for _ in range(2))
    moments, others = L.adamw_moments(p, bits), L.adamw_moments(q, bits)
    names, norm = kernels(lambda: L.gradient_norm(d))
    most = 176
    assert sum("gradient_norm_kernel" in n for n in names) == -(-tensors // most) and sum("gradient_norm_join_kernel" in n for n in names) == (tensors > 2)
    want = math.sqrt(sum(float(t.double().square().sum()) for t in d))
    assert abs(float(norm) - want) <= 2 * ref.U * want
    names, _ = kernels(lambda: L.adamw_step(p, d, moments, 3))
    assert sum(f"adamw_kernel<{bits}>" in n for n in names) == len(names) == -(-tensors // (58 if bits == 8 else 76))
    for i, (a, b, t, m) in enumerate(zip(p, q, d, others)):
        if bits == 32 or i == 0:                            # (random bits depend on the place among the tensors)
            L.adamw_step([b], [t], [m], 3)
            assert torch.equal(a, b)
