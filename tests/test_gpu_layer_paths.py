"""Every kernel of the products with 8-bit weights, by the sizes at which it is chosen, against the definition in 64 bits.

Each case names the kernels that it stands for, and the profiler says which ones ran: a change of the estimates that choose them cannot take a kernel out
of these tests unnoticed.  Bounds are those of ``test_gpu_layers``; the definition is computed on the GPU in float64 (sums of 8-bit products are exact
there)."""

import re
import warnings

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_layers import BF16, F16, F32, LEFT, OUT, U, L, gen, values  # noqa: F401

FEW, JOIN = "linear_few_kernel", "product_join_kernel"
S64, S128X64, S128, S128DEEP, S256 = "2, 2, 4>", "4, 2, 3>", "4, 4, 2>", "4, 4, 4>", "product_kernel_256<"


def kernels(call):
    """The names of the kernels that `call` launched, and its result."""
    from torch.profiler import ProfilerActivity, profile
    torch.cuda.synchronize()
    with warnings.catch_warnings():
        warnings.simplefilter("ignore")
        with profile(activities=[ProfilerActivity.CUDA]) as p:
            out = call()
            torch.cuda.synchronize()
        names = [re.sub(r"^void |tictac::|\(.*", "", e.name) for e in p.events() if "tictac::" in e.name]
    return names, out


def ran(names, want):
    """Whether a kernel with each of the names in `want` (pieces of a name) was launched, and a join only where it is among them."""
    assert all(any(w in n for n in names) for w in want), names
    assert any(JOIN in n for n in names) == (JOIN in want), names


def near(got, want, bound, dtype):
    rel, least = OUT[dtype]
    assert got.shape == want.shape and bool(torch.isfinite(got).all())
    off = (got.double() - want).abs() - (bound + rel * (want.abs() + bound) + least)
    assert float(off.max()) <= 0, float(off.max())


def normal8(L, g, rows, cols, scale=1.0):
    """8-bit rows of normal values, made on the GPU (rows of different sizes), and what they stand for in float64."""
    x = torch.randn(rows, cols, generator=g, device="cuda") * torch.exp(0.5 * torch.randn(rows, 1, generator=g, device="cuda")) * scale
    r = L.quantize_rows(x)
    return r, r.q[:, :cols].double(), r.scale.double()


# rows, columns, outputs, type of the output, kernels
FORWARD = [
    (5, 2050, 2100, F32, ["linear_few_kernel<1, 1>"]), (3, 20000, 9000, BF16, ["linear_few_kernel<1, 1>", JOIN]),
    (12, 2050, 2100, F16, ["linear_few_kernel<1, 2>", JOIN]), (16, 20000, 4096, BF16, ["linear_few_kernel<1, 2>", JOIN]),
    (20, 20000, 1030, F16, ["linear_few_kernel<2, 1>", JOIN]), (32, 2048, 4096, F32, ["linear_few_kernel<2, 4>", JOIN]),
    (27, 20000, 2101, BF16, ["linear_few_kernel<2, 4>", JOIN]), (32, 2048, 9000, F16, ["linear_few_kernel<2, 4>"]),
    (50, 3000, 1999, BF16, ["linear_few_kernel<4, 1>", JOIN]), (64, 20000, 4096, F16, ["linear_few_kernel<4, 4>", JOIN]),
    (61, 2050, 2101, F32, ["linear_few_kernel<4, 4>", JOIN]), (64, 2048, 9001, BF16, ["linear_few_kernel<4, 4>"]),
    (100, 777, 1001, F32, [S64]), (130, 4096, 2000, BF16, [S64, JOIN]), (130, 4100, 2001, F16, [S64, JOIN]), (900, 8192, 900, F16, [S64]),
    (1000, 520, 2000, BF16, [S128X64]), (1500, 300, 1501, F32, [S128X64]), (1024, 8192, 2048, F16, [S128X64]),
    (2048, 4096, 2048, F16, [S128DEEP]), (2040, 4100, 2043, F32, [S128DEEP]),
    (1000, 2000, 5000, F32, [S128]), (1800, 600, 2301, BF16, [S128]), (2100, 100, 2060, F16, [S128]),
    # more tiles than compute units, of which the last ones are not whole; few steps, an odd number of them too
    (8192, 512, 16384, F16, [S256]), (8192, 512, 16384, F32, [S256]), (16000, 300, 16104, BF16, [S256]), (16000, 300, 16104, F32, [S256]), (16000, 300, 16101, BF16, [S256]),
]


@pytest.mark.parametrize("rows,cols,outs,dtype,want", FORWARD)
def test_products(L, rows, cols, outs, dtype, want):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(rows + cols + outs)
    (x8, q, s), (w8, qw, sw) = normal8(L, g, rows, cols), normal8(L, g, outs, cols, cols ** -0.5)
    bias = torch.randn(outs, generator=g, device="cuda")
    print(rows, cols, outs, dtype, flush=True)
    names, got = kernels(lambda: L.linear_q8(x8, w8, bias, dtype))
    ran(names, want)
    part = (q @ qw.t()) * s * sw.t()
    near(got, part + bias.double(), 5 * U * (part.abs() + bias.double().abs()), dtype)
    del part
    other = normal8(L, g, rows, cols)[0]
    for _ in range(4):                                      # (nothing waits between them)
        L.linear_q8(other, w8, bias, dtype)
        assert torch.equal(L.linear_q8(x8, w8, bias, dtype), got)


# rows, columns, outputs, kernels; by the number of bf16 pieces that a type is cut into
FEW_BACK = ["linear_dx_few_kernel", "linear_dw_few_kernel"]
BACKWARD = [
    # (16 cuts of the 282 blocks of k at most: more than one for each of the eight waves)
    (5, 4096, 9000, F16, FEW_BACK + [JOIN]), (5, 1100, 1031, F32, FEW_BACK + [JOIN]), (32, 8000, 9001, BF16, FEW_BACK + [JOIN]), (27, 4096, 9024, F32, FEW_BACK + [JOIN]),
    (64, 2104, 9000, F16, FEW_BACK + [JOIN]), (50, 4096, 9001, F32, FEW_BACK + [JOIN]), (64, 200, 1030, BF16, FEW_BACK + [JOIN]), (64, 4096, 4096, F32, FEW_BACK + [JOIN]),
    (65, 200, 100, F32, [S64]), (96, 520, 256, BF16, [S64]), (130, 264, 640, F16, [S64, JOIN]), (1030, 190, 2070, F32, [S64, JOIN]), (1030, 190, 2070, BF16, [S64, JOIN]),
    (300, 1000, 1024, BF16, [S128X64]), (300, 1000, 1024, F32, [S128X64, JOIN]), (500, 1000, 1000, F16, [S128X64, JOIN]), (1500, 1100, 2051, F16, [S128X64]),
    (700, 2000, 900, F32, [S128DEEP]), (700, 2000, 900, F16, [S128DEEP]), (700, 2000, 896, BF16, [S128DEEP]),
    (1500, 2048, 2048, F32, [S128]), (1500, 2048, 2048, BF16, [S128]), (3000, 2500, 1100, F16, [S128, JOIN]), (2048, 2048, 1024, BF16, [S128, JOIN]),
    (4096, 4096, 4096, BF16, [S256]), (4096, 4096, 4096, F16, [S256]), (4096, 4096, 4096, F32, [S256]), (3000, 4104, 3000, F32, [S256]), (3000, 4104, 3008, BF16, [S256]),
    (3000, 4100, 3000, F16, [S256]),
]


@pytest.mark.parametrize("rows,cols,outs,dtype,want", BACKWARD)
def test_gradients(L, rows, cols, outs, dtype, want):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(rows + cols + outs)
    (x8, q, s), (w8, qw, sw) = normal8(L, g, rows, cols), normal8(L, g, outs, cols, cols ** -0.5)
    dy = (0.01 * torch.randn(rows, outs, generator=g, device="cuda") * torch.exp(0.5 * torch.randn(rows, 1, generator=g, device="cuda"))).to(dtype)
    print(rows, cols, outs, dtype, flush=True)
    names, got = kernels(lambda: L.linear_q8_backward(dy, x8, w8))
    ran(names, want)
    x, w, d = q * s, qw * sw, dy.double()

    def bound(k, size):
        return (LEFT[dtype] + 2 * U + 6 * U * k) * size

    near(got[0], d @ w, bound(outs, d.abs() @ w.abs()), dtype)
    near(got[1], d.t() @ x, bound(rows, d.abs().t() @ x.abs()), dtype)
    near(got[2], d.sum(0), (rows + 2) * U * d.abs().sum(0), dtype)
    del x, w, d
    room = torch.full((rows, outs + 64), 3.0, dtype=dtype, device="cuda")           # (rows at another stride, on 16-byte boundaries where they were)
    room[:, 8:8 + outs] = dy
    other = dy.flip(0).contiguous()
    for again in (dy, room[:, 8:8 + outs], dy):
        L.linear_q8_backward(other, x8, w8)
        assert all(torch.equal(a, b) for a, b in zip(L.linear_q8_backward(again, x8, w8), got))
