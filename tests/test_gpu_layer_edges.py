"""The layers' operators where they can go wrong: gradients asked for one at a time, and others below.  Helpers and bounds are those of
``test_gpu_layers``."""

import ctypes

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from layer_calls import call
from test_gpu_layers import BF16, F16, F32, L, TYPES, gen, values, weights  # noqa: F401

CODE = {F32: 0, F16: 1, BF16: 2}


def linear_backward_of(dy, x8, w8, which):
    """The C call with the outputs in `which` alone, and only the inputs that they take: {name: tensor}."""
    from paper_1803_03288_amd import binding
    (rows, outs), cols, code = dy.shape, x8.cols, CODE[dy.dtype]
    out = {n: torch.full(shape, 7.0, dtype=dy.dtype, device="cuda") for n, shape in (("dx", (rows, cols)), ("dw", (outs, cols)), ("db", (outs,))) if n in which}
    at = lambda n: out[n].data_ptr() if n in out else None  # noqa: E731
    size = ctypes.c_size_t()
    call("tictac_linear_q8_backward_workspace", code, rows, cols, outs, ctypes.addressof(size))
    room = torch.empty(max(size.value, 256), dtype=torch.uint8, device="cuda")
    x = (x8.q.data_ptr(), x8.q.stride(0), x8.scale.data_ptr()) if "dw" in which else (None, 0, None)
    w = (w8.q.data_ptr(), w8.q.stride(0), w8.scale.data_ptr()) if "dx" in which else (None, 0, None)
    call("tictac_linear_q8_backward", code, rows, cols, outs, dy.data_ptr(), outs, *x, *w, at("dx"), cols, at("dw"), cols, at("db"), room.data_ptr(), room.numel(), binding._stream())
    return out


# (both sides of 64 rows, where other kernels take over; rows on and off 16-byte boundaries; sums cut along k; the largest tiles)
@pytest.mark.parametrize("rows,cols,outs", [(1, 64, 48), (20, 200, 61), (64, 128, 1100), (65, 200, 61), (130, 264, 640), (300, 153, 587), (2100, 2100, 2060)])
@pytest.mark.parametrize("dtype", TYPES)
def test_linear_gradients_one_at_a_time(L, rows, cols, outs, dtype):  # noqa: F811
    """The same bits whichever of them are asked for, without the inputs that they do not take."""
    g = gen(rows + cols)
    x8, w8, dy = L.quantize_rows(values(g, rows, cols, F32).cuda()), weights(L, g, outs, cols), values(g, rows, outs, dtype, size=0.01).cuda()
    want = dict(zip(("dx", "dw", "db"), L.linear_q8_backward(dy, x8, w8)))
    for which in (("db",), ("dx",), ("dw",), ("dx", "db"), ("dw", "db"), ("dx", "dw")):
        print(rows, cols, outs, dtype, which, flush=True)
        for name, got in linear_backward_of(dy, x8, w8, which).items():
            assert torch.equal(got, want[name]), (which, name)


# (by few rows with and without cuts along k, and by tiles with and without)
@pytest.mark.parametrize("rows,outs", [(1, 16), (20, 200), (40, 5000), (70, 60), (300, 2100), (600, 6000)])
def test_the_largest_sum(L, rows, outs):  # noqa: F811
    """131 072 products of -128 and -128 are 2^31, and of -128 and 127 the least there is."""
    cols = 131072
    q = torch.full((rows, cols), -128, dtype=torch.int8, device="cuda")
    p = torch.full((outs, cols), -128, dtype=torch.int8, device="cuda")
    q[::2], p[1::3], p[2::3, -1] = 127, 127, -127
    one = torch.ones(max(rows, outs), 1, device="cuda")
    got = L.linear_q8(L.Rows8(q, one[:rows], cols), L.Rows8(p, one[:outs], cols))
    ends = torch.full((rows, 1), -128.0, dtype=torch.float64), torch.full((outs, 1), -128.0, dtype=torch.float64)
    ends[0][::2], ends[1][1::3] = 127, 127
    want = cols * ends[0] * ends[1].t()
    want[:, 2::3] = ((cols - 1) * -128.0 - 127) * ends[0]
    assert rows == 1 or float(want.max()) == 2.0 ** 31
    assert torch.equal(got.cpu(), want.float())
