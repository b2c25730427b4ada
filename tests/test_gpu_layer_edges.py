"""The layers' operators where they can go wrong: gradients asked for one at a time, the largest sums, infinities and NaN.  Helpers and bounds are those of
``test_gpu_layers``."""

import ctypes

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from layer_calls import call
from test_gpu_layers import (ADDS, BF16, F16, F32, LEFT, OUT, TYPES, U, L, check_norm_grads, close, gen, norm64, norm_tolerance,  # noqa: F401
                             rows8_values, values, weights)

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
@pytest.mark.parametrize("rows,outs", [(1, 16), (20, 200), (40, 5000), (70, 60), (300, 2100), (600, 6000), (1024, 16384)])
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


def check_with_infinities(got, want, bound):
    """`got` where the definition in 64 bits is finite, its infinities with their signs, its NaN."""
    got = got.cpu().double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(got.isposinf(), want.isposinf()) and torch.equal(got.isneginf(), want.isneginf())
    fine = torch.isfinite(want)
    assert float(((got - want).abs() - bound)[fine].max()) <= 0


@pytest.mark.parametrize("rows,cols,outs", [(5, 100, 61), (40, 264, 136), (64, 130, 48), (90, 200, 77), (300, 264, 640), (2100, 2100, 2060)])
@pytest.mark.parametrize("dtype", TYPES)
def test_linear_gradients_of_infinities(L, rows, cols, outs, dtype):  # noqa: F811
    """One infinity, one minus infinity and one NaN in dy: dx has them in their rows, dw in theirs, with the signs of the 8-bit values; a zero gives NaN."""
    g = gen(rows)
    x8, w8 = L.quantize_rows(values(g, rows, cols, F32).cuda()), weights(L, g, outs, cols)
    dy = values(g, rows, outs, dtype, size=0.01)
    dy[1, 2], dy[3, 30], dy[rows - 1, outs - 1] = float("inf"), -float("inf"), float("nan")
    dx, dw, db = L.linear_q8_backward(dy.cuda(), x8, w8)
    x, w, d = rows8_values(x8), rows8_values(w8), dy.double()
    small = torch.nan_to_num(d, nan=0.0, posinf=0.0, neginf=0.0).abs()

    def tol(k, size):                       # (that of test_linear_backward, and the rounding of the output)
        return (LEFT[dtype] + 2 * U + 6 * U * k + OUT[dtype][0]) * 1.01 * size + OUT[dtype][1]

    def product(a, b):                      # (an infinity times zero is NaN, whatever the library's product does with zeros)
        odd = ~torch.isfinite(a)
        y = torch.where(odd, 0.0, a) @ b
        for i, k in odd.nonzero().tolist():
            y[i] = y[i] + a[i, k] * b[k]
        return y

    check_with_infinities(dx, product(d, w), tol(outs, small @ w.abs()))
    check_with_infinities(dw, product(d.t(), x), tol(rows, small.t() @ x.abs()))
    check_with_infinities(db, d.sum(0), tol(rows, small.sum(0)))


@pytest.mark.parametrize("rows,cols", [(6, 100), (30, 1400), (5, 20000), (1500, 130), (600, 9000)])
@pytest.mark.parametrize("kept", [False, True])
def test_layer_norm_gradients_of_spoilt_rows(L, rows, cols, kept):  # noqa: F811
    """A NaN in x, one in dy, an infinity in each: dx is NaN in those rows alone, dw in all columns of a spoilt x, db in those of a spoilt dy."""
    g = gen(cols)
    x, dy = values(g, rows, cols, F32), values(g, rows, cols, F32)
    gamma = (1 + 0.3 * torch.randn(cols, generator=g)).cuda()
    _, mean, rstd, x8 = L.layer_norm(x.cuda(), gamma, save=True)
    clean = L.layer_norm_backward(dy.cuda(), x8 if kept else x.cuda(), gamma, mean, rstd)
    bad = dy.clone()
    bad[1, 5], bad[2, 7] = float("nan"), float("inf")
    dx, dw, db = L.layer_norm_backward(bad.cuda(), x8 if kept else x.cuda(), gamma, mean, rstd)
    others = [i for i in range(rows) if i not in (1, 2)]
    assert torch.equal(dx[others], clean[0][others]) and bool(torch.isnan(dx[1]).all()) and not bool(torch.isfinite(dx[2]).any())
    columns = torch.ones(cols, dtype=torch.bool)
    columns[[5, 7]] = False
    assert torch.isnan(dw[5]) and not torch.isfinite(dw[7]) and torch.equal(dw[columns], clean[1][columns])
    assert torch.isnan(db[5]) and db[7] == float("inf") and torch.equal(db[columns], clean[2][columns])
    x[3, 9], x[4, 0] = float("nan"), -float("inf")
    _, mean, rstd, x8 = L.layer_norm(x.cuda(), gamma, save=True)
    dx, dw, db = L.layer_norm_backward(dy.cuda(), x8 if kept else x.cuda(), gamma, mean, rstd)
    others = [i for i in range(rows) if i not in (3, 4)]
    assert torch.equal(dx[others], clean[0][others]) and bool(torch.isnan(dx[[3, 4]]).all()) and bool(torch.isnan(dw).all()) and torch.equal(db, clean[2])


def test_gradients_of_a_row_of_many_columns(L):  # noqa: F811
    """2^27 columns and five: more workgroups for dweight and dbias than a grid holds threads of.  One row: the sums are its own values."""
    cols = (1 << 27) + 5
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dy = (torch.randn(1, cols, generator=g, device="cuda") for _ in range(2))
    mean, rstd = torch.tensor([0.25], device="cuda"), torch.tensor([2.0], device="cuda")
    _, dw, db = L.layer_norm_backward(dy, x, None, mean, rstd)
    assert torch.equal(db, dy[0])
    assert torch.equal(dw, dy[0] * ((x[0] - 0.25) * 2.0))


@pytest.mark.parametrize("cols", [16391, 1 << 20, (1 << 22) + 5])
@pytest.mark.parametrize("dtype", TYPES)
def test_long_rows_to_the_bound_of_short_ones(L, cols, dtype):  # noqa: F811
    """A constant row, whose sums round the same way every time, one on an offset and one around zero: mean, rstd, y and dx to the bounds of any length."""
    g = gen(cols)
    x, dy = torch.randn(3, cols, generator=g), 0.1 + 0.01 * torch.randn(3, cols, generator=g)
    x[0], dy[0] = 0.1, 0.1
    x[1] += 3.0
    x, dy = x.to(dtype), dy.to(dtype)
    gamma = 1 + 0.3 * torch.randn(cols, generator=g)
    y, mean, rstd = L.layer_norm(x.cuda(), gamma.cuda(), None)
    wy, wm, wr, xh = norm64(x, gamma, None, 1e-5)
    close(mean, wm, ADDS * U * x.double().abs().mean(1), F32)
    close(rstd, wr, ADDS * U * wr * (1 + x.double().abs().mean(1) * wr), F32)
    close(y, wy, norm_tolerance(x, wm, wr, xh, gamma, None), dtype)
    dx, dw, db = L.layer_norm_backward(dy.cuda(), x.cuda(), gamma.cuda(), mean, rstd)
    check_norm_grads(dx, dw, db, dy, x.double(), gamma, mean.cpu().double(), rstd.cpu().double(), dtype, F32)
    spoilt = x.clone()
    spoilt[1, 7], spoilt[2, 9] = float("inf"), -float("inf")
    mean = L.layer_norm(spoilt.cuda())[1].tolist()
    assert mean[1:] == [float("inf"), -float("inf")]


def test_views_with_turned_signs(L):  # noqa: F811
    """Tensors whose memory holds the negatives of their values (torch's lazy negation) count as their values."""
    g = gen(12)
    neg = torch._neg_view
    x, dy, gamma, beta = (torch.randn(*s, generator=g).cuda() for s in ((6, 200), (6, 200), (200,), (200,)))
    w, bias = weights(L, g, 200, 200), torch.randn(200, generator=g).cuda()
    z = torch.view_as_complex(torch.randn(5, 2, generator=g).cuda()).conj().imag[:, None]
    assert z.is_neg() and torch.equal(L.layer_norm(z, eps=1.0)[1], z[:, 0].clone())
    n = L.layer_norm(-x, -gamma, -beta, save=True)
    x8, back = n[3], L.layer_norm_backward(-dy, -x, -gamma, -n[1], -n[2])
    turned = L.Rows8(w.q, -w.scale, 200)

    def same(a, b):
        assert all(torch.equal(s, t) for s, t in zip(a, b) if isinstance(s, torch.Tensor))

    same(L.quantize_rows(neg(x)), L.quantize_rows(-x))
    same(L.layer_norm(neg(x), neg(gamma), neg(beta), save=True)[:3], n[:3])
    same(L.layer_norm_backward(neg(dy), neg(x), neg(gamma), neg(n[1]), neg(n[2])), back)
    same([L.linear_q8(neg(x), L.Rows8(w.q, neg(w.scale), 200), neg(bias))], [L.linear_q8(-x, turned, -bias)])
    same(L.linear_q8_backward(neg(dy), L.quantize_rows(x), w), L.linear_q8_backward(-dy, L.quantize_rows(x), w))
    same([L.dequantize_rows(L.Rows8(x8.q, neg(x8.scale), 200, 128))], [-L.dequantize_rows(x8)])


def test_outputs_carry_no_graph(L):  # noqa: F811
    """As the module says: no output requires a gradient, whatever the inputs do."""
    x, gamma, dy = (torch.randn(*s, device="cuda", requires_grad=True) for s in ((4, 200), (200,), (4, 200)))
    w = weights(L, gen(1), 200, 200)
    y, mean, rstd, x8 = L.layer_norm(x, gamma, save=True)
    out = [y, mean, rstd, x8.q, x8.scale, L.linear_q8(x, w, gamma), L.dequantize_rows(x8)]
    out += L.layer_norm_backward(dy, x, gamma, mean, rstd) + L.linear_q8_backward(dy, L.quantize_rows(x), w)
    assert not any(t.requires_grad or t.grad_fn for t in out) and "no autograd" in L.__doc__
