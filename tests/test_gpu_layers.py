"""The layers' operators (``paper_1803_03288_amd.layers``) against their definitions in 64 bits.

Tolerances follow from the arithmetic, before any run: ``u = 2**-24`` for each float32 operation or addition on the way of a value, the rounding
of the output's type (8 bits of bfloat16, 11 of float16), and for the gradients of products the part of ``dy * scale`` that the bf16 pieces
leave out.  8-bit rows and exact sums are compared bit by bit."""

import ctypes
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from layer_calls import call

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
TYPES = [F32, F16, BF16]
U = 2.0 ** -24
OUT = {F32: (U, 2.0 ** -149), F16: (2.0 ** -11, 2.0 ** -25), BF16: (2.0 ** -8, 2.0 ** -134)}
ADDS = 64           # float32 operations on the way of a row's sum: up to 32 per thread, the tree, what follows


@pytest.fixture(scope="module")
def L():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1803_03288_amd import layers
    return layers


def gen(seed):
    return torch.Generator().manual_seed(seed)


def values(g, rows, cols, dtype, size=1.0, offset=0.0):
    return ((torch.randn(rows, cols, generator=g) * torch.exp(0.5 * torch.randn(rows, 1, generator=g)) + offset) * size).to(dtype)


def close(got, want, tol, dtype):
    """|got - want| within `tol` and the rounding to `dtype`."""
    got = got.cpu().double()
    rel, least = OUT[dtype]
    off = (got - want).abs() - (tol + rel * (want.abs() + tol) + least)
    assert got.shape == want.shape and torch.isfinite(got).all()
    assert float(off.max()) <= 0, float(off.max())


def rows8(x, group):
    """The definition in float32, on the CPU: (q [rows][cols] int8, scale)."""
    x = x.float()
    rows, cols = x.shape
    n = group or cols
    q, s = torch.zeros(rows, cols, dtype=torch.int8), []
    for lo in range(0, cols, n):
        part = x[:, lo:lo + n]
        amax = part.abs().max(1, keepdim=True).values                  # (torch's maximum keeps NaN)
        bad, small = ~torch.isfinite(amax), amax < 2.0 ** -116
        most = torch.full_like(amax, 127.0)         # (a quotient of tensors is one division; with a number it is a reciprocal and a product)
        inv = torch.where(bad | small, torch.zeros_like(amax), most / amax)
        k = torch.where(bad | small, torch.zeros_like(part), torch.round(part * inv))
        q[:, lo:lo + n] = torch.nan_to_num(k).to(torch.int8)
        s.append(torch.where(bad, torch.full_like(amax, math.nan), torch.where(small, torch.zeros_like(amax), (amax / most).clamp(max=float.fromhex("0x1.020406p121")))))
    return q, torch.cat(s, 1)


def check_rows8(r, x, group):
    q, s = rows8(x, group)
    cols = x.shape[1]
    got_q, got_s = r.q.cpu(), r.scale.cpu()
    assert r.cols == cols and r.group == group and got_q.shape[1] == -(-cols // 128) * 128
    assert torch.equal(got_q[:, :cols], q)
    assert int(got_q[:, cols:].abs().sum()) == 0                      # zeros up to the stride
    assert np.array_equal(got_s.numpy(), s.numpy(), equal_nan=True)
    return q, s


def rows8_values(r):
    q, s = r.q.cpu()[:, :r.cols].double(), r.scale.cpu().double()
    return q * (s if r.group == 0 else torch.repeat_interleave(s, 128, 1)[:, :r.cols])


# ---- 8-bit rows ---------------------------------------------------------------------------------------------

@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (5, 127), (2, 128), (33, 129), (17, 1000), (4, 2049), (300, 256), (3, 20000), (2, 40000)])
def test_rows_in_8_bits(L, rows, cols, dtype, group):
    g = gen(rows * 1000 + cols)
    x = values(g, rows, cols, dtype)
    x[0, 0] = 0.0
    r = L.quantize_rows(x.cuda(), group)
    check_rows8(r, x, group)
    back = L.dequantize_rows(r, dtype)
    want = (r.q.cpu()[:, :cols].float() * (r.scale.cpu() if group == 0 else torch.repeat_interleave(r.scale.cpu(), 128, 1)[:, :cols])).to(dtype)
    assert torch.equal(back.cpu(), want)


@pytest.mark.parametrize("group", [0, 128])
def test_rows_in_8_bits_at_the_ends_of_the_range(L, group):
    x = torch.zeros(9, 300)
    x[1] = 2.0 ** -116                                   # the smallest that is kept
    x[2] = 2.0 ** -116 * (1 - 2.0 ** -24)                # below
    x[3, 5], x[3, 200] = 3.4028234663852886e38, -3.0e38  # the largest
    x[4, 299] = math.inf
    x[5, 0] = math.nan
    x[6] = torch.linspace(-1, 1, 300)
    x[7] = 2.0 ** -149                                   # the smallest there is
    x[8, :] = torch.arange(300) - 150.5                  # halves: ties go to even
    r = L.quantize_rows(x.cuda(), group)
    check_rows8(r, x, group)
    back = L.dequantize_rows(r).cpu()
    assert torch.isnan(back[4, 256:]).all() and torch.isnan(back[5, :128]).all()
    if group == 0:
        assert torch.isnan(back[4]).all() and torch.isnan(back[5]).all()
    assert torch.isfinite(back[[0, 1, 2, 3, 6, 7, 8]]).all() and not back[[0, 2, 7]].any()


def strided(x, kind):
    """`x` on the GPU with rows at another stride, off 16-byte boundaries, transposed, or one row for all."""
    rows, cols = x.shape
    if kind == "wide":
        room = torch.full((rows, cols + 24), 7.0, dtype=x.dtype, device="cuda")
        room[:, 8:8 + cols] = x.cuda()
        return room[:, 8:8 + cols]
    if kind == "odd":
        room = torch.full((rows, cols + 5), 7.0, dtype=x.dtype, device="cuda")
        room[:, 3:3 + cols] = x.cuda()
        return room[:, 3:3 + cols]
    if kind == "transposed":
        return x.cuda().t().contiguous().t()
    assert kind == "repeated"
    return x[:1].cuda().expand(rows, cols)


STRIDES = ["wide", "odd", "transposed", "repeated"]


@pytest.mark.parametrize("kind", STRIDES)
@pytest.mark.parametrize("dtype", TYPES)
def test_strides(L, kind, dtype):
    g = gen(5)
    rows, cols, outs = 70, 264, 136
    x = values(g, rows, cols, dtype)
    dy = values(g, rows, outs, dtype)
    sx, sdy = strided(x, kind), strided(dy, kind)
    x, dy = sx.contiguous(), sdy.contiguous()
    w = L.quantize_rows(torch.randn(outs, cols, generator=g).cuda())
    gamma, beta = torch.randn(cols, generator=g).cuda(), torch.randn(cols, generator=g).cuda()

    def same(a, b):
        a, b = (t if isinstance(t, tuple) else (t,) for t in (a, b))
        for s, t in zip(a, b):
            if isinstance(s, torch.Tensor):
                assert torch.equal(s, t)

    for group in (0, 128):
        same(L.quantize_rows(sx, group), L.quantize_rows(x, group))
    n = L.layer_norm(x, gamma, beta, save=True)
    same(L.layer_norm(sx, gamma, beta, save=True)[:3], n[:3])
    same(tuple(L.layer_norm(sx, gamma, beta, save=True)[3]), tuple(n[3]))
    same(tuple(L.layer_norm_q8(sx, gamma, beta)[0]), tuple(L.layer_norm_q8(x, gamma, beta)[0]))
    dn, sdn = values(g, rows, cols, dtype).cuda(), None
    sdn = strided(dn.cpu(), kind)
    dn = sdn.contiguous()
    for src, ssrc in ((x, sx), (n[3], n[3])):
        same(L.layer_norm_backward(sdn, ssrc, gamma, n[1], n[2]), L.layer_norm_backward(dn, src, gamma, n[1], n[2]))
    same(L.linear_q8(sx, w), L.linear_q8(x, w))
    x8 = L.quantize_rows(x)
    same(L.linear_q8_backward(sdy, x8, w), L.linear_q8_backward(dy, x8, w))
    # 8-bit rows at a larger stride
    room = torch.full((rows, x8.q.shape[1] + 128), 99, dtype=torch.int8, device="cuda")
    room[:, :x8.q.shape[1]] = x8.q
    far = L.Rows8(room[:, :x8.q.shape[1]], x8.scale, cols)
    same(L.linear_q8(far, w, dtype=dtype), L.linear_q8(x8, w, dtype=dtype))
    same(L.linear_q8_backward(dy, far, w), L.linear_q8_backward(dy, x8, w))
    same(L.dequantize_rows(far), L.dequantize_rows(x8))


# ---- layer norm ---------------------------------------------------------------------------------------------

def norm64(x, gamma, beta, eps):
    x = x.double()
    mean = x.mean(1)
    d = x - mean[:, None]
    rstd = 1 / torch.sqrt(d.square().mean(1) + eps)
    xh = d * rstd[:, None]
    y = xh * (1 if gamma is None else gamma.double()) + (0 if beta is None else beta.double())
    return y, mean, rstd, xh


def norm_tolerance(x, mean, rstd, xh, gamma, beta):
    """Of y before it is rounded: the mean's error carried through, that of the variance, and the operations on each element."""
    w = 1.0 if gamma is None else gamma.double().abs()
    size = x.double().abs().mean(1, keepdim=True) * rstd[:, None]
    b = 0.0 if beta is None else beta.double().abs()
    return ADDS * U * (w * (size + xh.abs()) + b)


NORM_SIZES = [(1, 1), (1, 5), (7, 64), (5, 511), (9, 512), (6, 513), (130, 777), (4, 1024), (3, 1025), (2, 2048), (33, 3000), (2, 4096),
              (3, 4099), (2, 8192), (3, 9000), (2, 16384), (2, 16391)]


@pytest.mark.parametrize("rows,cols", NORM_SIZES)
@pytest.mark.parametrize("dtype", TYPES)
def test_layer_norm(L, rows, cols, dtype):
    g = gen(cols)
    x = values(g, rows, cols, dtype, offset=0.5)
    gamma, beta = 1 + 0.3 * torch.randn(cols, generator=g), torch.randn(cols, generator=g)
    eps = 1e-5
    y, mean, rstd, x8 = L.layer_norm(x.cuda(), gamma.cuda(), beta.cuda(), eps, save=True)
    wy, wm, wr, xh = norm64(x, gamma, beta, eps)
    tol = norm_tolerance(x, wm, wr, xh, gamma, beta)
    close(y, wy, tol, dtype)
    close(mean, wm, ADDS * U * x.double().abs().mean(1), F32)
    close(rstd, wr, ADDS * U * wr * (1 + x.double().abs().mean(1) * wr), F32)
    check_rows8(x8, x, 128)
    y8, mean2, rstd2 = L.layer_norm_q8(x.cuda(), gamma.cuda(), beta.cuda(), eps)
    assert torch.equal(mean2, mean) and torch.equal(rstd2, rstd)
    amax = wy.abs().max(1, keepdim=True).values
    s = y8.scale.cpu().double()
    assert float(((s * 127 - amax).abs() - (tol.max(1, keepdim=True).values + 2 * U * amax)).max()) <= 0
    # half a step, and what y itself may be off
    off = (rows8_values(y8) - wy).abs() - (0.5 * s * (1 + 2.0 ** -15) + tol)
    assert float(off.max()) <= 0
    assert int(y8.q.cpu()[:, cols:].abs().sum()) == 0


@pytest.mark.parametrize("of", ["type", "float32", "none"])
def test_layer_norm_parameters(L, of):
    g = gen(3)
    for dtype in TYPES:
        for cols in (96, 101, 5000):
            x = values(g, 5, cols, dtype)
            as_type = dtype if of == "type" else F32
            gamma, beta = (None, None) if of == "none" else (torch.randn(cols, generator=g).to(as_type), torch.randn(cols, generator=g).to(as_type))
            put = lambda t: None if t is None else t.cuda()  # noqa: E731
            y, mean, rstd = L.layer_norm(x.cuda(), put(gamma), put(beta), 1e-3)
            wy, wm, wr, xh = norm64(x, gamma, beta, 1e-3)
            close(y, wy, norm_tolerance(x, wm, wr, xh, gamma, beta), dtype)
            dy = values(g, 5, cols, dtype)
            dx, dw, db = L.layer_norm_backward(dy.cuda(), x.cuda(), put(gamma), mean, rstd)
            assert dw.dtype == db.dtype == as_type
            check_norm_grads(dx, dw, db, dy, x.double(), gamma, mean.cpu().double(), rstd.cpu().double(), dtype, as_type)


def check_norm_grads(dx, dw, db, dy, x, gamma, mean, rstd, dtype, of):
    dy = dy.double()
    m, r = mean[:, None], rstd[:, None]
    d = x - m
    xh = d * r
    g = dy * (1 if gamma is None else gamma.double())
    a, b = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
    # (x and the mean are floats: their difference is off by an operation, relative to itself)
    tol = ADDS * U * r * (g.abs() + g.abs().mean(1, keepdim=True) + xh.abs() * (g * xh).abs().mean(1, keepdim=True))
    close(dx, r * (g - a - xh * b), tol, dtype)
    rows = dy.shape[0]
    adds = (-(-rows // 512) + 64) * U
    close(dw, (dy * xh).sum(0), adds * (dy * xh).abs().sum(0), of)
    close(db, dy.sum(0), adds * dy.abs().sum(0), of)


@pytest.mark.parametrize("rows,cols", NORM_SIZES + [(1500, 130), (700, 1400), (5, 20000)])
@pytest.mark.parametrize("dtype", TYPES)
def test_layer_norm_backward(L, rows, cols, dtype):
    g = gen(cols + 1)
    x, dy = values(g, rows, cols, dtype, offset=0.5), values(g, rows, cols, dtype, size=0.01)
    gamma = 1 + 0.3 * torch.randn(cols, generator=g)
    _, mean, rstd, x8 = L.layer_norm(x.cuda(), gamma.cuda(), None, save=True)
    for src, as64 in ((x.cuda(), x.double()), (x8, rows8_values(x8))):
        dx, dw, db = L.layer_norm_backward(dy.cuda(), src, gamma.cuda(), mean, rstd)
        check_norm_grads(dx, dw, db, dy, as64, gamma, mean.cpu().double(), rstd.cpu().double(), dtype, F32)
        again = L.layer_norm_backward(dy.cuda(), src, gamma.cuda(), mean, rstd)
        assert torch.equal(again[0], dx) and torch.equal(again[1], dw) and torch.equal(again[2], db)


def test_layer_norm_gradient_against_differences(L):
    g = gen(8)
    rows, cols, h = 4, 40, 1e-6
    x, dy = torch.randn(rows, cols, generator=g), torch.randn(rows, cols, generator=g)
    gamma, beta = 1 + 0.3 * torch.randn(cols, generator=g), torch.randn(cols, generator=g)
    _, mean, rstd = L.layer_norm(x.cuda(), gamma.cuda(), beta.cuda())
    dx, dw, db = (t.cpu().double() for t in L.layer_norm_backward(dy.cuda(), x.cuda(), gamma.cuda(), mean, rstd))

    def loss(x, gamma, beta):
        return float((norm64(x, gamma, beta, 1e-5)[0] * dy.double()).sum())

    at = [x.double(), gamma.double(), beta.double()]
    for k, grad in enumerate((dx, dw, db)):
        v = torch.randn(at[k].shape, generator=g).double()
        up, down = (loss(*(t + s * h * v if i == k else t for i, t in enumerate(at))) for s in (1, -1))
        # differences: cancellation 2^-52 |loss| / h, and h^2; the kernels: float32
        assert abs((up - down) / (2 * h) - float((grad * v).sum())) <= 1e-4 * float((grad * v).abs().sum()) + 1e-7


def test_layer_norm_on_a_row_that_spoils_itself_only(L):
    g = gen(4)
    x = values(g, 6, 700, F32)
    x[1, 3], x[2, 4], x[4] = math.inf, math.nan, 0.0
    y, mean, rstd, x8 = L.layer_norm(x.cuda(), None, None, save=True)
    y8 = L.layer_norm_q8(x.cuda())[0]
    for t in (y, L.dequantize_rows(y8)):
        bad = torch.isnan(t.cpu()).all(1)
        assert bad.tolist() == [False, True, True, False, False, False]
        assert torch.isfinite(t.cpu()[[0, 3, 4, 5]]).all()
    assert not y[4].any() and float(mean[4]) == 0
    check_rows8(x8, x, 128)


# ---- products -----------------------------------------------------------------------------------------------

LINEAR_SIZES = [(1, 1, 1), (1, 100, 17), (3, 128, 16), (16, 1000, 33), (17, 129, 64), (32, 4096, 31), (33, 640, 40), (64, 2304, 130), (65, 200, 100),
                (100, 777, 1001), (257, 1100, 300), (513, 64, 515), (2100, 300, 2060), (4096, 256, 4000)]


def weights(L, g, outs, cols):
    return L.quantize_rows((torch.randn(outs, cols, generator=g) / math.sqrt(cols)).cuda())


@pytest.mark.parametrize("rows,cols,outs", LINEAR_SIZES)
def test_linear(L, rows, cols, outs):
    g = gen(rows + cols)
    w = weights(L, g, outs, cols)
    bias = torch.randn(outs, generator=g)
    qw, sw = w.q.cpu()[:, :cols].double(), w.scale.cpu().double()
    for dtype in TYPES:
        x = values(g, rows, cols, dtype)
        x8 = L.quantize_rows(x.cuda())
        q, s = check_rows8(x8, x, 0)
        got = L.linear_q8(x.cuda(), w, bias.cuda())
        part = (q.double() @ qw.t()) * (s.double() * sw.t())
        close(got, part + bias.double(), 5 * U * (part.abs() + bias.double().abs()), dtype)
        assert torch.equal(L.linear_q8(x8, w, bias.cuda(), dtype), got)
        close(L.linear_q8(x8, w, dtype=dtype), part, 5 * U * part.abs(), dtype)
        if dtype != F32:
            close(L.linear_q8(x8, w, bias.to(dtype).cuda(), dtype), part + bias.to(dtype).double(), 5 * U * (part.abs() + bias.double().abs()), dtype)


def test_linear_sums_are_exact(L):
    """Products of the largest magnitudes whose sum passes what float32 holds, on each path."""
    for rows, cols in ((1, 131072), (20, 131072), (130, 4096), (700, 4096)):
        g = gen(rows)
        outs = 200
        q = torch.randint(-128, 128, (rows, cols), generator=g, dtype=torch.int8)
        p = torch.randint(-128, 128, (outs, cols), generator=g, dtype=torch.int8)
        q[0], p[0] = -128, -128                                           # 2^31 / 131072 each: 131072 would overflow, see below
        if cols == 131072:
            q[0, 0] = -127
        one = torch.ones(rows, 1), torch.ones(outs, 1)
        x8, w8 = L.Rows8(q.cuda(), one[0].cuda(), cols), L.Rows8(p.cuda(), one[1].cuda(), cols)
        want = q.double() @ p.double().t()
        assert float(want.abs().max()) <= 2.0 ** 31 - 1
        assert torch.equal(L.linear_q8(x8, w8).cpu(), want.float())       # (one rounding, of the exact sum)


@pytest.mark.parametrize("rows", [4, 90])
def test_linear_on_a_row_that_spoils_itself_only(L, rows):
    g = gen(11)
    x, w = values(g, rows, 300, F32), weights(L, g, 50, 300)
    x[1, 7], x[2, 9], x[3] = math.nan, -math.inf, 0.0
    y = L.linear_q8(x.cuda(), w).cpu()
    assert torch.isnan(y[1]).all() and torch.isnan(y[2]).all() and not y[3].any()
    assert torch.isfinite(y[[i for i in range(rows) if i not in (1, 2)]]).all()


LEFT = {F32: 2.0 ** -22, F16: 2.0 ** -15, BF16: 2.0 ** -8}            # of dy * scale, by the pieces


def check_linear_grads(got, dy, x8, w8, dtype):
    dx, dw, db = got
    dy = dy.double()
    x, w = rows8_values(x8), rows8_values(w8)
    rows, outs = dy.shape

    def tol(k, size):                                                  # (each piece's sum is float32, whatever the order)
        return (LEFT[dtype] + 2 * U + 2 * U * 3 * k) * size

    close(dx, dy @ w, tol(outs, dy.abs() @ w.abs()), dtype)
    close(dw, dy.t() @ x, tol(rows, dy.abs().t() @ x.abs()), dtype)
    close(db, dy.sum(0), (rows + 2) * U * dy.abs().sum(0), dtype)


@pytest.mark.parametrize("rows,cols,outs", LINEAR_SIZES)
@pytest.mark.parametrize("dtype", TYPES)
def test_linear_backward(L, rows, cols, outs, dtype):
    g = gen(rows + outs)
    w8 = weights(L, g, outs, cols)
    x8 = L.quantize_rows(values(g, rows, cols, F32).cuda())
    dy = values(g, rows, outs, dtype, size=0.01)
    got = L.linear_q8_backward(dy.cuda(), x8, w8)
    check_linear_grads(got, dy, x8, w8, dtype)
    again = L.linear_q8_backward(dy.cuda(), x8, w8)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


def test_linear_gradient_against_differences(L):
    g = gen(21)
    rows, cols, outs, h = 5, 30, 7, 1e-3
    w8 = weights(L, g, outs, cols)
    x8 = L.quantize_rows(torch.randn(rows, cols, generator=g).cuda())
    dy = torch.randn(rows, outs, generator=g)
    dx, dw, db = (t.cpu().double() for t in L.linear_q8_backward(dy.cuda(), x8, w8))
    at = [rows8_values(x8), rows8_values(w8), torch.zeros(outs).double()]

    def loss(x, w, b):
        return float(((x @ w.t() + b) * dy.double()).sum())

    for k, grad in enumerate((dx, dw, db)):
        v = torch.randn(at[k].shape, generator=g).double()
        up, down = (loss(*(t + s * h * v if i == k else t for i, t in enumerate(at))) for s in (1, -1))
        assert abs((up - down) / (2 * h) - float((grad * v).sum())) <= 1e-5 * float((grad * v).abs().sum()) + 1e-9


def test_large_and_small_gradients(L):
    """dy over the range of its type: the pieces neither overflow nor lose the small ones."""
    g = gen(22)
    rows, cols, outs = 70, 200, 90
    w8 = weights(L, g, outs, cols)
    x8 = L.quantize_rows(values(g, rows, cols, F32).cuda())
    for dtype, size in ((F32, 1e30), (F32, 1e-25), (BF16, 1e30), (BF16, 1e-25), (F16, 1e3), (F16, 1e-6)):
        dy = values(g, rows, outs, dtype, size=size)
        check_linear_grads(L.linear_q8_backward(dy.cuda(), x8, w8), dy, x8, w8, dtype)


# ---- sizes at which other kernels take over -----------------------------------------------------------------

MORE_NORMS = [(4200, 136), (4200, 1200), (4200, 1207), (1200, 1999), (1100, 2300), (400, 8100), (400, 9001), (600, 9000), (150, 16384), (130, 20001)]


@pytest.mark.parametrize("rows,cols", MORE_NORMS)
@pytest.mark.parametrize("dtype", TYPES)
def test_layer_norm_of_more_rows(L, rows, cols, dtype):
    """Workgroups that take several rows, and gradients whose sums do not fit the registers: bounds as above."""
    test_layer_norm(L, rows, cols, dtype)
    test_layer_norm_backward(L, rows, cols, dtype)


@pytest.mark.parametrize("rows,cols,outs", [(2100, 2100, 2100), (1030, 190, 2070), (1500, 1100, 2051), (300, 153, 587)])
@pytest.mark.parametrize("dtype", TYPES)
def test_linear_backward_of_more_rows(L, rows, cols, outs, dtype):
    """The largest tiles, sums cut along k, and dy by halves."""
    test_linear_backward(L, rows, cols, outs, dtype)


# ---- use ----------------------------------------------------------------------------------------------------

def test_no_rows(L):
    x = torch.empty(0, 130, device="cuda", dtype=BF16)
    w = weights(L, gen(1), 60, 130)
    assert L.dequantize_rows(L.quantize_rows(x, 128)).shape == (0, 130)
    y, mean, rstd, x8 = L.layer_norm(x, save=True)
    assert y.shape == (0, 130) and mean.shape == rstd.shape == (0,) and x8.q.shape == (0, 256)
    dx, dw, db = L.layer_norm_backward(x, x8, None, mean, rstd)
    assert dx.shape == (0, 130) and not dw.any() and not db.any() and dw.shape == (130,)
    assert L.linear_q8(x, w).shape == (0, 60)
    dx, dw, db = L.linear_q8_backward(torch.empty(0, 60, device="cuda", dtype=BF16), L.quantize_rows(x), w)
    assert dx.shape == (0, 130) and dw.shape == (60, 130) and not dw.any() and not db.any()


def test_more_dimensions(L):
    g = gen(2)
    x = values(g, 12, 96, BF16).cuda()
    w = weights(L, g, 40, 96)
    gamma = torch.randn(96, generator=g).cuda()
    for shape in ((96,), (3, 4, 96), (2, 3, 2, 96)):
        flat = x[:math.prod(shape[:-1])].reshape(-1, 96) if len(shape) > 1 else x[:1]
        v = flat.reshape(shape)
        y = L.layer_norm(v, gamma)[0]
        assert y.shape == v.shape and torch.equal(y.reshape(-1, 96), L.layer_norm(flat, gamma)[0])
        z = L.linear_q8(v, w)
        assert z.shape == shape[:-1] + (40,) and torch.equal(z.reshape(-1, 40), L.linear_q8(flat, w))
        _, mean, rstd = L.layer_norm(v, gamma)
        assert L.layer_norm_backward(y, v, gamma, mean, rstd)[0].shape == v.shape
        assert L.linear_q8_backward(z, L.quantize_rows(v), w)[0].shape == v.shape


def test_outputs_at_a_stride_leave_the_rest_alone(L):
    """Through the C calls: rows of y, dx and dw inside a larger array."""
    from paper_1803_03288_amd import binding
    g = gen(6)
    for rows, cols, outs in ((5, 100, 61), (150, 136, 264)):
        x, w = values(g, rows, cols, BF16).cuda(), weights(L, g, outs, cols)
        x8 = L.quantize_rows(x)
        dy = values(g, rows, outs, BF16).cuda()
        y, (dx, dw, _) = L.linear_q8(x, w), L.linear_q8_backward(dy, x8, w)
        room = [torch.full((r, c + 9), 5.0, dtype=BF16, device="cuda") for r, c in ((rows, outs), (rows, cols), (outs, cols))]
        space = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
        s = binding._stream()
        call("tictac_linear_q8", 2, rows, cols, outs, x.data_ptr(), cols, None, 0, None, w.q.data_ptr(), w.q.stride(0), w.scale.data_ptr(), 0, None,
                room[0].data_ptr() + 6, outs + 9, space.data_ptr(), space.numel(), s)
        call("tictac_linear_q8_backward", 2, rows, cols, outs, dy.data_ptr(), outs, x8.q.data_ptr(), x8.q.stride(0), x8.scale.data_ptr(), w.q.data_ptr(),
                w.q.stride(0), w.scale.data_ptr(), room[1].data_ptr() + 6, cols + 9, room[2].data_ptr() + 6, cols + 9, None, space.data_ptr(), space.numel(), s)
        for t, want in zip(room, (y, dx, dw)):
            n = want.shape[1]
            assert torch.equal(t[:, 3:3 + n], want)
            t[:, 3:3 + n] = 5.0
            assert bool((t == 5.0).all())


def test_another_stream_and_a_graph(L):
    """The same bits on a stream of the caller's and from a captured graph, replayed on new inputs."""
    g = gen(9)
    rows, cols, outs = 96, 520, 260
    w = weights(L, g, outs, cols)
    gamma = (1 + 0.2 * torch.randn(cols, generator=g)).cuda()
    inputs = [(values(g, rows, cols, BF16).cuda(), values(g, rows, outs, BF16).cuda()) for _ in range(3)]

    def step(x, dy):
        y8, mean, rstd, x8 = L.layer_norm_q8(x, gamma, save=True)
        y = L.linear_q8(y8, w, dtype=BF16)
        dn, dw, db = L.linear_q8_backward(dy, y8, w)
        return (y, dw, db) + L.layer_norm_backward(dn, x8, gamma, mean, rstd) + (L.linear_q8(x, w),)

    want = [step(*i) for i in inputs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for i, e in zip(inputs, want):
            assert all(torch.equal(a, b) for a, b in zip(step(*i), e))
    torch.cuda.current_stream().wait_stream(side)
    x, dy = (t.clone() for t in inputs[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(x, dy)
    for turn in range(2):
        for i, e in zip(inputs, want):
            x.copy_(i[0])
            dy.copy_(i[1])
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, e))
            assert all(torch.equal(a, b) for a, b in zip(step(*i), e))


def test_refusals(L):
    x = torch.randn(4, 256, device="cuda")
    w = L.quantize_rows(torch.randn(8, 256, device="cuda"))
    x8, kept = L.quantize_rows(x), L.quantize_rows(x, 128)
    mean = rstd = torch.ones(4, device="cuda")
    bad = [
        (ValueError, lambda: L.quantize_rows(x, 64)), (TypeError, lambda: L.quantize_rows(x.double())), (ValueError, lambda: L.quantize_rows(x.cpu())),
        (ValueError, lambda: L.quantize_rows(x[:, :0])), (TypeError, lambda: L.dequantize_rows(x8, torch.int8)),
        (ValueError, lambda: L.layer_norm(x, torch.ones(255, device="cuda"))), (TypeError, lambda: L.layer_norm(x, torch.ones(256, device="cuda").double())),
        (ValueError, lambda: L.layer_norm(x, torch.ones(256))),
        (TypeError, lambda: L.layer_norm(x.half(), torch.ones(256, device="cuda"), torch.ones(256, device="cuda").half())),
        (ValueError, lambda: L.layer_norm_backward(x, x8, None, mean, rstd)), (ValueError, lambda: L.layer_norm_backward(x[:3], x, None, mean, rstd)),
        (TypeError, lambda: L.layer_norm_backward(x.half(), x, None, mean, rstd)), (ValueError, lambda: L.layer_norm_backward(x, x, None, mean[:3], rstd)),
        (ValueError, lambda: L.linear_q8(x[:, :200], w)), (ValueError, lambda: L.linear_q8(kept, w)), (ValueError, lambda: L.linear_q8(x, kept)),
        (TypeError, lambda: L.linear_q8(x, w, dtype=torch.float16)), (ValueError, lambda: L.linear_q8(x, w, torch.ones(7, device="cuda"))),
        (ValueError, lambda: L.linear_q8(x, L.Rows8(w.q[:, :200], w.scale, 200))), (ValueError, lambda: L.linear_q8(x, L.Rows8(w.q, w.scale[:3], 256))),
        (ValueError, lambda: L.linear_q8_backward(x, x8, w)),
    ]
    for error, call in bad:
        with pytest.raises(error):
            call()
    from paper_1803_03288_amd import binding
    with pytest.raises(binding.TicTacError) as e:                       # the library's own: a stride that is no multiple of 128
        room = torch.zeros(8, 256 + 16, dtype=torch.int8, device="cuda")
        L.linear_q8(x, L.Rows8(room[:, :256], w.scale, 256))
    assert e.value.code == -9
    with pytest.raises(binding.TicTacError) as e:
        L.layer_norm(x, eps=-1.0)
    assert e.value.code == -9
