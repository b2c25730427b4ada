"""AdamW over many tensors and the norm of their gradients (``paper_1803_03288_amd.layers``) against their definitions in 64 bits (``f8_reference``).

Tolerances count the float32 roundings on a value's way (``U`` each, the constants' own among them): m three, v four, the parameter's decayed part two and its step ten (m's,
half of v's, the root, the bias corrections, the quotient, the product); then half a step of the output's type.  Moments in 8 bits come from the same float32
operations in the same order, and are compared bit by bit."""

import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import f8_reference as ref
from f8_reference import U

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
TYPES = [F32, F16, BF16]
HALF = {F32: (2.0 ** -24, 2.0 ** -149), F16: (2.0 ** -11, 2.0 ** -25), BF16: (2.0 ** -8, 2.0 ** -134)}
SHAPES = [(1,), (7,), (8,), (127,), (128,), (129,), (33, 64), (2047,), (2048,), (4095,), (4097,), (3, 5, 7, 11), (10001,), (), (0,)]


@pytest.fixture(scope="module")
def L():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1803_03288_amd import layers
    return layers


def gen(seed):
    return torch.Generator().manual_seed(seed)


def state(L, g, shapes, dtype, grad, bits):
    p = [(torch.randn(s, generator=g) * 0.1).to(dtype).cuda() for s in shapes]
    d = [(torch.randn(s, generator=g) * 10.0 ** (i % 5 - 4)).to(grad).cuda() for i, s in enumerate(shapes)]
    moments = L.adamw_moments(p, bits)
    for t, m in zip(p, moments):
        n = t.numel()
        if bits == 32:
            m.m.copy_(torch.randn(n, generator=g) * 1e-3)
            m.v.copy_(torch.rand(n, generator=g) * 1e-5)
        elif n:
            for of, x in ((m.m, torch.randn(1, n, generator=g) * 1e-3), (m.v, torch.rand(1, n, generator=g) * 3e-3)):
                r = L.quantize_f8(x.cuda())
                of.q.copy_(r.q)
                of.scale.view(torch.uint8).copy_(r.scale.view(torch.uint8))
    return p, d, moments


def wide(m):
    """(m, v) in float64."""
    if torch.is_tensor(m.m):
        return flat(m.m), flat(m.v)
    return ref.values(m.m)[0], ref.values(m.v)[0] ** 2


def close(got, want, bound, dtype):
    got = got.cpu().double()
    rel, least = HALF[dtype]
    off = (got - want).abs() - (bound + rel * (want.abs() + bound) + least)
    assert got.shape == want.shape and torch.isfinite(got).all()
    assert got.numel() == 0 or float(off.max()) <= 0, float(off.max())


def flat(t):
    """The elements in the order in which they lie, float64."""
    return torch.as_strided(t, (t.numel(),), (1,)).cpu().double()


def float32_moments(before, g, scale, betas):
    """m and the root of v in 8 bits as the step forms them before rounding: float32 operations, each rounded by itself."""
    b1, b2 = betas
    f = lambda v: torch.tensor(v, dtype=F32)  # noqa: E731
    m, r = (ref.values(x)[0].float() for x in before)
    x = g.float() * f(scale)
    v = (r * r) * f(b2) + (x * x) * f(1 - b2)
    return m * f(b1) + x * f(1 - b1), torch.sqrt(v)


def check(L, p, d, moments, step, copies=None, scale=1.0, seed=0, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=1e-2, **more):
    before = [(flat(t), wide(m), [type(x)(x.q.clone(), x.scale.clone(), x.cols, x.block) for x in m] if not torch.is_tensor(m.m) else None) for t, m in zip(p, moments)]
    L.adamw_step(p, d, moments, step, lr=lr, betas=betas, eps=eps, weight_decay=weight_decay, copies=copies, seed=seed, **more)
    for i, (t, g, m, (p0, (m0, v0), kept)) in enumerate(zip(p, d, moments, before)):
        if t.numel() == 0:
            continue
        gd = torch.empty_strided(t.shape, t.stride(), dtype=g.dtype, device="cuda").copy_(g)        # in the parameter's order
        gd = flat(gd) * scale
        want, m1, v1 = ref.adamw(p0, gd, m0, v0, step, lr, betas, eps, weight_decay)
        size_m = betas[0] * m0.abs() + (1 - betas[0]) * gd.abs()
        quotient = (v1 / (1 - betas[1] ** step)).sqrt() + eps
        moved = abs(lr) * size_m / (1 - betas[0] ** step) / quotient
        bound = U * (2 * p0.abs() + 2 * abs(lr) * weight_decay * p0.abs() + 16 * moved) + 2.0 ** -140
        close(flat(t), want, bound, t.dtype)
        if copies and copies[i] is not None:
            close(flat(copies[i]), want, bound + U * want.abs(), copies[i].dtype)
        if kept is None:
            close(flat(m.m), m1, 5 * U * size_m, F32)
            close(flat(m.v), v1, 7 * U * v1, F32)
        else:
            mf, rf = float32_moments(kept, torch.as_strided(torch.empty_strided(t.shape, t.stride(), dtype=g.dtype, device="cuda").copy_(g), (t.numel(),), (1,)).cpu(), scale, betas)
            bits = ref.random_bits(seed, step, i, t.numel())
            for of, x, u in ((m.m, mf, bits & 0xFFFF), (m.v, rf, bits >> 16)):
                q, byte = ref.at_random(x, u)
                assert torch.equal(of.scale.cpu().view(torch.uint8)[0, :byte.numel()], byte)
                assert torch.equal(of.q.cpu()[0, :t.numel()].double(), q) and not of.q.cpu().view(torch.uint8)[0, t.numel():].any()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("grad", TYPES)
def test_adamw(L, dtype, grad, bits):
    g = gen(1)
    p, d, moments = state(L, g, SHAPES, dtype, grad, bits)
    copies = [torch.full_like(t, 7.0, dtype=(BF16, F16)[i % 2]) if i % 3 else None for i, t in enumerate(p)] if dtype == F32 else None
    for step in (1, 2, 1000):
        check(L, p, d, moments, step, copies, seed=step << 33 | 5)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_options(L, bits):
    g = gen(2)
    for more in (dict(lr=0.1, betas=(0.0, 0.0), eps=1e-3, weight_decay=0.0), dict(lr=0.0), dict(betas=(0.99, 0.9), weight_decay=0.5, lr=-1e-2), dict(grad_scale=2.0 ** -10, scale=2.0 ** -10)):
        p, d, moments = state(L, g, [(300,), (40, 50)], F32, F32, bits)
        check(L, p, d, moments, 3, **more)


def test_more_tensors_than_a_launch_describes(L):
    g = gen(3)
    shapes = [(1 + (i * 37) % 400,) for i in range(203)]
    p, d, moments = state(L, g, shapes, BF16, BF16, 32)
    small = [L.adamw_moments([t], 8)[0] if i % 2 else m for i, (t, m) in enumerate(zip(p, moments))]        # some in 8 bits, some in 32
    check(L, p, d, small, 10, seed=9)
    want = math.sqrt(sum(float(t.double().square().sum()) for t in d))
    assert abs(float(L.gradient_norm(d)) - want) <= 2 * U * want


def test_large_tensors(L):
    """More chunks than workgroups of the norm; a tensor's end inside a chunk."""
    g = gen(4)
    n = (1 << 24) + 4097
    d = [torch.randn(n, generator=g).cuda(), torch.randn(1000, generator=g).cuda().to(BF16)]
    want = math.sqrt(sum(float(t.double().square().sum()) for t in d)) * 0.5
    norm = L.gradient_norm(d, 0.5)
    assert norm.shape == () and abs(float(norm) - want) <= 2 * U * want
    p = [torch.zeros(n, device="cuda"), torch.zeros(1000, device="cuda")]
    for bits in (8, 32):
        moments = L.adamw_moments(p, bits)
        L.adamw_step(p, d, moments, 1, lr=1.0, weight_decay=0.0, eps=0.0)
        for t, grad in zip(p, d):                           # the first step from zeros: the gradient's sign
            assert float((t + torch.sign(grad.float())).abs().max()) <= 16 * U
            t.zero_()


@pytest.mark.parametrize("bits", [32, 8])
def test_places_and_strides(L, bits):
    """Parameters at odd places and in other orders than rows; gradients in another order or apart; moments with the parameter's strides."""
    g = gen(5)
    room = torch.randn(4000, generator=g).cuda()
    p = [room[1:1001], room[1003:2003].reshape(20, 50).t(), torch.randn(2, 6, 5, 4, generator=g).cuda().contiguous(memory_format=torch.channels_last), room.to(BF16)[2051:2300]]
    d = [torch.randn(2000, generator=g).cuda()[::2], torch.randn(50, 20, generator=g).cuda(), torch.randn(2, 6, 5, 4, generator=g).cuda().half(), torch._neg_view(torch.randn(249, generator=g).cuda())]
    moments = L.adamw_moments(p, bits)
    copies = [None, torch.empty(20, 50, device="cuda", dtype=F16).t(), None, None]
    rest = room.clone()
    for step in (1, 2):
        check(L, p, d, moments, step, copies)
    rest[1:1001], rest[1003:2003] = room[1:1001], room[1003:2003]
    assert torch.equal(rest, room)                          # what lies between is left alone
    if bits == 32:
        m = [L.Moments(torch.zeros_like(p[1]), torch.zeros_like(p[1]))]
        check(L, p[1:2], d[1:2], m, 1)


def test_norm_and_clipping(L):
    g = gen(6)
    shapes = [(3000,), (70, 130), (1,)]
    for grad in TYPES:
        p, d, moments = state(L, g, shapes, F32, grad, 32)
        want = math.sqrt(sum(float(t.double().square().sum()) for t in d)) / 8
        norm = L.gradient_norm(d, 1 / 8)
        assert abs(float(norm) - want) <= 2 * U * want
        for most in (want / 3, want * 3):
            scale = float(torch.tensor(1 / 8, dtype=F32) * torch.clamp(torch.tensor(most, dtype=F32) / norm.cpu(), max=1.0))
            check(L, p, d, moments, 5, scale=scale, grad_scale=1 / 8, norm=norm, max_norm=most)
    # no gradient at all, and squares that leave float32's range on both sides
    zero = [torch.zeros(5, device="cuda"), torch.zeros(0, device="cuda")]
    assert float(L.gradient_norm(zero)) == 0
    for size in (1e30, 1e-30):
        t = torch.full((1000,), size, device="cuda")
        assert abs(float(L.gradient_norm([t])) / (size * math.sqrt(1000)) - 1) < 1e-6
    p, _, moments = state(L, g, [(5,), (0,)], F32, F32, 32)
    check(L, p, zero, moments, 2, norm=L.gradient_norm(zero), max_norm=1.0)
    assert torch.equal(L.gradient_norm(d), L.gradient_norm(d))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_no_step_with_gradients_that_are_not_finite(L, bits, bad):
    g = gen(7)
    p, d, moments = state(L, g, [(300,), (77,)], F32, F16, bits)
    copies = [torch.zeros(300, device="cuda", dtype=BF16), None]
    d[1][5] = bad
    norm = L.gradient_norm(d)
    assert not math.isfinite(float(norm))
    held = [t.clone() for m in moments for x in m for t in ([x] if torch.is_tensor(x) else [x.q.view(torch.uint8), x.scale.view(torch.uint8)])] + [t.clone() for t in p]
    L.adamw_step(p, d, moments, 1, norm=norm, copies=copies)
    now = [t for m in moments for x in m for t in ([x] if torch.is_tensor(x) else [x.q.view(torch.uint8), x.scale.view(torch.uint8)])] + p
    assert all(torch.equal(a, b) for a, b in zip(held, now)) and not copies[0].any()
    # without the norm the step is taken, and what is not finite spoils its element, in 8 bits its block
    L.adamw_step(p, d, moments, 1)
    assert torch.isfinite(p[0]).all() and not torch.isfinite(p[1][5]) and torch.isfinite(p[1][:5]).all()
    if bits == 8:
        assert torch.isnan(moments[1].m.q[0, :77].float()).all() and not moments[1].m.q[0, 77:].float().any()


def test_moments_in_8_bits_follow_those_in_32(L):
    """Over many steps of one gradient and its noise the moments stay unbiased: their means over 8192 elements, against those in 32 bits.  A step's rounding is off by at most a step of
    the type, 2^-3 of the value, with mean zero; what is left of 1000 of them after the decay is below 2^-3 / sqrt(8192) times sqrt(0.125 / 2 * 1000) of a value, or 1.1 %; bound 5 %."""
    g = gen(8)
    n = 8192
    p = [torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")]
    m8, m32 = L.adamw_moments(p[:1], 8), L.adamw_moments(p[1:], 32)
    torch.manual_seed(0)
    for step in range(1, 1201):
        d = [0.3 + torch.randn(n, device="cuda")]
        L.adamw_step(p[:1], d, m8, step, lr=1e-3, weight_decay=0.0)
        L.adamw_step(p[1:], d, m32, step, lr=1e-3, weight_decay=0.0)
    a, b = ref.values(m8[0].v)[0], m32[0].v.cpu().double().sqrt()
    assert abs(float(a.mean() / b.mean()) - 1) < 0.05
    assert abs(float((ref.values(m8[0].m)[0].mean() - m32[0].m.double().mean()).abs())) < 0.05 * float(m32[0].m.double().abs().mean())
    assert abs(float(p[0].mean() / p[1].mean()) - 1) < 0.05


@pytest.mark.parametrize("bits", [32, 8])
def test_a_captured_step_goes_on(L, bits):
    """step and lr from the device, read at every replay; the same bits as steps by numbers, and two graphs of one state in turn."""
    g = gen(9)
    shapes = [(500,), (33, 70), (1,)]
    p, d, moments = state(L, g, shapes, F32, BF16, bits)
    q = [t.clone() for t in p]
    other = [L.Moments(*(x.clone() if torch.is_tensor(x) else L.Float8(x.q.clone(), x.scale.clone(), x.cols, x.block) for x in m)) for m in moments]
    step, lr = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(1, device="cuda")
    grads = [t.clone() for t in d]

    def run():
        step.add_(1)
        norm = L.gradient_norm(grads)
        L.adamw_step(p, grads, moments, step, lr=lr, norm=norm, max_norm=0.5, seed=3)

    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for graph in graphs:
        with torch.cuda.graph(graph):
            run()
    for k in range(1, 7):
        rate = 1e-3 / k
        lr.fill_(rate)
        for t, s in zip(grads, d):
            t.copy_(s * (1 + k))
        graphs[k % 2].replay()
        torch.cuda.synchronize()
        L.adamw_step(q, grads, other, k, lr=float(lr), norm=L.gradient_norm(grads), max_norm=0.5, seed=3)
        for a, b in zip(p, q):
            assert float((a - b).abs().max()) <= 4 * U * float(b.abs().max() + rate)       # (the factors of a step are formed by other functions on the device)
        for m, o in zip(moments, other):
            for x, y in zip(m, o):
                assert torch.equal(x, y) if torch.is_tensor(x) else torch.equal(x.q.view(torch.uint8), y.q.view(torch.uint8)) and torch.equal(x.scale.view(torch.uint8), y.scale.view(torch.uint8))
    assert int(step) == 6


def test_another_stream(L):
    g = gen(10)
    p, d, moments = state(L, g, [(5000,), (77,)], F32, F32, 8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        check(L, p, d, moments, 4, norm=L.gradient_norm(d))
    torch.cuda.current_stream().wait_stream(side)


def test_autograd_sees_the_change(L):
    """What a backward pass kept of a parameter is not used after a step has changed it."""
    w = torch.randn(8, device="cuda", requires_grad=True)
    loss = (w * w).sum()
    L.adamw_step([w], [torch.ones(8, device="cuda")], L.adamw_moments([w], 8), 1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_refusals(L):
    p = [torch.randn(300, device="cuda"), torch.randn(4, 5, device="cuda")]
    d = [torch.randn_like(t) for t in p]
    m8, m32 = L.adamw_moments(p, 8), L.adamw_moments(p, 32)
    one = torch.ones(1, device="cuda")
    half = L.Moments(m8[0].m, m32[0].v)
    e5 = L.quantize_f8(p[0][None], 1, torch.float8_e5m2)
    room = torch.zeros(1, 16, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)
    odd = L.Float8(m8[0].m.q, room[:, 1:13], 300)
    bad = [
        (ValueError, lambda: L.adamw_step(p, d[:1], m8, 1)), (ValueError, lambda: L.adamw_step(p, d, m8[:1], 1)), (ValueError, lambda: L.adamw_step(p, d, m8, 0)),
        (TypeError, lambda: L.adamw_step(p, d, m8, 1.5)), (TypeError, lambda: L.adamw_step(p, d, m8, 1, lr="a")), (ValueError, lambda: L.adamw_step(p, d, m8, one)),
        (ValueError, lambda: L.adamw_step(p, d, m8, torch.ones(1, dtype=torch.int64))), (ValueError, lambda: L.adamw_step(p, d, m8, 1, lr=torch.ones(2, device="cuda"))),
        (ValueError, lambda: L.adamw_step(p, d, m8, 1, betas=(0.9,))), (ValueError, lambda: L.adamw_step(p, d, m8, 1, max_norm=1.0)), (ValueError, lambda: L.adamw_step(p, d, m8, 1, norm=one, max_norm=0.0)),
        (ValueError, lambda: L.adamw_step(p, [d[0], d[1].t()], m8, 1)), (TypeError, lambda: L.adamw_step(p, [d[0], d[1].double()], m8, 1)), (ValueError, lambda: L.adamw_step(p, [d[0], d[1].cpu()], m8, 1)),
        (ValueError, lambda: L.adamw_step([p[0][::2]], [d[0][::2]], L.adamw_moments([p[0][::2]]), 1)), (ValueError, lambda: L.adamw_step([p[0][:1].expand(9)], [d[0][:9]], L.adamw_moments([d[0][:9]]), 1)),
        (TypeError, lambda: L.adamw_step([p[0].double()], d[:1], m8[:1], 1)), (TypeError, lambda: L.adamw_step(p, d, [m8[0], p[1]], 1)), (ValueError, lambda: L.adamw_step(p, d, [m8[0], m8[0]], 1)),
        (ValueError, lambda: L.adamw_step(p[:1], d[:1], [half], 1)), (ValueError, lambda: L.adamw_step(p[:1], d[:1], [L.Moments(e5, e5)], 1)), (ValueError, lambda: L.adamw_step(p[:1], d[:1], [L.Moments(odd, m8[0].v)], 1)),
        (ValueError, lambda: L.adamw_step(p, d, m8, 1, copies=[None])), (ValueError, lambda: L.adamw_step(p, d, m8, 1, copies=[None, d[1].t()])), (TypeError, lambda: L.gradient_norm([p[0].double()])),
        (ValueError, lambda: L.gradient_norm([p[0].cpu()])), (TypeError, lambda: L.adamw_step(p, d, m8, 1, seed="x")),
    ]
    held = [t.clone() for t in p]
    for error, call in bad:
        with pytest.raises(error):
            call()
    from paper_1803_03288_amd import binding
    for call in (lambda: L.adamw_step([p[0], p[0]], [d[0], d[0]], [m8[0], L.adamw_moments(p[:1])[0]], 1), lambda: L.adamw_step(p, d, m8, 1, betas=(1.0, 0.9)), lambda: L.adamw_step(p, d, m8, 1, eps=-1.0),
                 lambda: L.adamw_step(p[:1], d[:1], m8[:1], 1, copies=[p[0]]), lambda: L.gradient_norm(d, math.inf)):
        with pytest.raises(binding.TicTacError) as e:
            call()
        assert e.value.code == -9
    assert all(torch.equal(a, b) for a, b in zip(held, p))
