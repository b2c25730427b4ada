"""The definitions behind products in 8-bit floats and the update, on the CPU: for tests.

Powers of two as scales make rounding exact arithmetic, so blocks are compared bit by bit.  What the matrix instructions for 8-bit floats cut off follows from how they add: of
eight products of neighbouring k each is cut, toward zero, at 2^-13 of the power of two of the largest (the sum of the two operands' exponents, those of subnormal values
being the least of the type); the rest is float32.  So seven of eight are off by less than 2^-13 of the largest, or of what the least exponents would give."""

import torch

F8 = {torch.float8_e4m3fn: (448.0, -6, 3), torch.float8_e5m2: (57344.0, -14, 2)}        # largest, least exponent, bits of fraction
U = 2.0 ** -24


def exponent(x):
    """floor(log2 |x|) of float64 values, 0 for 0."""
    return torch.where(x == 0, torch.zeros_like(x), torch.frexp(x)[1].double() - 1)


def two_to(e):
    return torch.ldexp(torch.ones_like(e, dtype=torch.float64), e.to(torch.int32))


def blocks(x, block=1, dtype=torch.float8_e4m3fn):
    """``(q, scale, byte)``: the values of the type and the scales, each [rows][cols] in float64, and the bytes of the scales [blocks of rows][blocks of columns]."""
    largest, least, bits = F8[dtype]
    x = x.double().cpu()
    rows, cols = x.shape
    up, along = -(-rows // block), -(-cols // 128)
    amax = torch.zeros(up * block, along * 128, dtype=torch.float64)
    amax[:rows, :cols] = x.abs()
    amax = amax.reshape(up, block, along, 128).amax((1, 3))
    bad = ~torch.isfinite(amax)
    m, e = torch.frexp(torch.where(bad, torch.ones_like(amax), amax))       # (0.5 <= m < 1; largest = 0.875 2^top)
    top = 9 if largest == 448.0 else 16
    e = torch.where(amax == 0, torch.full_like(e, -126), (e - top + (m > 0.875).int()).clamp(min=-126))
    byte = torch.where(bad, torch.full_like(e, 255), e + 127).to(torch.uint8)
    wide = lambda t: t.repeat_interleave(block, 0).repeat_interleave(128, 1)[:rows, :cols]  # noqa: E731
    scale = wide(two_to(e))
    y = x / scale
    step = two_to(exponent(y).clamp(min=least) - bits)
    q = torch.where(wide(bad), torch.full_like(y, float("nan")), torch.round(torch.nan_to_num(y) / step) * step)
    below = 2.0 ** 128 / scale * (1 - 2.0 ** -(bits + 1))                   # the largest value that float32 holds too
    return torch.where(q.abs() * scale >= 2.0 ** 128, torch.copysign(below, q), q), scale, byte


def parts(r):
    """``(q, scale)`` of a Float8, each [rows][cols] in float64."""
    rows = r.q.shape[0]
    byte = r.scale.cpu().view(torch.uint8)[:, :-(-r.cols // 128)]
    e = byte.double() - 127
    s = torch.where(byte == 255, torch.full_like(e, float("nan")), two_to(e))
    return r.q.cpu()[:, :r.cols].double(), s.repeat_interleave(r.block, 0).repeat_interleave(128, 1)[:rows, :r.cols]


def values(r):
    q, s = parts(r)
    return q * s


def along(t):
    return t.t().contiguous()


def product(a, b, cut):
    """``(sums, bound)`` of a @ b.T for operands (q, scale, least exponent of the type), k last: with `cut` by the matrix instructions for 8-bit floats, else by those for bf16."""
    (qa, sa, la), (qb, sb, lb) = a, b
    k = qa.shape[1]
    want, size = (qa * sa) @ along(qb * sb), (qa * sa).abs() @ along((qb * sb).abs())
    bound = 2 * U * (k + 16) * size
    if cut:
        def groups(q, s, least):
            m = torch.where(q == 0, torch.zeros_like(q), q.abs().clamp(min=2.0 ** least)) * s
            return torch.nn.functional.pad(m, (0, -k % 8)).reshape(m.shape[0], -1, 8).amax(2)
        bound = bound + 7 * 2.0 ** -13 * groups(qa, sa, la) @ along(groups(qb, sb, lb))
    return want, bound


def gradients(dy, x, w, dtype, cut):
    """``((dx, bound), (dw, bound))`` from dy, and Float8 x and w."""
    def operand(v, dt):
        q, s, _ = blocks(v, 1, dt)
        return q, s, F8[dt][1]

    e4 = torch.float8_e4m3fn
    if w.block == 128:
        q, s = parts(w)
        wc = (along(q), along(s), -6)
        again = operand(along(values(w)), e4)              # (the same values; where a block has other exponents the cut may differ)
        assert torch.equal(again[0] * again[1], wc[0] * wc[1])
        wc = again
    else:
        wc = operand(along(values(w)), e4)
    dx = product(operand(dy, dtype), wc, cut)
    dw = product(operand(along(dy), dtype), operand(along(values(x)), e4), cut)
    return dx, dw


# ---- the update ----

def mixed(x):
    x = ((x ^ (x >> 16)) * 0x9E3779B9) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0x6A09E667) & 0xFFFFFFFF
    return x ^ (x >> 16)


def random_bits(seed, step, index, n):
    key = torch.tensor(0, dtype=torch.int64)
    for part in (seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF, step & 0xFFFFFFFF, index):
        key = mixed((key + part) & 0xFFFFFFFF)
    return mixed((key + torch.arange(n)) & 0xFFFFFFFF)


def at_random(x, bits):
    """``(q, byte)`` of a row x (float32) in e4m3 blocks, rounded by 16 random bits an element: exact arithmetic in float64 but for one float32 sum."""
    n = x.numel()
    _, scale, byte = blocks(x.reshape(1, -1))
    y = x.double() / scale[0]
    step = two_to(exponent(y).clamp(min=-6) - 3)
    t = (y.abs() / step).float() + bits.float() * 2.0 ** -16                # (the quotient is exact; the sum is rounded as float32)
    return torch.copysign(torch.floor(t).double() * step, y)[:n], byte[0]


def root_at_random(x, bits):
    """The same for the root of the second moment: a positive one is a step of the type at least (the last, 2^-9 of the scale; larger values have eight steps and more)."""
    q, byte = at_random(x, bits)
    return torch.where((q == 0) & (x > 0), torch.full_like(q, 2.0 ** -9), q), byte


def adamw(p, g, m, v, step, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=1e-2):
    """New (p, m, v) in float64."""
    b1, b2 = betas
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    return p - lr * weight_decay * p - lr * (m / (1 - b1 ** step)) / ((v / (1 - b2 ** step)).sqrt() + eps), m, v
