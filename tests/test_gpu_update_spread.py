"""AdamW with moments in 8 bits where the gradients of one block of 128 have very different sizes (``paper_1803_03288_amd.layers``).

e4m3 spans 2^-17 of a block's largest value and a half.  The root of the second moment divides the step, so a positive root is not rounded to zero: elements below that
range count as of one step of the type, and move less.

A single step.  |m| <= B sqrt(v), B = (1 - b1) / sqrt(1 - b2) / sqrt(1 - b1^2 / b2) = 7.27 for (0.9, 0.999), by Cauchy and Schwarz over the gradients so far; the bias corrections' quotient is 1 at most
where B is reached, and 3.2 at the first step, where |m| = 3.2 sqrt(v).  The stored root is no less than half of the root, and no less than a step q_r of the type; the stored m is off
by a step q_m of its own type, q_m / q_r <= 2 max|m| / max sqrt(v) <= 2 B.  So a step is at most 4 B = 29.1 learning rates.

The way of 300 steps.  1 / root is at most 9 / 8 of what it is on average (a value between one and two steps), which goes to the way of float32 moments as a factor; a rounding
of m, off by q_m at most and unbiased, lives on for sum b1^i = 10 steps, so the way's standard deviation is at most 10 sqrt(300) q_m / q_r learning rates."""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import f8_reference as ref
from test_gpu_update import L, float32_moments, gen  # noqa: F401

RATIOS = [1.0, 2.0 ** -10, 2.0 ** -14, 2.0 ** -17, 2.0 ** -18, 2.0 ** -20, 2.0 ** -24]
B = 0.1 / 0.001 ** 0.5 / (1 - 0.81 / 0.999) ** 0.5


def sizes(ratio, blocks=16):
    """One element of size 1 in each block of 128, the others at a ratio."""
    s = torch.full((blocks, 128), ratio)
    s[:, 0] = 1.0
    return s.flatten()


@pytest.mark.parametrize("ratio", RATIOS)
@pytest.mark.parametrize("kind", ["noise", "drift", "rare"])
def test_elements_far_below_their_blocks_largest(L, ratio, kind):  # noqa: F811
    g, lr, steps = gen(1), 1e-3, 300
    size = sizes(ratio)
    n = size.numel()
    p8, p32 = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    m8, m32 = L.adamw_moments([p8], 8), L.adamw_moments([p32], 32)
    largest = torch.zeros(n, device="cuda")
    for step in range(1, steps + 1):
        x = torch.randn(n, generator=g)
        if kind == "drift":
            x = 1 + 0.1 * x
        elif kind == "rare":
            x = x * (torch.rand(n, generator=g) < 0.01)
        d = [(x * size).cuda()]
        before = p8.clone()
        L.adamw_step([p8], d, m8, step, lr=lr, weight_decay=0.0)
        L.adamw_step([p32], d, m32, step, lr=lr, weight_decay=0.0)
        largest = torch.maximum(largest, (p8 - before).abs())
    small = size.cuda() < 1 if ratio < 1 else size.cuda() > 0
    way, way32 = float(p8[small].abs().max()), float(p32[small].abs().max())
    print(kind, ratio, "largest step", float(largest.max()) / lr, "way", way, "in 32 bits", way32, flush=True)
    assert float(largest.max()) <= 4 * B * lr
    ratio_q = 2 * float(m32[0].m.abs().max() / m32[0].v.sqrt().max())
    assert way <= 9 / 8 * way32 + 5 * 10 * steps ** 0.5 * max(2.0, ratio_q) * lr


@pytest.mark.parametrize("betas", [(0.9, 0.999), (0.0, 0.0)])
def test_the_least_root(L, betas):  # noqa: F811
    """Bit by bit: roots from far below one step of the type to well above it, and exact zeros, which stay."""
    g = gen(2)
    n = 128 * 40 + 77
    d = torch.randn(n, generator=g) * 2.0 ** (-30 * torch.rand(n, generator=g))
    d[::128], d[5::9] = 1.0, 0.0
    p = [torch.zeros(n, device="cuda")]
    moments = L.adamw_moments(p, 8)
    below = 0
    for step in range(1, 4):
        kept = [type(x)(x.q.clone(), x.scale.clone(), x.cols, x.block) for x in moments[0]]
        L.adamw_step(p, [d.cuda()], moments, step, betas=betas, seed=7)
        m, r = float32_moments(kept, d, 1.0, betas)
        bits = ref.random_bits(7, step, 0, n)
        below += int(((ref.at_random(r, bits >> 16)[0] == 0) & (r > 0)).sum())
        for of, (q, byte) in ((moments[0].m, ref.at_random(m, bits & 0xFFFF)), (moments[0].v, ref.root_at_random(r, bits >> 16))):
            assert torch.equal(of.scale.cpu().view(torch.uint8)[0, :byte.numel()], byte)
            assert torch.equal(of.q.cpu()[0, :n].double(), q) and not of.q.cpu().view(torch.uint8)[0, n:].any()
        assert torch.equal(moments[0].v.q.cpu()[0, :n].double() == 0, r == 0)
    assert below > 1000                                     # (there were such roots)


@pytest.mark.parametrize("tensors", [58, 59])
def test_every_tensor_of_full_launches(L, tensors):  # noqa: F811
    """Moments of zeros: a step's new parameters do not depend on random bits, so each tensor's are what it gets by itself."""
    g = torch.Generator(device="cuda").manual_seed(tensors)
    d = [torch.randn(1 + 300 * i % 977, generator=g, device="cuda") for i in range(tensors)]
    p, q = ([torch.ones_like(t) for t in d] for _ in range(2))
    L.adamw_step(p, d, L.adamw_moments(p, 8), 3)
    for a, b, t in zip(p, q, d):
        L.adamw_step([b], [t], L.adamw_moments([b], 8), 3)
        assert torch.equal(a, b) and not torch.equal(a, torch.ones_like(a))
