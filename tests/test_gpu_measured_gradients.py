"""Gradients of the measured iteration (``paper_1803_03288_amd.measured``) op by op."""

import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_1803_03288_amd import measured


def run_and_keep(it, *names):
    """The outputs of the named ops as they were when the op ended (some are changed in place by the next)."""
    kept = {}

    def op(name, call):
        out = call()
        if name in names:
            kept[name] = out.clone() if isinstance(out, torch.Tensor) else out[0].clone()
        return out

    return it.run(op), kept


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_relu_passes_the_gradients_of_what_rounds_to_zero(dtype):
    """A large activation in a row makes the small ones zero in 8 bits; they are positive all the same.  A row of NaN keeps its gradients."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    g = torch.Generator(device="cuda").manual_seed(7)
    rows, width, hidden = 40, 128, 256
    p = measured.random_layers(1, width, hidden, seed=8)[0]
    b1 = p.b1.clone()
    b1[5] = 1e4
    x = torch.randn(rows, width, generator=g, device="cuda").to(dtype)
    x[3, 7] = float("nan")
    it = measured.Iteration([p._replace(b1=b1)], x, torch.randn(rows, width, generator=g, device="cuda"))
    (_, grads), kept = run_and_keep(it, "forward.linear1.0", "backward.linear2.0", "backward.relu0")
    u, du, got = kept["forward.linear1.0"], kept["backward.linear2.0"], kept["backward.relu0"]
    assert bool(torch.isnan(u[3]).all()) and int(((u > 0) & (u < 39)).sum()) > rows * hidden // 4       # (1e4 / 254 = 39)
    assert torch.equal(torch.nan_to_num(got, nan=9.0), torch.nan_to_num(torch.where(u <= 0, torch.zeros_like(du), du), nan=9.0))
    assert bool(torch.isnan(got[3]).any()) and bool(torch.isnan(grads[0].w1).any())


def test_float16_gradients_of_a_mean_over_many():
    """At 4096 x 1024 the loss's own gradients are subnormal in float16: they are taken times a power of two, each rounded to 11 bits.  The iteration's
    are as near to float32's as its activations are.  Bound of those: activations in float16 step to another 8-bit value in one of 16 places, by 1 / 127 of a row's largest (some four times the typical one): 1 % of
    their norm, on two layers' ops and both passes."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    g = torch.Generator(device="cuda").manual_seed(9)
    rows, width = 4096, 1024
    stack = measured.random_layers(2, width, 1024, seed=10)
    x, target = (torch.randn(rows, width, generator=g, device="cuda") for _ in range(2))
    x = x.half()
    (loss32, want), _ = run_and_keep(measured.Iteration(stack, x.float(), target))
    (loss16, got), kept = run_and_keep(measured.Iteration(stack, x, target), "forward.add1", "loss")
    dx, exact = kept["loss"].double(), (kept["forward.add1"].double() - target.double()) / target.numel()
    scale = 2.0 ** round(math.log2(float(dx.norm() / exact.norm())))
    assert float((dx - scale * exact).norm()) <= 2.0 ** -11 * scale * float(exact.norm())
    assert abs(float(loss16) - float(loss32)) <= 1e-2 * float(loss32)
    for a, b in zip(got, want):
        for name in measured.Layer._fields:
            s, t = getattr(a, name), getattr(b, name)
            off = float((s - t).norm() / t.norm())
            print(name, off, flush=True)
            assert s.dtype == torch.float32 and off <= 0.04, name
