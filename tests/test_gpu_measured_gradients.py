"""Gradients of the measured iteration (``paper_1803_03288_amd.measured``) op by op."""

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
