"""The measured iteration (``paper_1803_03288_amd.measured``): its graph on the CPU, and a small one run, timed and ordered on the GPU."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import oracle
from paper_1803_03288_amd import measured


def test_graph_of_the_iteration():
    g = measured.iteration_graph(3, 64, 256)
    n, row_ptr, col_idx, recv_ids = g.csr()
    assert len(g.recvs) == 15 and len(g.ops) == 31 and n == 46
    assert list(recv_ids) == list(range(15)) and not np.diff(row_ptr)[:15].any()            # recvs are roots
    assert all(col_idx[row_ptr[v]:row_ptr[v + 1]].max() < v for v in range(15, n))          # in the order in which they run
    dep = oracle.find_dependencies(n, row_ptr, col_idx, recv_ids)
    names = [r[0] for r in g.recvs] + [o[0] for o in g.ops]
    bits = {name: {i for i in range(15) if int(dep[v, 0]) >> i & 1} for v, name in enumerate(names)}
    assert bits["forward.norm0"] == {0} and bits["forward.linear1.0"] == {0, 1, 2} and bits["forward.add0"] == {0, 1, 2, 3, 4}
    assert bits["forward.norm1"] == {0, 1, 2, 3, 4, 5} and bits["loss"] == bits["backward.add0"] == set(range(15))
    assert g.recvs[1] == ("w1.0", 64 * 256 + 4 * 256, 4 * 64 * 256)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
def test_measured_iteration(dtype):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    out = measured.main(["--layers", "2", "--width", "200", "--hidden", "328", "--rows", "150", "--runs", "3", "--dtype", dtype])
    for found in out.values():
        for r in found.values():
            assert np.isfinite(r["makespan"]) and r["makespan"] >= r["bound"] > 0 and 0 <= r["efficiency"] <= 1
        assert found["tac"]["makespan"] <= found["random"]["makespan"] * (1 + 1e-12)
    assert out["8 bits"]["tac"]["makespan"] < out["32 bits"]["tac"]["makespan"]


@pytest.mark.gpu
def test_gradients_lead_downhill():
    """A step along the gradients of the whole stack lowers the loss by what they say, up to second order and rounding."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    g = torch.Generator(device="cuda").manual_seed(3)
    stack = measured.random_layers(2, 128, 256, seed=4)
    it = measured.Iteration(stack, torch.randn(300, 128, generator=g, device="cuda"), torch.randn(300, 128, generator=g, device="cuda"))
    loss, grads = it.run()
    names = measured.Layer._fields
    size = sum(float(getattr(d, n).double().square().sum()) for d in grads for n in names)
    step = 0.02 * float(loss) / size                                    # to lower the loss by 2 %, to first order
    it.stack = [measured.Layer(*(getattr(p, n) - step * getattr(d, n) for n in names)) for p, d in zip(stack, grads)]
    it.refresh()
    after, _ = it.run()
    assert 0.01 * float(loss) < float(loss) - float(after) < 0.03 * float(loss)
