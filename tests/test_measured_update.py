"""The server's update in the measured iteration (``paper_1803_03288_amd.measured``): which steps count."""

import math
from types import SimpleNamespace

import pytest
import torch

from paper_1803_03288_amd import layers, measured


def test_steps_that_are_not_taken_do_not_count():
    """``adamw_step`` changes nothing where the norm is not finite, so the next one has the same number."""
    norms, seen, refreshed = [math.inf, 2.0, math.nan, 3.0, 0.0], [], []

    class Layers:
        adamw_moments = staticmethod(layers.adamw_moments)

        @staticmethod
        def gradient_norm(grads):
            return torch.tensor(norms[len(seen)])

        @staticmethod
        def adamw_step(params, grads, moments, step, **more):
            seen.append((float(more["norm"]), int(step)))

    stack = [measured.Layer(*(torch.ones(4) for _ in measured.Layer._fields))]
    update = measured.Update(SimpleNamespace(layers=Layers, stack=stack, x=torch.ones(2), refresh=lambda: refreshed.append(1)), 32)
    for _ in norms:
        update.run(stack)
    assert [step for norm, step in seen if math.isfinite(norm)] == [1, 2, 3]
    assert int(update.step) == 3 and len(refreshed) == 5


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [8, 32])
def test_a_skipped_step_leaves_no_trace(bits):
    """An overflow, then a step: the bits of a first step, as it is called and from a captured graph."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")

    def one():
        g = torch.Generator(device="cuda").manual_seed(5)
        x, target = (torch.randn(70, 96, generator=g, device="cuda") for _ in range(2))
        it = measured.BlockIteration(measured.random_layers(1, 96, 136, seed=6), x, target)
        return it, measured.Update(it, bits)

    (a, first), (b, second), (c, third) = one(), one(), one()
    grads = a.run()[1]
    held = [measured.Layer(*(t.clone() for t in d)) for d in grads]
    bad = [measured.Layer(*(torch.full_like(t, math.inf) for t in d)) for d in grads]
    first.run(grads)
    second.run(bad)
    assert all(torch.equal(s, t) for s, t in zip(second.params, third.params)) and int(second.step) == 0
    second.run(held)
    flow = [measured.Layer(*(t.clone() for t in d)) for d in bad]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        third.run(flow)
    for now, steps in ((bad, 0), (bad, 0), (held, 1)):
        for d, s in zip(flow, now):
            for t, u in zip(d, s):
                t.copy_(u)
        graph.replay()
        torch.cuda.synchronize()
        assert int(third.step) == steps
    assert int(first.step) == int(second.step) == 1
    for s, t, u in zip(first.params, second.params, third.params):
        assert torch.equal(s, t) and torch.equal(s, u)
