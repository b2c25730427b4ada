"""Steps of training with the operators together (``paper_1803_03288_amd.measured``): norm, products in 8-bit floats and their gradients, the gradients' norm, AdamW with moments in
8 bits, and weights rounded again."""

import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import f8_reference as ref

measured = None


@pytest.fixture(scope="module", autouse=True)
def module():
    global measured
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1803_03288_amd import measured as m
    measured = m


def iteration(kind, dtype, n=2, rows=150, width=200, hidden=328, seed=3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x, target = (torch.randn(rows, width, generator=g, device="cuda") for _ in range(2))
    return getattr(measured, kind)(measured.random_layers(n, width, hidden, seed=seed + 1), x.to(dtype), target)


def rounded(x, block=1):
    q, scale, _ = ref.blocks(x, block)
    return q * scale


def definition(it):
    """The loss and the gradients of a BlockIteration of float32, in float64: roundings count as the identity."""
    x, target, kept = it.x.cpu().double(), it.target.cpu().double(), []
    stack = [[t.cpu().double() for t in p] for p in it.stack]
    weights = [(rounded(p[2].float(), 128), rounded(p[4].float(), 128)) for p in stack]
    for (gamma, beta, _, b1, _, b2), (w1, w2) in zip(stack, weights):
        mean, rstd = x.mean(1, keepdim=True), (x.var(1, unbiased=False, keepdim=True) + 1e-5) ** -0.5
        y = rounded((x - mean) * rstd * gamma + beta)
        u = y @ w1.t() + b1
        a = rounded(u.clamp(min=0))
        kept.append((x, mean, rstd, y, u, a))
        x = x + a @ w2.t() + b2
    loss, dx, grads = 0.5 * (x - target).square().mean(), (x - target) * (it.scale / x.numel()), []

    def backward(dy, x, w):
        return rounded(dy) @ w, rounded(ref.along(dy)) @ ref.along(rounded(ref.along(x))), dy.sum(0)

    for (gamma, *_), (w1, w2), (x, mean, rstd, y, u, a) in zip(stack[::-1], weights[::-1], kept[::-1]):
        du, dw2, db2 = backward(dx, a, w2)
        dn, dw1, db1 = backward(du * (u > 0), y, w1)
        h = (x - mean) * rstd
        d = dn * gamma
        dx = dx + rstd * (d - d.mean(1, keepdim=True) - h * (d * h).mean(1, keepdim=True))
        grads.append([t / it.scale for t in ((dn * h).sum(0), dn.sum(0), dw1, db1, dw2, db2)])
    return loss, grads[::-1]


def test_gradients_of_the_blocks():
    """Between the iteration in float32 and its definition lie the elements that round to the other neighbour, and relus that open on one side only.  A sum of 328 products is off by some 2^-20 of its
    size, a step of e4m3 is 2^-4 of the value at least: one element in 2^15 rounds otherwise, by 2^-3 of itself at most, or 2^-10 of the norm; four layers' products, each rounded three
    times on the way to a gradient, and as many roundings of x and w again: 16 of them at once are below 2^-6."""
    it = iteration("BlockIteration", torch.float32)
    loss, grads = it.run()
    want, exact = definition(it)
    assert abs(float(loss) - float(want)) <= 2.0 ** -6 * float(want)
    for got, d in zip(grads, exact):
        for name, a, b in zip(measured.Layer._fields, got, d):
            off = float((a.cpu().double() - b).norm() / b.norm())
            print(name, off, flush=True)
            assert a.dtype == torch.float32 and a.shape == b.shape and off <= 2.0 ** -6, name


@pytest.mark.parametrize("kind", ["Iteration", "BlockIteration"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("bits", [8, 32])
def test_steps_and_their_graph(kind, dtype, bits):
    """Steps as they are called and from a captured graph, replayed between other work: the same bits in losses, norms, parameters and weights."""
    its = [iteration(kind, dtype) for _ in range(2)]
    updates = [measured.Update(it, bits) for it in its]

    def step(it, update):
        it.refresh()                                        # (a graph reads what it wrote itself)
        loss, grads = it.run()
        return loss, update.run(grads)

    want = []
    for _ in range(5):
        loss, norm = step(its[0], updates[0])
        want.append((float(loss), float(norm)))
        if len(want) < 5:
            held = [t.clone() for t in updates[0].params]
    assert all(math.isfinite(v) for pair in want for v in pair) and all(not torch.equal(a, b) for a, b in zip(held, updates[0].params))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss, norm = step(its[1], updates[1])
    for k in range(5):
        graph.replay()
        torch.cuda.synchronize()
        assert (float(loss), float(norm)) == want[k]
        its[0].run()
    assert int(updates[1].step) == 5 and all(torch.equal(a, b) for a, b in zip(updates[0].params, updates[1].params))
    for a, b in zip(its[0].w1 + its[0].w2, its[1].w1 + its[1].w2):
        assert torch.equal(a.q.view(torch.uint8), b.q.view(torch.uint8)) and torch.equal(a.scale.view(torch.uint8), b.scale.view(torch.uint8))


def test_a_step_is_what_its_operators_give():
    """One update from an iteration's own gradients, clipped by their norm, against AdamW in 64 bits: bounds as in ``test_gpu_update``, with the clipping factor in float32 (three roundings more)."""
    it = iteration("BlockIteration", torch.bfloat16)
    _, grads = it.run()
    update = measured.Update(it, 32, lr=1e-2, max_norm=1e-3)
    flat = [t for d in grads for t in d]
    held = [t.cpu().double() for t in update.params]
    norm = update.run(grads)
    size = math.sqrt(sum(float(t.double().square().sum()) for t in flat))
    assert abs(float(norm) - size) <= 2 * ref.U * size and size > 1e-3
    for p, p0, g, m in zip(update.params, held, flat, update.moments):
        g = g.cpu().double() * (1e-3 / size)
        want, m1, v1 = ref.adamw(p0, g, torch.zeros_like(g), torch.zeros_like(g), 1, lr=1e-2)
        moved = 1e-2 * (m1 / 0.1).abs() / ((v1 / 1e-3).sqrt() + 1e-8)
        # (the first step: eps beside a gradient of any size, whose relative error is the factor's)
        off = (p.cpu().double() - want).abs() - ref.U * (4 * p0.abs() + 32 * moved) - 2.0 ** -140
        assert float(off.max()) <= 0
        assert float(((m.m.cpu().double().reshape(g.shape) - m1).abs() - 8 * ref.U * m1.abs() - 2.0 ** -149).max()) <= 0


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("bits", ["8", "32"])
def test_command(dtype, bits):
    out = measured.main(["--layers", "2", "--width", "200", "--hidden", "328", "--rows", "150", "--runs", "3", "--dtype", dtype, "--blocks", "--update", bits])
    update = out.pop("update")
    assert sorted(update) == ["update.norm", "update.step", "update.weights"] and all(0 < t < 1 for t in update.values())
    for found in out.values():
        for r in found.values():
            assert np.isfinite(r["makespan"]) and r["makespan"] >= r["bound"] > 0 and 0 <= r["efficiency"] <= 1
