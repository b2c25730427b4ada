"""A worker's iteration with measured times: ``python -m paper_1803_03288_amd.measured``.

The graphs of ``workloads`` stand in for traced models; here the ops are run.  A stack of residual layers

    x <- x + relu(norm(x) W1' + b1) W2' + b2

takes its weights as 8-bit rows, as they would be transferred, and keeps its activations in 8 bits for the backward pass (``layers``), with a mask of
where the relu is flat: what is positive and rounds to zero has a gradient.  With ``--blocks`` both are 8-bit floats with a scale per block of 128 instead, and the norms
keep their inputs as they are; with ``--update`` the server's part, AdamW over all parameters, is run and timed as well.
Every op of a training iteration is timed on the device in several runs; the smallest time of each is the time oracle (Sec. 5,
"Time Oracle": ``time_oracle_min``).  The graph of the iteration (recvs are roots, a gradient op depends on the gradient behind it, on the forward op whose
activations it reads and on the weights it reads) then gets its TIC and TAC orders and the makespan and Scheduling
Efficiency of the iteration under each, beside transfers in random order, with the parameters in 8 and in 32 bits.
"""

from __future__ import annotations

import argparse
import math
from typing import Callable, Dict, List, NamedTuple, Tuple

import numpy as np
import torch

from .workloads import LINK_BITS_PER_S


class Layer(NamedTuple):
    """Parameters of one residual layer: float32 vectors and matrices."""
    gamma: torch.Tensor
    beta: torch.Tensor
    w1: torch.Tensor            # [hidden][width]
    b1: torch.Tensor
    w2: torch.Tensor            # [width][hidden]
    b2: torch.Tensor


def random_layers(n: int, width: int, hidden: int, seed: int = 0) -> List[Layer]:
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    return [Layer(1 + 0.1 * normal(width), 0.1 * normal(width), normal(hidden, width) / width ** 0.5, 0.1 * normal(hidden),
                  normal(width, hidden) / hidden ** 0.5, 0.1 * normal(width)) for _ in range(n)]


class Graph:
    """Ops with their predecessors: recvs first, then compute ops in the order in which they run."""

    def __init__(self):
        self.recvs: List[Tuple[str, int, int]] = []         # name, bytes in 8 bits, bytes in 32 bits
        self.ops: List[Tuple[str, List[str]]] = []

    def recv(self, name: str, bytes8: int, bytes32: int) -> str:
        self.recvs.append((name, bytes8, bytes32))
        return name

    def op(self, name: str, *after: str) -> str:
        self.ops.append((name, list(after)))
        return name

    def csr(self):
        """``(n_ops, row_ptr, col_idx, recv_ids)`` as ``binding.build_deps`` takes them."""
        at = {name: i for i, name in enumerate([r[0] for r in self.recvs] + [o[0] for o in self.ops])}
        R = len(self.recvs)
        preds = [[] for _ in range(R)] + [[at[a] for a in after] for _, after in self.ops]
        row_ptr = np.concatenate([[0], np.cumsum([len(p) for p in preds])]).astype(np.int32)
        return len(preds), row_ptr, np.array([a for p in preds for a in p], dtype=np.int32), np.arange(R, dtype=np.int32)


def iteration_graph(n: int, width: int, hidden: int, blocks: bool = False) -> Graph:
    """The iteration of ``Iteration.run`` (``blocks``: of ``BlockIteration.run``), op by op."""
    g = Graph()
    vector, matrix = 4 * width, width * hidden
    scales1, scales2 = (4 * hidden, 4 * width) if not blocks else (-(-width // 128) * -(-hidden // 128),) * 2      # a float per output, or a byte per block
    params = []
    for i in range(n):
        params.append((g.recv(f"norm{i}", 2 * vector, 2 * vector),
                       g.recv(f"w1.{i}", matrix + scales1, 4 * matrix), g.recv(f"b1.{i}", 4 * hidden, 4 * hidden),
                       g.recv(f"w2.{i}", matrix + scales2, 4 * matrix), g.recv(f"b2.{i}", vector, vector)))
    before = None
    for i, (norm, w1, b1, w2, b2) in enumerate(params):
        x = [before] if before else []
        g.op(f"forward.norm{i}", norm, *x)
        g.op(f"forward.linear1.{i}", f"forward.norm{i}", w1, b1)
        g.op(f"forward.relu{i}", f"forward.linear1.{i}")
        g.op(f"forward.linear2.{i}", f"forward.relu{i}", w2, b2)
        before = g.op(f"forward.add{i}", f"forward.linear2.{i}", *x)
    before = g.op("loss", before)
    for i in reversed(range(n)):
        norm, w1, _, w2, _ = params[i]
        g.op(f"backward.linear2.{i}", before, f"forward.relu{i}", w2)
        g.op(f"backward.relu{i}", f"backward.linear2.{i}", f"forward.relu{i}")
        g.op(f"backward.linear1.{i}", f"backward.relu{i}", f"forward.norm{i}", w1)
        g.op(f"backward.norm{i}", f"backward.linear1.{i}", f"forward.norm{i}", norm)
        before = g.op(f"backward.add{i}", f"backward.norm{i}", before)
    return g


class Iteration:
    """One training iteration of a stack of layers; every op goes through ``op(name, call)``, which may time it."""

    def __init__(self, stack: List[Layer], x: torch.Tensor, target: torch.Tensor):
        from . import layers
        self.layers, self.stack, self.x, self.target = layers, stack, x, target
        # The loss is a mean: its gradients in float16 would be subnormal (2^-22 at 4096 x 1024).  They are taken times a power of two, and what is returned is
        # divided by it in float32: values of dx are then of the order of 1 / sqrt(rows), their sums over the rows of sqrt(rows) at most.
        self.scale = 2.0 ** round(math.log2(x.shape[1] * math.sqrt(max(1, x.shape[0]))))
        self.refresh()

    def refresh(self) -> None:
        """The weights as they are sent: 8-bit rows, a scale per output."""
        self.w1 = [self.layers.quantize_rows(p.w1) for p in self.stack]
        self.w2 = [self.layers.quantize_rows(p.w2) for p in self.stack]

    # what an op of a layer calls, and what is kept of its input
    def norm(self, x, p):
        return self.layers.layer_norm_q8(x, p.gamma, p.beta, save=True)

    def linear(self, x, w, bias):
        return self.layers.linear_q8(x, w, bias, self.x.dtype)

    def rounded(self, x):
        return self.layers.quantize_rows(x)

    def linear_backward(self, dy, x, w):
        return self.layers.linear_q8_backward(dy, x, w)

    def run(self, op: Callable = lambda name, call: call()):
        """``(loss, gradients)``: a ``Layer`` of float32 gradients for each layer."""
        x, kept = self.x, []
        for i, p in enumerate(self.stack):
            y8, mean, rstd, x8 = op(f"forward.norm{i}", lambda: self.norm(x, p))
            u = op(f"forward.linear1.{i}", lambda: self.linear(y8, self.w1[i], p.b1))
            flat, u8 = op(f"forward.relu{i}", lambda: (u <= 0, self.rounded(u.relu_())))       # (a NaN is not flat)
            v = op(f"forward.linear2.{i}", lambda: self.linear(u8, self.w2[i], p.b2))
            kept.append((y8, mean, rstd, x8, flat, u8))
            x = op(f"forward.add{i}", lambda: x + v)
        dx, loss = op("loss", lambda: self._loss(x))
        grads: List[Layer] = []
        for i in reversed(range(len(self.stack))):
            p, (y8, mean, rstd, x8, flat, u8) = self.stack[i], kept.pop()
            du, dw2, db2 = op(f"backward.linear2.{i}", lambda: self.linear_backward(dx, u8, self.w2[i]))
            du = op(f"backward.relu{i}", lambda: du.masked_fill_(flat, 0))
            dn, dw1, db1 = op(f"backward.linear1.{i}", lambda: self.linear_backward(du, y8, self.w1[i]))
            dn, dgamma, dbeta = op(f"backward.norm{i}", lambda: self.layers.layer_norm_backward(dn, x8, p.gamma, mean, rstd))
            dx = op(f"backward.add{i}", lambda: dx + dn)
            grads.append(Layer(*(t.float() / self.scale for t in (dgamma, dbeta, dw1, db1, dw2, db2))))
        return loss, grads[::-1]

    def _loss(self, x):
        d = x.float() - self.target
        return (d * (self.scale / d.numel())).to(x.dtype), 0.5 * d.square().mean()


class BlockIteration(Iteration):
    """The iteration with weights and kept activations in 8-bit floats with a scale per block of 128; the norms keep their inputs as they are."""

    def refresh(self) -> None:
        self.w1 = [self.layers.quantize_f8(p.w1, 128) for p in self.stack]
        self.w2 = [self.layers.quantize_f8(p.w2, 128) for p in self.stack]

    def norm(self, x, p):
        y, mean, rstd = self.layers.layer_norm(x, p.gamma, p.beta)
        return self.layers.quantize_f8(y), mean, rstd, x

    def linear(self, x, w, bias):
        return self.layers.linear_f8(x, w, bias, self.x.dtype)

    def rounded(self, x):
        return self.layers.quantize_f8(x)

    def linear_backward(self, dy, x, w):
        return self.layers.linear_f8_backward(dy, x, w)


class Update:
    """The parameter server's part of a step: the gradients' norm, AdamW over all parameters of an iteration's layers, in place, and the weights as they are sent next."""

    def __init__(self, it: Iteration, bits: int = 8, lr: float = 1e-3, max_norm: float = 1.0):
        self.it, self.max_norm = it, max_norm
        self.params = [t for p in it.stack for t in p]
        self.moments = it.layers.adamw_moments(self.params, bits)
        # on the device, so that a captured step goes on
        self.step = torch.zeros(1, dtype=torch.int64, device=it.x.device)
        self.lr = torch.full((1,), lr, device=it.x.device)

    def run(self, grads: List[Layer], op: Callable = lambda name, call: call()):
        """Takes one step, where the gradients' norm is finite; that norm."""
        ly, flat = self.it.layers, [t for d in grads for t in d]
        norm = op("update.norm", lambda: ly.gradient_norm(flat))
        self.step.add_(norm < math.inf)                     # (a step that changes nothing is not counted)
        op("update.step", lambda: ly.adamw_step(self.params, flat, self.moments, self.step, lr=self.lr, norm=norm, max_norm=self.max_norm))
        op("update.weights", self.it.refresh)
        return norm


def measure(it: Iteration, names: List[str], runs: int) -> torch.Tensor:
    """Seconds of every op in each run, float64 ``[runs][ops]`` on the device, in the order of ``names``."""
    it.run()                                                # (the first run loads the kernels)
    return _timed(it.run, names, runs)


def measure_update(it: Iteration, bits: int, runs: int) -> Dict[str, float]:
    """Seconds of the ops of ``Update.run``, the smallest of each."""
    from . import binding as tt
    _, grads = it.run()
    update, names = Update(it, bits), ["update.norm", "update.step", "update.weights"]
    update.run(grads)
    return dict(zip(names, tt.time_oracle_min(_timed(lambda op: update.run(grads, op), names, runs)).tolist()))


def _timed(run: Callable, names: List[str], runs: int) -> torch.Tensor:
    at = {name: i for i, name in enumerate(names)}
    times = torch.zeros(runs, len(names), dtype=torch.float64)
    for r in range(runs):
        events = []

        def timed(name, call):
            begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            begin.record()
            out = call()
            end.record()
            events.append((at[name], begin, end))
            return out

        run(timed)
        torch.cuda.synchronize()
        for i, begin, end in events:
            times[r, i] = begin.elapsed_time(end) * 1e-3
    return times.cuda()


def orders(graph: Graph, op_time: torch.Tensor, recv_time: np.ndarray, seed: int = 0, samples: int = 64) -> Dict[str, Dict[str, float]]:
    """Makespan (s) and Scheduling Efficiency of the iteration with the transfers in random order (mean over ``samples``), by TIC and by TAC."""
    from . import binding as tt
    dag = tt.build_deps(*graph.csr())
    R = len(graph.recvs)
    recv = torch.from_numpy(np.broadcast_to(recv_time, (samples, R)).copy()).cuda()
    op = op_time.reshape(1, -1).expand(samples, -1).contiguous()
    shuffled = np.random.default_rng(seed).permuted(np.tile(np.arange(R, dtype=np.int32), (samples, 1)), axis=1)
    random = tt.simulate(dag, torch.from_numpy(shuffled).cuda(), op, recv)
    tic = tt.simulate(dag, tt.tic_priority(dag)[1], op, recv)
    tac = tt.tac_simulate(dag, op, recv)[4:]
    out = {name: {"makespan": float(r[0].mean()), "efficiency": float(r[1].mean()), "bound": float(r[3].max())} for name, r in (("random", random), ("tic", tic), ("tac", tac))}
    dag.close()
    return out


def main(argv=None) -> Dict[str, Dict]:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--layers", type=int, default=8)
    ap.add_argument("--width", type=int, default=1024)
    ap.add_argument("--hidden", type=int, default=4096)
    ap.add_argument("--rows", type=int, default=4096, help="rows (tokens, samples) of a worker's batch")
    ap.add_argument("--runs", type=int, default=5, help="measured runs of the iteration")
    ap.add_argument("--link", type=float, default=LINK_BITS_PER_S / 1e9, help="Gb/s of the link to the parameter server (that of the presets)")
    ap.add_argument("--dtype", choices=("bfloat16", "float16", "float32"), default="bfloat16")
    ap.add_argument("--blocks", action="store_true", help="weights and kept activations in 8-bit floats with a scale per block of 128")
    ap.add_argument("--update", type=int, choices=(8, 32), help="run and time the server's update too, with moments in so many bits")
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args(argv)
    from . import binding as tt
    graph = iteration_graph(a.layers, a.width, a.hidden, a.blocks)
    g = torch.Generator(device="cuda").manual_seed(a.seed + 1)
    x = torch.randn(a.rows, a.width, generator=g, device="cuda").to(getattr(torch, a.dtype))
    it = (BlockIteration if a.blocks else Iteration)(random_layers(a.layers, a.width, a.hidden, a.seed), x, torch.randn(a.rows, a.width, generator=g, device="cuda"))
    names = [name for name, _ in graph.ops]
    op_time = tt.time_oracle_min(measure(it, names, a.runs))
    out = {}
    print(f"{len(names)} ops, {len(graph.recvs)} recvs; all ops {1e3 * float(op_time.sum()):.3f} ms")
    for bits, column in ((8, 1), (32, 2)):
        recv_time = 8.0 * np.array([r[column] for r in graph.recvs], dtype=np.float64) / (a.link * 1e9)
        out[f"{bits} bits"] = found = orders(graph, op_time, recv_time, a.seed)
        print(f"parameters in {bits} bits: transfers {1e3 * recv_time.sum():.3f} ms")
        for name, r in found.items():
            print(f"  {name:6s} makespan {1e3 * r['makespan']:.3f} ms, efficiency {r['efficiency']:.3f}")
    if a.update:
        out["update"] = measure_update(it, a.update, a.runs)
        print(f"update with moments in {a.update} bits: " + ", ".join(f"{name[7:]} {1e3 * t:.3f} ms" for name, t in out["update"].items()))
    return out


if __name__ == "__main__":
    main()
