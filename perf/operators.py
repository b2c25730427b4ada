"""Timed cases of the operators of a worker's layers: ``paper_1803_03288_amd.layers``.

A worker's iteration receives its parameters as transfers and runs ops on them.  These are the ops whose
parameters come as 8-bit rows with a scale per output channel, and whose activations are kept in 8 bits for the
backward pass.

Kinds
-----
checkpoint   activations kept in 8 bits, a scale per 128 columns, and brought back: ``quantize_rows``, ``dequantize_rows``.
norm         layer norm, forward; with ``save`` also the checkpoint of its input, brought back as the backward pass has it.
norm_grad    layer norm, backward, from its input (``saved`` "exact") or from the 8-bit checkpoint of it ("rows8").
linear       a product with 8-bit weights; the input is rounded to 8 bits, a scale per row, within the call.
norm_linear  layer norm with its output in 8 bits, and the product that takes it.
linear_grad  gradients of the product's input, weights and bias from the 8-bit rows that the forward pass kept.

8-bit rows are int8 ``[rows][ld]``, ``ld`` the number of columns rounded up to 128, zeros behind the last column, and
float32 scales: ``x = q * s`` with ``s = amax / 127``, ``q = round(x * (127 / amax))``.
"""

from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5
GROUP = 128
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}


# ---- the cases ----------------------------------------------------------------------------------------------

def listed():
    return [
        # activations of a small batch before a classifier of 1 000 outputs, an odd number of rows
        {"name": "checkpoint small", "kind": "checkpoint", "rows": 33, "cols": 1000, "dtype": "f32"},
        # the activations of a large batch between two layers
        {"name": "checkpoint large", "kind": "checkpoint", "rows": 16384, "cols": 4096, "dtype": "bf16"},
        # one token or sample while serving
        {"name": "norm one row", "kind": "norm", "rows": 1, "cols": 4096, "dtype": "bf16", "save": False},
        # a training batch: the output and the checkpoint of the input
        {"name": "norm training", "kind": "norm", "rows": 8192, "cols": 4096, "dtype": "bf16", "save": True},
        # a small training batch on the exact input, odd width, float32
        {"name": "norm_grad small", "kind": "norm_grad", "rows": 77, "cols": 1023, "dtype": "f32", "saved": "exact"},
        # a large training batch from the 8-bit checkpoint
        {"name": "norm_grad large", "kind": "norm_grad", "rows": 16384, "cols": 4096, "dtype": "bf16", "saved": "rows8"},
        # the second fully connected layer of VGG-16 for one sample
        {"name": "linear one row", "kind": "linear", "rows": 1, "cols": 4096, "outs": 4096, "dtype": "bf16"},
        # its first one for the batch of 32 images that the preset has
        {"name": "linear vgg16 fc6", "kind": "linear", "rows": 32, "cols": 25088, "outs": 4096, "dtype": "f16"},
        # a pre-norm layer that widens four times, large batch
        {"name": "norm_linear large", "kind": "norm_linear", "rows": 8192, "cols": 4096, "outs": 16384, "dtype": "bf16"},
        # a narrow layer on a small batch in float32, nothing a multiple of anything
        {"name": "linear_grad small", "kind": "linear_grad", "rows": 101, "cols": 777, "outs": 1001, "dtype": "f32"},
        # VGG-16's first fully connected layer, training with 32 images: the gradient of the weights is written once
        {"name": "linear_grad vgg16 fc6", "kind": "linear_grad", "rows": 32, "cols": 25088, "outs": 4096, "dtype": "f16"},
        # a large batch through a square layer
        {"name": "linear_grad large", "kind": "linear_grad", "rows": 8192, "cols": 4096, "outs": 4096, "dtype": "bf16"},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["checkpoint", "norm", "norm_grad", "linear", "norm_linear", "linear_grad"])
    # (a layer whose 8-bit operand comes out of float32 arithmetic has 16-bit outputs)
    case = {"kind": kind, "dtype": rng.choice(["f16", "bf16"] if kind == "norm_linear" else ["f32", "f16", "bf16"])}
    if kind in ("checkpoint", "norm", "norm_grad"):
        cols = _log(rng, 64, 16384)
        if rng.random() < 0.5:
            cols = -(-cols // 64) * 64
        case.update(rows=_log(rng, 1, max(1, min(16384, (1 << 26) // cols))), cols=cols)
        if kind == "norm":
            case["save"] = rng.random() < 0.5
        if kind == "norm_grad":
            case["saved"] = rng.choice(["exact", "rows8"])
        return case
    cols, outs = _log(rng, 64, 25088), _log(rng, 64, 16384)
    if rng.random() < 0.5:
        cols, outs = -(-cols // 64) * 64, -(-outs // 64) * 64
    most = (8192 * 4096 * 16384 if kind != "linear_grad" else 8192 * 4096 * 4096) // (cols * outs)
    case.update(rows=_log(rng, 1, max(1, min(8192, most))), cols=cols, outs=outs)
    return case


# ---- inputs -------------------------------------------------------------------------------------------------

def _activations(g, rows, cols, dtype):
    """Normal values on an offset, rows of different sizes, a few columns several times as large (as layers have them)."""
    x = torch.randn(rows, cols, generator=g, device="cuda")
    size = torch.exp(0.5 * torch.randn(rows, 1, generator=g, device="cuda"))
    wide = torch.where(torch.rand(cols, generator=g, device="cuda") < 0.01, 6.0, 1.0)
    return ((x * wide + 0.25) * size).to(dtype)


def _gradients(g, rows, cols, dtype):
    x = torch.randn(rows, cols, generator=g, device="cuda")
    return (x * 1e-2 * torch.exp(0.5 * torch.randn(rows, 1, generator=g, device="cuda"))).to(dtype)


def _padded(q):
    """int8 rows at a stride of a multiple of 128, zeros behind the last column."""
    rows, cols = q.shape
    out = torch.zeros(rows, -(-cols // 128) * 128, dtype=torch.int8, device=q.device)
    out[:, :cols] = q
    return out


def _weights(g, outs, cols):
    """A layer's weights as they arrive: 8-bit rows, a scale per output channel."""
    w = torch.randn(outs, cols, generator=g, device="cuda") / math.sqrt(cols)
    q, s = _rows8(w, 0)
    return _padded(q), s


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dtype, rows, cols = DTYPES[case["dtype"]], case["rows"], case["cols"]
    state = dict(case, eps=EPS, dtype=dtype)
    kind = case["kind"]
    if kind == "linear_grad":
        x = _activations(g, rows, cols, torch.float32)
        q, s = _rows8(x, 0)
        state.update(dy=_gradients(g, rows, case["outs"], dtype), xq=_padded(q), xs=s)
    else:
        state["x"] = _activations(g, rows, cols, dtype)
    if kind in ("norm", "norm_grad", "norm_linear"):
        state["gamma"] = 1.0 + 0.2 * torch.randn(cols, generator=g, device="cuda")
        state["beta"] = 0.1 * torch.randn(cols, generator=g, device="cuda")
    if kind == "norm_grad":
        state["dy"] = _gradients(g, rows, cols, dtype)
        x = state["x"].float()
        mean = x.mean(1)
        state["mean"], state["rstd"] = mean, torch.rsqrt((x - mean[:, None]).square().mean(1) + EPS)
        if case["saved"] == "rows8":
            q, s = _rows8(x, GROUP)
            state.update(xq=_padded(q), xs=s)
            del state["x"]
    if kind in ("linear", "norm_linear", "linear_grad"):
        state["wq"], state["ws"] = _weights(g, case["outs"], cols)
        if kind != "linear_grad":
            state["bias"] = 0.1 * torch.randn(case["outs"], generator=g, device="cuda")
    return state


# ---- the operators in their plain form ----------------------------------------------------------------------

def _groups(x, group):
    """[rows][groups][columns of a group], zeros behind the last column."""
    rows, cols = x.shape
    group = group or cols
    n = -(-cols // group)
    if n * group != cols:
        x = torch.cat([x, x.new_zeros(rows, n * group - cols)], 1)
    return x.reshape(rows, n, group)


def _rows8(x, group):
    rows, cols = x.shape
    x = _groups(x.float(), group)
    amax = x.abs().amax(2, keepdim=True)
    small = amax < 2.0 ** -116
    most = torch.full_like(amax, 127.0)         # (a quotient of tensors is one division; with a number it is a reciprocal and a product)
    q = torch.where(small, 0.0, torch.round(x * (most / amax)))
    s = torch.where(small, 0.0, amax / most)
    return q.to(torch.int8).reshape(rows, -1)[:, :cols], s[:, :, 0]


def _values(q, s, cols, group):
    x = _groups(q[:, :cols].float(), group) * s[:, :, None]
    return x.reshape(q.shape[0], -1)[:, :cols]


def _norm(x, gamma, beta, eps):
    x = x.float()
    mean = x.mean(1, keepdim=True)
    d = x - mean
    rstd = torch.rsqrt(d.square().mean(1, keepdim=True) + eps)
    return d * rstd * gamma + beta, mean[:, 0], rstd[:, 0]


def _product(q, s, wq, ws, cols, bias):
    return (q[:, :cols].float() @ wq[:, :cols].float().t()) * (s * ws.t()) + bias


def _run_plain(st):
    kind, dtype, cols = st["kind"], st["dtype"], st["cols"]
    if kind == "checkpoint":
        q, s = _rows8(st["x"], GROUP)
        return _values(q, s, cols, GROUP).to(dtype)
    if kind == "norm":
        y, mean, rstd = _norm(st["x"], st["gamma"], st["beta"], st["eps"])
        if not st["save"]:
            return y.to(dtype), mean, rstd
        q, s = _rows8(st["x"], GROUP)
        return y.to(dtype), mean, rstd, _values(q, s, cols, GROUP).to(dtype)
    if kind == "norm_grad":
        x = st["x"].float() if st["saved"] == "exact" else _values(st["xq"], st["xs"], cols, GROUP)
        dy = st["dy"].float()
        xh = (x - st["mean"][:, None]) * st["rstd"][:, None]
        g = dy * st["gamma"]
        dx = st["rstd"][:, None] * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
        return dx.to(dtype), (dy * xh).sum(0), dy.sum(0)
    if kind == "linear":
        q, s = _rows8(st["x"], 0)
        return _product(q, s, st["wq"], st["ws"], cols, st["bias"]).to(dtype)
    if kind == "norm_linear":
        y, mean, rstd = _norm(st["x"], st["gamma"], st["beta"], st["eps"])
        q, s = _rows8(y, 0)
        return _product(q, s, st["wq"], st["ws"], cols, st["bias"]).to(dtype), mean, rstd
    dy, w = st["dy"].float(), st["wq"][:, :cols].float() * st["ws"]
    x = st["xq"][:, :cols].float() * st["xs"]
    return (dy @ w).to(dtype), (dy.t() @ x).to(dtype), dy.sum(0).to(dtype)


def _run_own(st):
    from paper_1803_03288_amd import layers
    kind, dtype, cols = st["kind"], st["dtype"], st["cols"]
    if kind == "checkpoint":
        return layers.dequantize_rows(layers.quantize_rows(st["x"], GROUP), dtype)
    if kind == "norm":
        if not st["save"]:
            return layers.layer_norm(st["x"], st["gamma"], st["beta"], st["eps"])
        y, mean, rstd, saved = layers.layer_norm(st["x"], st["gamma"], st["beta"], st["eps"], save=True)
        return y, mean, rstd, layers.dequantize_rows(saved, dtype)
    if kind == "norm_grad":
        x = st["x"] if st["saved"] == "exact" else layers.Rows8(st["xq"], st["xs"], cols, GROUP)
        return layers.layer_norm_backward(st["dy"], x, st["gamma"], st["mean"], st["rstd"])
    w = layers.Rows8(st["wq"], st["ws"], cols)
    if kind == "linear":
        return layers.linear_q8(st["x"], w, st["bias"])
    if kind == "norm_linear":
        y, mean, rstd = layers.layer_norm_q8(st["x"], st["gamma"], st["beta"], st["eps"])
        return layers.linear_q8(y, w, st["bias"], dtype), mean, rstd
    return layers.linear_q8_backward(st["dy"], layers.Rows8(st["xq"], st["xs"], cols), w)


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- what a pass cannot do without --------------------------------------------------------------------------

def work(case):
    t, k, size, kind = case["rows"], case["cols"], SIZE[case["dtype"]], case["kind"]
    saved = t * k + 4 * t * -(-k // GROUP)                  # a checkpoint in 8 bits
    if kind == "checkpoint":
        return {"bytes": 2 * t * k * size + 2 * saved, "flops": 4 * t * k}
    if kind == "norm":
        more = (2 * saved + t * k * size, 4 * t * k) if case["save"] else (0, 0)
        return {"bytes": 2 * t * k * size + 8 * k + 8 * t + more[0], "flops": 8 * t * k + more[1]}
    if kind == "norm_grad":
        x = t * k * size if case["saved"] == "exact" else saved
        return {"bytes": 2 * t * k * size + x + 8 * t + 12 * k, "flops": 14 * t * k}
    n = case["outs"]
    weights = n * k + 4 * n
    if kind in ("linear", "norm_linear"):
        norm = (8 * k + 8 * t, 8 * t * k) if kind == "norm_linear" else (0, 0)
        return {"bytes": t * k * size + weights + 4 * n + t * n * size + norm[0], "flops": 2 * t * k * n + 4 * t * k + norm[1]}
    return {"bytes": t * n * size + (t * k + 4 * t) + weights + (t * k + n * k + n) * size, "flops": 4 * t * k * n + 3 * t * n}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------

def _exact_rows(x, width):
    """What 8 bits keep of the rows of x, a scale per `width` columns: whole multiples of amax/127."""
    back = torch.empty_like(x)
    for lo in range(0, x.shape[1], width):
        part = x[:, lo:lo + width]
        step = part.abs().max(1, keepdim=True).values / 127
        back[:, lo:lo + width] = torch.where(step > 0, torch.round(part / step) * step, torch.zeros_like(part))
    return back


def exact(case, seed):
    st = prepare(case, seed)
    kind, cols = case["kind"], case["cols"]
    f64 = lambda name: st[name].double()  # noqa: E731
    if kind == "checkpoint":
        return _exact_rows(f64("x"), GROUP)
    if kind in ("linear", "linear_grad", "norm_linear"):
        w = f64("wq")[:, :cols] * f64("ws")
    if kind == "linear_grad":
        dy = f64("dy")
        x = f64("xq")[:, :cols] * f64("xs")
        return torch.matmul(dy, w), torch.matmul(dy.t().contiguous(), x), torch.sum(dy, 0)
    if kind == "linear":
        return torch.addmm(f64("bias"), _exact_rows(f64("x"), cols), w.t().contiguous())
    if kind == "norm_grad":
        if case["saved"] == "exact":
            x = f64("x")
        else:
            x = (f64("xq") * torch.repeat_interleave(f64("xs"), GROUP, 1)[:, :st["xq"].shape[1]])[:, :cols]
        dy, r = f64("dy"), f64("rstd").unsqueeze(1)
        xh = (x - f64("mean").unsqueeze(1)) * r
        g = dy * f64("gamma")
        along = torch.sum(g * xh, 1, keepdim=True) / cols
        return (g - torch.sum(g, 1, keepdim=True) / cols - xh * along) * r, torch.sum(dy * xh, 0), torch.sum(dy, 0)
    x = f64("x")
    mean = torch.sum(x, 1) / cols
    var = torch.sum(x * x, 1) / cols - mean * mean
    rstd = 1 / torch.sqrt(var + EPS)
    y = f64("beta") + f64("gamma") * (x - mean.unsqueeze(1)) * rstd.unsqueeze(1)
    if kind == "norm_linear":
        return torch.addmm(f64("bias"), _exact_rows(y, cols), w.t().contiguous()), mean, rstd
    return (y, mean, rstd, _exact_rows(x, GROUP)) if case["save"] else (y, mean, rstd)
