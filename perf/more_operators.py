"""Timed cases of a training step in 8-bit floating point: ``paper_1803_03288_amd.layers``.

A worker's iteration ends with the update of the parameters whose transfers begin the next one.  These are the ops of that
step where operands are 8-bit floats with a power of two as the scale of each block of 128: parameters as they are sent, products,
their gradients, the norm of all gradients, and the update with its moments in 32 or in 8 bits.

Kinds
-----
blocks       weights or activations in 8-bit floats and back: ``quantize_f8``, ``dequantize_f8``.
linear       a product with 8-bit weights; the input is rounded to 8 bits in the call, or comes as such (``ready``).
linear_grad  gradients of the product's input, weights and bias, ``dy`` rounded to 8 bits along either way that it is summed over.
update       AdamW over many tensors, with ``clip`` by the norm of all gradients, which is formed before (``gradient_norm``, ``adamw_step``).

8-bit floats are e4m3 or e5m2, ``[rows][ld]``, ``ld`` the number of columns rounded up to 128, zeros behind the last column.  A block is 128 columns of
one row, or of 128 rows; its scale is the smallest power of two, at least 2^-126, with which its largest magnitude fits the type (448 or 57344), held
as the exponent plus 127 in a byte, ``[blocks of rows][blocks of columns rounded up to 4]``.

Moments in 8 bits are one such row for each tensor: e4m3 values of the first moment, and of the root of the second.  They are rounded at random, by hashes of the
seed, the step, the tensor's number and the element's (an EMA of 0.1 % a step never passes half a step of an 8-bit type if it is rounded to nearest).
"""

from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
F8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
TOP = {"e4m3": 9, "e5m2": 16}                   # the largest value is 0.875 * 2^TOP
LR, BETAS, EPS, DECAY, MAX_NORM, SEED = 1e-3, (0.9, 0.999), 1e-8, 0.01, 1.0, 0x1234_5678_9ABC


# ---- the cases ----------------------------------------------------------------------------------------------

def listed():
    return [
        # activations of a small batch before a classifier of 1 000 outputs, an odd number of rows, as they are kept for the backward pass
        {"name": "blocks small", "kind": "blocks", "rows": 33, "cols": 1000, "dtype": "f32", "block": 1, "f8": "e5m2"},
        # a layer's float32 weights as they are sent after an update, and as another worker's copy in bfloat16
        {"name": "blocks weights", "kind": "blocks", "rows": 16384, "cols": 4096, "dtype": "bf16", "block": 128, "f8": "e4m3"},
        # one token or sample while serving, through a layer that widens four times
        {"name": "linear one row", "kind": "linear", "rows": 1, "cols": 4096, "outs": 16384, "dtype": "bf16", "wblock": 128, "ready": False},
        # the first fully connected layer of VGG-16 for the batch of 32 images that the preset has
        {"name": "linear vgg16 fc6", "kind": "linear", "rows": 32, "cols": 25088, "outs": 4096, "dtype": "f16", "wblock": 128, "ready": False},
        # nothing a multiple of anything, a scale per output and 128 inputs, float32
        {"name": "linear odd", "kind": "linear", "rows": 333, "cols": 1001, "outs": 777, "dtype": "f32", "wblock": 1, "ready": False},
        # a large batch through a layer that widens four times
        {"name": "linear large", "kind": "linear", "rows": 8192, "cols": 4096, "outs": 16384, "dtype": "bf16", "wblock": 128, "ready": False},
        # a narrow layer on a small batch in float32, gradients with the wider range of e5m2
        {"name": "linear_grad small", "kind": "linear_grad", "rows": 101, "cols": 777, "outs": 1001, "dtype": "f32", "wblock": 128, "f8": "e5m2"},
        # VGG-16's first fully connected layer, training with 32 images
        {"name": "linear_grad vgg16 fc6", "kind": "linear_grad", "rows": 32, "cols": 25088, "outs": 4096, "dtype": "f16", "wblock": 128, "f8": "e4m3"},
        # a large batch through a layer that widens four times
        {"name": "linear_grad large", "kind": "linear_grad", "rows": 8192, "cols": 4096, "outs": 16384, "dtype": "bf16", "wblock": 128, "f8": "e4m3"},
        # the parameters of a small classifier, all states in float32
        {"name": "update small", "kind": "update", "tensors": 6, "numel": 10007, "dtype": "f32", "grad": "f32", "bits": 32, "copies": "", "clip": False},
        # all 161 tensors of the ResNet-50 preset, states in float32
        {"name": "update resnet50", "kind": "update", "tensors": 161, "numel": 0, "dtype": "f32", "grad": "f32", "bits": 32, "copies": "", "clip": True},
        # the layers of a large model on one worker: float32 parameters with copies in bfloat16, moments in 8 bits
        {"name": "update large 8 bits", "kind": "update", "tensors": 49, "numel": 1 << 26, "dtype": "f32", "grad": "bf16", "bits": 8, "copies": "bf16", "clip": True},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["blocks", "linear", "linear", "linear_grad", "linear_grad", "update"])
    case = {"kind": kind, "dtype": rng.choice(["f32", "f16", "bf16"])}
    if kind == "blocks":
        cols = _log(rng, 64, 16384)
        if rng.random() < 0.5:
            cols = -(-cols // 64) * 64
        case.update(rows=_log(rng, 1, max(1, min(16384, (1 << 26) // cols))), cols=cols, block=rng.choice([1, 128]), f8=rng.choice(["e4m3", "e5m2"]))
        return case
    if kind == "update":
        bits = rng.choice([8, 32])
        case.update(tensors=_log(rng, 1, 200), numel=_log(rng, 1000, 1 << 26), grad=rng.choice(["f32", "f16", "bf16"]), bits=bits,
                    copies=rng.choice(["", "f16", "bf16"]) if case["dtype"] == "f32" else "", clip=rng.random() < 0.5)
        return case
    cols, outs = _log(rng, 64, 25088), _log(rng, 64, 16384)
    if rng.random() < 0.5:
        cols, outs = -(-cols // 64) * 64, -(-outs // 64) * 64
    case.update(rows=_log(rng, 1, max(1, min(8192, 8192 * 4096 * 16384 // (cols * outs)))), cols=cols, outs=outs, wblock=rng.choice([1, 128, 128]))
    if kind == "linear":
        case["ready"] = rng.random() < 0.3
    else:
        case["f8"] = rng.choice(["e4m3", "e5m2"])
    return case


def _numels(case):
    """The tensors of an update by their number of elements."""
    if case["numel"]:
        rng = random.Random(case["tensors"] * 1000003 + case["numel"])
        share = [math.exp(rng.gauss(0.0, 1.5)) for _ in range(case["tensors"])]
        return [max(1, int(case["numel"] * s / sum(share))) for s in share]
    sizes, cin = [49 * 3 * 64], 64                          # ResNet-50: 16 blocks of three convolutions, 4 projections, scale and offset of every normalisation
    for blocks, mid, out in ((3, 64, 256), (4, 128, 512), (6, 256, 1024), (3, 512, 2048)):
        for k in range(blocks):
            sizes += [cin, cin, cin * mid, mid, mid, 9 * mid * mid, mid, mid, mid * out] + ([cin * out, out, out] if k == 0 else [])
            cin = out
    return sizes + [2048, 2048, 2048 * 1000, 1000]


def _starts(numels):
    """Where the tensors lie in one buffer: on multiples of 512 elements, so that the scales of moments in 8 bits lie on multiples of 4."""
    at, starts = 0, []
    for n in numels:
        starts.append(at)
        at += -(-n // 512) * 512
    return starts, at


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


def _parts(q, exponents, cols, block):
    """8-bit floats as a program keeps them: ``(q, scale, cols, block)``."""
    rows, n = q.shape[0], exponents.shape[1]
    out = torch.zeros(rows, -(-cols // 128) * 128, dtype=q.dtype, device=q.device)
    out.view(torch.uint8)[:, :cols] = q.view(torch.uint8)[:, :cols]
    scale = torch.zeros(exponents.shape[0], -(-n // 4) * 4, dtype=torch.uint8, device=q.device)
    scale[:, :n] = exponents + 127
    return out, scale.view(torch.float8_e8m0fnu), cols, block


def _update_state(case, g, state):
    numels = _numels(case)
    starts, total = _starts(numels)
    held = torch.zeros(total, dtype=torch.bool, device="cuda")
    for at, n in zip(starts, numels):
        held[at:at + n] = True
    size = torch.zeros(total, device="cuda")                # every tensor's gradients have a size of their own
    for at, n in zip(starts, numels):
        size[at:at + n] = 1e-4 * 4.0 ** (hash((n, at)) % 5)
    loss_scale = 1024.0 if case["grad"] == "f16" else 1.0
    normal = lambda: torch.randn(total, generator=g, device="cuda") * held  # noqa: E731
    grad, m = normal() * size, normal() * size * 0.3
    v = (size * held * torch.exp(0.5 * normal())).square()
    state.update(numels=numels, starts=starts, total=total, step=100, grad_scale=1.0 / loss_scale,
                 p=(normal() * 0.02).to(state["dtype"]), g=(grad * loss_scale).to(DTYPES[case["grad"]]),
                 copy=torch.zeros(total, dtype=DTYPES[case["copies"]], device="cuda") if case["copies"] else None)
    if case["bits"] == 8:
        for name, x in (("m", m), ("v", v.sqrt())):
            q, e = _blocks(x[None], 1, "e4m3")
            state[name], state[name + "_scale"] = q[0], (e[0] + 127).to(torch.uint8).view(torch.float8_e8m0fnu)
    else:
        state["m"], state["v"] = m, v
    of = lambda t: [t[at:at + n] for at, n in zip(starts, numels)]  # noqa: E731
    state.update(params=of(state["p"]), grads=of(state["g"]), copies=None if state["copy"] is None else of(state["copy"]))
    if case["bits"] == 8:
        row = lambda name, at, n: (state[name][at:at + -(-n // 128) * 128][None], state[name + "_scale"][at // 128:at // 128 + -(-n // 512) * 4][None], n, 1)  # noqa: E731
        state["moments"] = [(row("m", at, n), row("v", at, n)) for at, n in zip(starts, numels)]
    else:
        state["moments"] = list(zip(of(state["m"]), of(state["v"])))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    state = dict(case, dtype=DTYPES[case["dtype"]])
    kind = case["kind"]
    if kind == "update":
        _update_state(case, g, state)
        return state
    dtype, rows, cols = state["dtype"], case["rows"], case["cols"]
    if kind == "blocks" and case["block"] == 128:
        state["x"] = (torch.randn(rows, cols, generator=g, device="cuda") / math.sqrt(cols)).to(dtype)
    elif kind == "linear_grad":
        state["x8"] = _parts(*_blocks(_activations(g, rows, cols, torch.float32), 1, "e4m3"), cols, 1)
        state["dy"] = _gradients(g, rows, case["outs"], dtype)
    else:
        state["x"] = _activations(g, rows, cols, dtype)
    if kind == "linear" and case["ready"]:
        state["x8"] = _parts(*_blocks(state.pop("x"), 1, "e4m3"), cols, 1)
    if kind != "blocks":
        w = torch.randn(case["outs"], cols, generator=g, device="cuda") / math.sqrt(cols)
        state["w8"] = _parts(*_blocks(w, case["wblock"], "e4m3"), cols, case["wblock"])
        state["bias"] = 0.1 * torch.randn(case["outs"], generator=g, device="cuda")
    return state


# ---- the operators in their plain form ----------------------------------------------------------------------

def _power(e):
    """2^e in float32, e from -126 to 127."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _in_blocks(x, block):
    """[blocks of rows][rows of a block][blocks of columns][128], zeros behind the ends."""
    rows, cols = x.shape
    up, along = -(-rows // block) * block - rows, -(-cols // 128) * 128 - cols
    if up or along:
        x = torch.nn.functional.pad(x, (0, along, 0, up))
    return x.reshape(-1, block, (cols + along) // 128, 128)


def _blocks(x, block, f8):
    """8-bit floats ``[rows][columns rounded up to 128]`` and the exponents of their scales."""
    rows = x.shape[0]
    x = _in_blocks(x.float(), block)
    part, e = torch.frexp(x.abs().amax((1, 3)))             # a fraction from 0.5 to 1 times 2^e
    e = torch.where(part == 0, -126, (e - TOP[f8] + (part > 0.875)).clamp(min=-126))
    q = (x * _power(-e)[:, None, :, None]).to(F8[f8])
    return q.reshape(-1, q.shape[2] * 128)[:rows], e


def _values(q, e, cols, block):
    rows = q.shape[0]
    x = _in_blocks(q.float(), block) * _power(e)[:, None, :, None]
    return x.reshape(-1, x.shape[2] * 128)[:rows, :cols]


def _values8(parts):
    q, scale, cols, block = parts
    return _values(q[:, :-(-cols // 128) * 128], scale.view(torch.uint8)[:, :-(-cols // 128)].to(torch.int32) - 127, cols, block)


def _rounded(x, f8, block=1):
    """The values that 8-bit floats keep of x."""
    return _values(*_blocks(x, block, f8), x.shape[1], block)


def _mixed(x):
    """A hash of 32-bit numbers (held in int64): shifts and products with odd numbers."""
    x = ((x ^ (x >> 16)) * 0x9E3779B9) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0x6A09E667) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _random_bits(st, step):
    """32 bits for each element of the buffer."""
    device = st["p"].device
    number = lambda v: torch.tensor(v & 0xFFFFFFFF, dtype=torch.int64, device=device)  # noqa: E731
    key = _mixed(number(_key(SEED, step)) + torch.arange(len(st["numels"]), device=device) & 0xFFFFFFFF)
    starts = torch.tensor(st["starts"], device=device)
    at = torch.arange(st["total"], device=device)
    tensor = torch.searchsorted(starts, at, right=True) - 1
    return _mixed(key[tensor] + (at - starts[tensor]) & 0xFFFFFFFF)


def _key(seed, step):
    mask = 0xFFFFFFFF

    def mixed(x):
        x = (x ^ x >> 16) * 0x9E3779B9 & mask
        x = (x ^ x >> 15) * 0x6A09E667 & mask
        return x ^ x >> 16

    return mixed(mixed(mixed(seed & mask) + (seed >> 32 & mask) & mask) + (step & mask) & mask)


def _rounded_at_random(x, bits, exponents):
    """e4m3 values of x in blocks of 128, up or down by 16 random bits."""
    part, e = torch.frexp(x.reshape(-1, 128).abs().amax(1))
    e = torch.where(part == 0, -126, (e - 9 + (part > 0.875)).clamp(min=-126))
    y = x.reshape(-1, 128) * _power(-e)[:, None]
    _, own_e = torch.frexp(y)
    own_e = torch.where(y == 0, -6, (own_e - 1).clamp(min=-6)) - 3          # 2^own_e: the distance of e4m3 values there
    k = torch.floor(y.abs() * _power(-own_e) + bits.reshape(-1, 128).float() * 2.0 ** -16)
    q = torch.copysign(k * _power(own_e), y).to(torch.float8_e4m3fn)
    exponents.view(torch.uint8).copy_((e + 127).to(torch.uint8))
    return q.reshape(-1)


def _update_plain(st):
    st["step"] = step = st["step"] + 1
    b1, b2 = BETAS
    f32 = lambda v: torch.tensor(v, dtype=torch.float32, device="cuda")  # noqa: E731
    scale, out = f32(st["grad_scale"]), {}
    if st["clip"]:
        norm = (st["g"].double().square().sum().sqrt() * st["grad_scale"]).float()
        scale = scale * torch.clamp(MAX_NORM / norm, max=1.0)
        out["norm"] = norm
    g = st["g"].float() * scale
    p = st["p"].float()
    if st["bits"] == 8:
        wide = lambda name: (st[name].float().reshape(-1, 128) * _power(st[name + "_scale"].view(torch.uint8).to(torch.int32) - 127)[:, None]).reshape(-1)  # noqa: E731
        m, r = wide("m"), wide("v")
        v = r * r
    else:
        m, v = st["m"], st["v"]
    m = m * f32(b1) + g * f32(1 - b1)
    v = v * f32(b2) + (g * g) * f32(1 - b2)
    r = torch.sqrt(v)
    p = p * (1 - LR * DECAY) - (LR / (1 - b1 ** step)) * m / (r / math.sqrt(1 - b2 ** step) + EPS)
    out["p"] = st["p"].copy_(p)
    if st["copy"] is not None:
        out["copy"] = st["copy"].copy_(p)
    if st["bits"] == 8:
        bits = _random_bits(st, step)
        st["m"].copy_(_rounded_at_random(m, bits & 0xFFFF, st["m_scale"]))
        st["v"].copy_(_rounded_at_random(r, bits >> 16, st["v_scale"]))
        out.update(m=wide("m").to(torch.bfloat16), v=wide("v").to(torch.bfloat16))
    else:
        out.update(m=st["m"].copy_(m), v=st["v"].copy_(v))
    return out


def _run_plain(st):
    kind, dtype = st["kind"], st["dtype"]
    if kind == "update":
        return _update_plain(st)
    if kind == "blocks":
        return _rounded(st["x"], st["f8"], st["block"]).to(dtype)
    w = _values8(st["w8"])
    if kind == "linear":
        x = _values8(st["x8"]) if st["ready"] else _rounded(st["x"], "e4m3")
        return (x @ w.t() + st["bias"]).to(dtype)
    dy, x = st["dy"].float(), _values8(st["x8"])
    # what is summed over the rows is rounded in blocks of 128 rows
    dy_rows, dy_cols, x_cols = _rounded(dy, st["f8"]), _rounded(dy.t(), st["f8"]), _rounded(x.t(), "e4m3")
    w_cols = w if st["wblock"] == 128 else _rounded(w.t(), "e4m3").t()
    return (dy_rows @ w_cols).to(dtype), (dy_cols @ x_cols.t()).to(dtype), dy.sum(0).to(dtype)


def _run_own(st):
    from paper_1803_03288_amd import layers
    kind, dtype = st["kind"], st["dtype"]
    if kind == "update":
        st["step"] += 1
        out = {}
        if st["clip"]:
            out["norm"] = layers.gradient_norm(st["grads"], st["grad_scale"])
        layers.adamw_step(st["params"], st["grads"], st["moments"], st["step"], lr=LR, betas=BETAS, eps=EPS, weight_decay=DECAY, grad_scale=st["grad_scale"],
                          norm=out.get("norm"), max_norm=MAX_NORM if st["clip"] else None, copies=st["copies"], seed=SEED)
        out["p"] = st["p"]
        if st["copy"] is not None:
            out["copy"] = st["copy"]
        for name in ("m", "v"):
            out[name] = st[name]
            if st["bits"] == 8:
                out[name] = layers.dequantize_f8((st[name][None], st[name + "_scale"][None], st["total"], 1), torch.bfloat16)[0]
        return out
    if kind == "blocks":
        return layers.dequantize_f8(layers.quantize_f8(st["x"], st["block"], F8[st["f8"]]), dtype)
    if kind == "linear":
        return layers.linear_f8(st["x8"], st["w8"], st["bias"], dtype) if st["ready"] else layers.linear_f8(st["x"], st["w8"], st["bias"])
    return layers.linear_f8_backward(st["dy"], st["x8"], st["w8"], F8[st["f8"]])


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- what a pass cannot do without --------------------------------------------------------------------------

def work(case):
    kind, size = case["kind"], SIZE[case["dtype"]]
    if kind == "update":
        n = sum(_numels(case))
        moments = 16 if case["bits"] == 32 else 4 + 4 / 128 + 2 * (3 + 1 / 128)        # read and written; in 8 bits the values are read from them too
        return {"bytes": n * (2 * size + SIZE[case["grad"]] + moments + (2 if case["copies"] else 0)), "flops": n * (20 if case["clip"] else 18)}
    t, k = case["rows"], case["cols"]
    kept = lambda rows, block: rows * k + -(-rows // block) * -(-k // 128)  # noqa: E731
    if kind == "blocks":
        return {"bytes": 2 * t * k * size + 2 * kept(t, case["block"]), "flops": 3 * t * k}
    n = case["outs"]
    weights = kept(n, case["wblock"])
    if kind == "linear":
        return {"bytes": (kept(t, 1) if case["ready"] else t * k * size) + weights + 4 * n + t * n * size, "flops": 2 * t * k * n}
    return {"bytes": t * n * size + kept(t, 1) + weights + (t * k + n * k + n) * size, "flops": 4 * t * k * n + t * n}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------

def _two_to(e):
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_scale(amax, largest):
    """The smallest power of two, from 2^-126 on, that times `largest` is no less than amax."""
    e = torch.ceil(torch.log2(torch.clamp(amax, min=1e-300) / largest)).to(torch.int64)
    e = e - (largest * _two_to(e - 1) >= amax).long()
    e = e + (largest * _two_to(e) < amax).long()
    return _two_to(torch.clamp(e, min=-126))


def _exact_step(y, least, bits):
    """The distance between neighbours of a type with `bits` of fraction and normal numbers from 2^least on, at y."""
    _, e = torch.frexp(torch.where(y == 0, torch.ones_like(y), y))
    return _two_to(torch.where(y == 0, torch.full_like(e, least), torch.clamp(e - 1, min=least)) - bits)


def _exact_f8(x, f8, block=1):
    largest, least, bits = (448.0, -6, 3) if f8 == "e4m3" else (57344.0, -14, 2)
    back = torch.empty_like(x)
    for lo in range(0, x.shape[1], 128):
        part = x[:, lo:lo + 128]
        amax = part.abs().max(1).values
        if block > 1:
            whole = torch.zeros(-(-len(amax) // block) * block, dtype=amax.dtype, device=amax.device)
            whole[:len(amax)] = amax
            amax = whole.view(-1, block).max(1).values.repeat_interleave(block)[:len(amax)]
        s = _exact_scale(amax, largest)[:, None]
        step = _exact_step(part / s, least, bits) * s
        back[:, lo:lo + 128] = torch.round(part / step) * step
    return back


def _exact_parts(parts):
    q, scale, cols, block = parts
    e = scale.view(torch.uint8).long()[:, :-(-cols // 128)] - 127
    s = _two_to(e).repeat_interleave(128, 1).repeat_interleave(block, 0)
    return q[:, :cols].double() * s[:q.shape[0], :cols]


def _exact_moment(x, bits):
    back = x.view(-1, 128)
    s = _exact_scale(back.abs().max(1).values, 448.0)[:, None]
    step = _exact_step(back / s, -6, 3) * s
    return (torch.sign(back) * torch.floor(back.abs() / step + bits.view(-1, 128).double() / 65536) * step).view(-1)


def _exact_update(st):
    step, (b1, b2) = st["step"] + 1, BETAS
    g = st["g"].double() * st["grad_scale"]
    norm = torch.sqrt(torch.dot(g, g))
    if st["clip"]:
        g = g * min(1.0, MAX_NORM / float(norm))
    if st["bits"] == 8:
        wide = lambda name: (st[name].double().view(-1, 128) * _two_to(st[name + "_scale"].view(torch.uint8).long() - 127)[:, None]).view(-1)  # noqa: E731
        m, v = wide("m"), wide("v") ** 2
    else:
        m, v = st["m"].double(), st["v"].double()
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g ** 2
    p = st["p"].double()
    p = p - LR * DECAY * p - LR * (m / (1 - b1 ** step)) / (torch.sqrt(v / (1 - b2 ** step)) + EPS)
    out = {"p": p}
    if st["clip"]:
        out["norm"] = norm
    if st["copy"] is not None:
        out["copy"] = p
    if st["bits"] == 8:
        bits = _random_bits(st, step)
        m, v = _exact_moment(m, bits & 0xFFFF), _exact_moment(torch.sqrt(v), bits >> 16)
    out.update(m=m, v=v)
    return out


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "update":
        return _exact_update(st)
    if kind == "blocks":
        return _exact_f8(st["x"].double(), case["f8"], case["block"])
    w = _exact_parts(st["w8"])
    if kind == "linear":
        x = _exact_parts(st["x8"]) if case["ready"] else _exact_f8(st["x"].double(), "e4m3")
        return torch.addmm(st["bias"].double(), x, w.t().contiguous())
    dy = st["dy"].double()
    across = lambda x, f8: _exact_f8(x.t().contiguous(), f8)  # noqa: E731
    w_cols = w if case["wblock"] == 128 else across(w, "e4m3").t().contiguous()
    return (torch.matmul(_exact_f8(dy, case["f8"]), w_cols), torch.matmul(across(dy, case["f8"]), across(_exact_parts(st["x8"]), "e4m3").t().contiguous()),
            torch.sum(dy, 0))
