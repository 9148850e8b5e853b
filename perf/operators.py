"""Timing cases of the operators around a Dion step: the global norm of many gradients, their clipping, and the
AdamW and Lion steps of the parameters that are not matrices (norm gains, biases, embeddings).

A case names its tensors as "rows x columns * count" classes.  The tensors of a class lie in one buffer each for gradients,
parameters and moments, every tensor at a pitch of whole 256 bytes (plus ``shift`` elements), its rows at a leading
dimension of columns + ``pad``; the elements between them are zeros and stay zeros.
"""
from __future__ import annotations

import math
from functools import partial

import torch

own = False

BETAS = {"adamw": (0.9, 0.95), "lion": (0.95, 0.98)}
EPS, LR, STEP, DECAY = 1e-8, 1e-3, 1000, 0.1
MAX_NORM = 1.0
GRAD_NORM = 3.0           # the norm that the gradients are drawn with: above the threshold, so that a pass clips
SHRINK = 0.9995           # in place: each pass clips to a little less than the pass before it left

# one transformer block 4096 wide: the matrices whose gradients a training step clips together, and its two norm gains
BLOCK = [(4096, 4096, 2), (1024, 4096, 2), (14336, 4096, 2), (4096, 14336, 1), (1, 4096, 2)]


def _text(classes, layers=1):
    return " ".join("%dx%d*%d" % (r, c, k * layers) for r, c, k in classes)


RAGGED = "1001x333*2 1x1*8 1x4097*24 257x63*16 30x5*12 5x20011*3"


def listed():
    return [
        # the smallest model of the benchmark, one matrix and two vectors: latency of one call
        {"name": "norm-256x512", "op": "norm", "tensors": "256x512*1 1x512*2", "g": "f32", "kind": "2", "each": False, "pad": 0, "shift": 0},
        # odd sizes, gradients that are column slices of wider buffers; a norm of each tensor for the log
        {"name": "norm-each-ragged", "op": "norm", "tensors": RAGGED, "g": "f32", "kind": "2", "each": True, "pad": 3, "shift": 1},
        # the gradients of eight blocks of a large model, before its step
        {"name": "norm-8-blocks", "op": "norm", "tensors": _text(BLOCK, 8), "g": "bf16", "kind": "2", "each": False, "pad": 0, "shift": 0},
        # gradients accumulated over micro-batches in 32 bits, handed to the step clipped and in bf16: the smallest model
        {"name": "clip-256x512", "op": "clip", "tensors": "256x512*1 1x512*2", "g": "f32", "out": "bf16", "pad": 0, "shift": 0},
        # the same for a model whose gradients fit the L2 cache
        {"name": "clip-2048sq-4", "op": "clip", "tensors": "2048x2048*4 1x2048*9", "g": "f32", "out": "bf16", "pad": 0, "shift": 0},
        # gradients of four blocks clipped where they are
        {"name": "clip-4-blocks-in-place", "op": "clip", "tensors": _text(BLOCK, 4), "g": "bf16", "out": "in place", "pad": 0, "shift": 0},
        # the norm gains of a 32-layer model: many short vectors, latency
        {"name": "adamw-65-gains", "op": "adamw", "tensors": "1x4096*65", "g": "f32", "m": "f32", "copy": False, "scaled": True, "pad": 0, "shift": 0},
        # embedding and head in mixed precision: bf16 gradients, a bf16 copy of the weights for the next forward pass
        {"name": "adamw-embedding-head", "op": "adamw", "tensors": "32768x4096*2 1x4096*65", "g": "bf16", "m": "f32", "copy": True, "scaled": True, "pad": 0, "shift": 0},
        # odd sizes, slices of wider buffers, the first moment in bf16
        {"name": "adamw-ragged", "op": "adamw", "tensors": RAGGED, "g": "f32", "m": "bf16", "copy": False, "scaled": False, "pad": 3, "shift": 1},
        # as for AdamW: gains, embedding and head (momentum in bf16: what Lion keeps least of), odd sizes
        {"name": "lion-65-gains", "op": "lion", "tensors": "1x4096*65", "g": "bf16", "m": "f32", "copy": False, "scaled": True, "pad": 0, "shift": 0},
        {"name": "lion-embedding-head", "op": "lion", "tensors": "32768x4096*2 1x4096*65", "g": "bf16", "m": "bf16", "copy": True, "scaled": True, "pad": 0, "shift": 0},
        {"name": "lion-ragged", "op": "lion", "tensors": RAGGED, "g": "f32", "m": "f32", "copy": True, "scaled": False, "pad": 3, "shift": 1},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "clip", "adamw", "lion"])
    most = {"norm": 8e8, "clip": 4e8, "adamw": 2e8, "lion": 2e8}[op]
    ragged = rng.random() < 0.3
    total = _log_uniform(rng, 2e3, 2e7 if ragged else most)      # (narrow slices of wider buffers: up to ten times the memory)
    classes = []
    kinds = rng.randint(1, 6)
    for _ in range(kinds):
        want = max(1.0, total / kinds * rng.uniform(0.3, 1.0))
        count = min(_log_uniform(rng, 1, 64), max(1, int(want)))
        size = max(1, int(want / count))
        cols = _log_uniform(rng, 1, max(1, min(size, 65536)))
        if rng.random() < 0.6 and cols >= 64:
            cols = cols // 64 * 64
        classes.append((max(1, size // cols), cols, count))
    case = {"op": op, "tensors": _text(classes), "g": rng.choice(["f32", "bf16"]),
            "pad": rng.randint(0, 9) if ragged else 0, "shift": rng.randint(0, 7) if ragged else 0}
    if op == "norm":
        case.update(kind=rng.choice(["2", "2", "2", "inf"]), each=rng.random() < 0.5)
    elif op == "clip":
        # a short list is clipped many times in a second: in place it would be clipped away
        case["out"] = rng.choice(["f32", "bf16"] + (["in place"] * 2 if total > 3e7 else []))
    else:
        case.update(m=rng.choice(["f32", "bf16"]), copy=rng.random() < 0.5, scaled=rng.random() < 0.5)
    return case


# ---- inputs ------------------------------------------------------------------------------------------------------

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _classes(case):
    """(rows, columns, count, leading dimension, elements from one tensor of the class to the next)"""
    found = []
    for part in case["tensors"].split():
        shape, count = part.split("*")
        rows, cols = (int(x) for x in shape.split("x"))
        ld = cols + case["pad"]
        found.append((rows, cols, int(count), ld, (rows * ld + case["shift"] + 127) // 128 * 128))
    return found


def _views(flat, rows, cols, ld, shift):
    """The tensors of a class's buffer."""
    return [flat[k, shift:shift + rows * ld].view(rows, ld)[:, :cols] for k in range(flat.shape[0])]


def _buffer(cls, shift, dtype, draw_one=None):
    """A class's buffer: zeros, or tensors drawn one by one with zeros between them."""
    rows, cols, count, ld, pitch = cls
    flat = torch.zeros(count, pitch, dtype=dtype, device="cuda")
    for v in _views(flat, rows, cols, ld, shift) if draw_one is not None else ():
        v.copy_(draw_one(v.shape))
    return flat


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))

    def randn(shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)

    op, shift = case["op"], case["shift"]
    classes = _classes(case)
    total = sum(r * c * k for r, c, k, _, _ in classes)
    std = GRAD_NORM / math.sqrt(total)
    state = {"op": op, "case": dict(case), "max_norm": MAX_NORM, "tensors": []}
    for n, (rows, cols, count, ld, pitch) in enumerate(classes):
        # layers differ in the size of their gradients; about half of an embedding's rows have seen no token of the batch
        level = std * (torch.rand((), generator=gen, device="cuda") + 0.5)
        embedding = op in BETAS and rows >= 8192
        if embedding:
            level = level * (torch.rand((rows, 1), generator=gen, device="cuda") < 0.5)
        buffer = partial(_buffer, (rows, cols, count, ld, pitch), shift)
        G = buffer(DTYPES[case["g"]], lambda shape, level=level: randn(shape) * level)
        one = {"G": G, "decay": DECAY if rows > 1 else 0.0, "lr_scale": 1.0 / math.sqrt(cols) if n == 0 and embedding else 1.0}
        if op == "clip":
            one["out"] = G if case["out"] == "in place" else buffer(DTYPES[case["out"]])
        elif op in BETAS:
            one["X"] = buffer(torch.float32, lambda shape: randn(shape) * 0.02)
            one["M"] = buffer(DTYPES[case["m"]], lambda shape: randn(shape) * (0.3 * std))
            if op == "adamw":
                one["V"] = buffer(torch.float32, lambda shape: (randn(shape).square() + 0.1) * std ** 2)
            if case["copy"]:
                one["X16"] = buffer(torch.bfloat16)
        state["tensors"].append(one)
    count = sum(c[2] for c in classes)
    state["norm"], state["coef"] = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    if case.get("each"):
        state["each"] = torch.zeros(count, device="cuda")
    if case.get("scaled"):
        state["scale"] = torch.rand(1, generator=gen, device="cuda") * 0.5 + 0.3
    if own:
        from paper_2504_05295_b200 import binding
        state["opt"], state["list"] = _context(), _descriptors(binding, state, classes)
    return state


_CONTEXT = []


def _context():
    """One library context, kept like a training program keeps its optimizer."""
    if not _CONTEXT:
        from paper_2504_05295_b200 import binding
        _CONTEXT.append(binding.Dion())
    return _CONTEXT[0]


def _descriptors(binding, state, classes):
    case, op = state["case"], state["op"]
    grads, outs, params = [], [], []
    for (rows, cols, _, ld, _), one in zip(classes, state["tensors"]):
        views = {k: _views(v, rows, cols, ld, case["shift"]) for k, v in one.items() if isinstance(v, torch.Tensor)}
        grads += views["G"]
        outs += views.get("out", [])
        if op in BETAS:
            for k, G in enumerate(views["G"]):
                params.append(binding.param_desc(views["X"][k], G, views["M"][k], views["V"][k] if op == "adamw" else None,
                                                 X16=views["X16"][k] if case["copy"] else None, lr_scale=one["lr_scale"],
                                                 weight_decay=one["decay"]))
    if op in BETAS:
        return binding.param_list(params)
    return binding.grad_list(grads, outs if op == "clip" and case["out"] != "in place" else None)


# ---- one pass ----------------------------------------------------------------------------------------------------

def run(state):
    op, case, tensors = state["op"], state["case"], state["tensors"]
    if op == "norm":
        return _norm(state, case)
    if op == "clip":
        max_norm = state["max_norm"]
        if case["out"] == "in place":
            state["max_norm"] *= SHRINK
        return _clip(state, max_norm)
    beta1, beta2 = BETAS[op]
    if own:
        if op == "adamw":
            state["opt"].adamw_step(state["list"], LR, step=STEP, beta1=beta1, beta2=beta2, eps=EPS, grad_scale=state.get("scale"))
        else:
            state["opt"].lion_step(state["list"], LR, beta1=beta1, beta2=beta2, grad_scale=state.get("scale"))
    else:
        for one in tensors:
            (_adamw if op == "adamw" else _lion)(one, state.get("scale"), beta1, beta2)
    return [{k: one[k] for k in ("X", "M", "V", "X16") if k in one} for one in tensors]


def _norm(state, case):
    if own:
        state["opt"].grad_norm(state["list"], norm_type=case["kind"], norm_out=state["norm"], each_out=state.get("each"))
        return {k: state[k] for k in ("norm", "each") if k in state}
    if case["kind"] == "inf":
        parts = torch.cat([one["G"].float().abs().amax(dim=1) for one in state["tensors"]])
        found = {"norm": parts.amax().reshape(1), "each": parts}
    else:
        parts = torch.cat([one["G"].float().square().sum(dim=1) for one in state["tensors"]])
        found = {"norm": parts.sum().sqrt().reshape(1), "each": parts.sqrt()}
    return {k: v for k, v in found.items() if k in state}


def _clip(state, max_norm):
    tensors = state["tensors"]
    if own:
        state["opt"].clip_grads(state["list"], max_norm, norm_out=state["norm"], coef_out=state["coef"])
        return [one["out"] for one in tensors], state["norm"], state["coef"]
    norm = torch.stack([one["G"].float().square().sum() for one in tensors]).sum().sqrt().reshape(1)
    coef = (max_norm / norm).clamp(max=1.0)
    for one in tensors:
        one["out"].copy_(one["G"].float() * coef)
    return [one["out"] for one in tensors], norm, coef


def _adamw(one, scale, beta1, beta2):
    g = one["G"].float() if scale is None else one["G"].float() * scale
    lr = LR * one["lr_scale"]
    m = one["M"].float() * beta1 + g * (1 - beta1)
    v = one["V"] * beta2 + g.square() * (1 - beta2)
    step = (m / (1 - beta1 ** STEP)) / ((v / (1 - beta2 ** STEP)).sqrt() + EPS)
    x = one["X"] * (1 - lr * one["decay"]) - lr * step
    _store(one, x, m, v)


def _lion(one, scale, beta1, beta2):
    g = one["G"].float() if scale is None else one["G"].float() * scale
    lr = LR * one["lr_scale"]
    # the sign of a sum that may cancel: taken in 64 bits
    wide = one["G"].double() if scale is None else one["G"].double() * scale.double()
    sign = (one["M"].double() * beta1 + wide * (1 - beta1)).sign().float()
    x = one["X"] * (1 - lr * one["decay"]) - lr * sign
    _store(one, x, one["M"].float() * beta2 + g * (1 - beta2))


def _store(one, x, m, v=None):
    one["X"].copy_(x)
    one["M"].copy_(m)
    if v is not None:
        one["V"].copy_(v)
    if "X16" in one:
        one["X16"].copy_(x)


# ---- the definition in 64 bits -----------------------------------------------------------------------------------

def exact(case, seed):
    """The operators' definitions tensor by tensor, in float64."""
    state = prepare(case, seed)
    op, classes = case["op"], _classes(case)
    scale = float(state["scale"].double()) if "scale" in state else 1.0
    if op in ("norm", "clip"):
        each = []
        for (rows, cols, _, ld, _), one in zip(classes, state["tensors"]):
            for G in _views(one["G"], rows, cols, ld, case["shift"]):
                g = G.double()
                each.append(g.abs().max() if case.get("kind") == "inf" else torch.linalg.vector_norm(g))
        each = torch.stack(each)
        norm = (each.max() if case.get("kind") == "inf" else torch.linalg.vector_norm(each)).reshape(1)
        if op == "norm":
            return {"norm": norm, "each": each} if case["each"] else {"norm": norm}
        coef = torch.clamp(MAX_NORM / norm, max=1.0)
        return [one["G"].double() * coef for one in state["tensors"]], norm, coef
    beta1, beta2 = BETAS[op]
    found = []
    for one in state["tensors"]:
        g, x, m = one["G"].double() * scale, one["X"].double(), one["M"].double()
        lr = LR * one["lr_scale"]
        x = x - lr * one["decay"] * x
        new = {}
        if op == "adamw":
            m = m + (1 - beta1) * (g - m)
            v = one["V"].double()
            v = v + (1 - beta2) * (g * g - v)
            x = x - lr * (m / (1 - beta1 ** STEP)) / (torch.sqrt(v / (1 - beta2 ** STEP)) + EPS)
            new["V"] = v
        else:
            x = x - lr * torch.sign(beta1 * m + (1 - beta1) * g)
            m = m + (1 - beta2) * (g - m)
        new["X"], new["M"] = x, m
        if "X16" in one:
            new["X16"] = x
        found.append(new)
    return found


# ---- what a pass cannot do without -------------------------------------------------------------------------------

def work(case):
    """Every gradient read once; of a clipped one the result written; of a parameter the weight and its moments read and written."""
    size = {"f32": 4, "bf16": 2}
    elements = sum(r * c * k for r, c, k, _, _ in _classes(case))
    g = size[case["g"]]
    if case["op"] == "norm":
        return {"bytes": float(elements * g), "flops": 2.0 * elements}
    if case["op"] == "clip":
        return {"bytes": float(elements * (g + (g if case["out"] == "in place" else size[case["out"]]))), "flops": 3.0 * elements}
    state = 8 + 2 * size[case["m"]] + (8 if case["op"] == "adamw" else 0) + (2 if case["copy"] else 0)
    return {"bytes": float(elements * (g + state)), "flops": (16.0 if case["op"] == "adamw" else 9.0) * elements}
