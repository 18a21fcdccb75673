"""The operators of a residual block in a trainable head over leaf ids, as a list of cases: between the layer norm of a
row's summed vectors and its classes, a block widens the row by a gated feed-forward and adds a product of that to the row;
its training step clips the gradients of all tensors together.

    "linear"     z = x weight^T + bias, y = residual + scale * act(z), and the gradients of x, weight and bias
    "gated"      z = x weight^T + bias, of which the first half of the columns are gates and the others values; y = act(gates) * values
    "clip"       the 2-norm of all gradients' values, and the gradients times min(1, limit / norm)

Fields of a case: op; way ("forward"; "keep": forward in training, which returns z too; "backward": from z and the gradient
of y); dtype ("f32", "bf16": of activations, weights and their gradients; bias and its gradient are float32); rows, dim, outs (columns of
y); act ("none", "relu", "gelu": x times the normal distribution's integral, "silu"); bias; for "linear" residual and scale.
For "clip": way ("new": results of their own; "in_place": norm below the limit, so that the gradients stay), the
tensors' shapes and types, separated by commas, and limit, in expected norms.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
MAX_FLOPS = 8 * 16_384 * 1024 * 4096   # of the largest listed case
MAX_VALUES = 16_384 * 8192             # of one array of activations
MAX_CLIP = 66_000_000


def _linear(name, way, dtype, rows, dim, outs, act="none", bias=True, residual=False, scale=1.0):
    return dict(name=name, op="linear", way=way, dtype=dtype, rows=rows, dim=dim, outs=outs, act=act, bias=bias, residual=residual, scale=scale)


def _gated(name, way, dtype, rows, dim, outs, act="silu", bias=True):
    return dict(name=name, op="gated", way=way, dtype=dtype, rows=rows, dim=dim, outs=outs, act=act, bias=bias)


def _clip(name, way, shapes, limit):
    return dict(name=name, op="clip", way=way, shapes=shapes, limit=limit)


def listed():
    return [
        # one record online through a small block: nothing but latency
        _gated("gated_record", "forward", "f32", 1, 64, 256),
        # a handful of records online through a wide block: the weights' bytes
        _gated("gated_few", "forward", "bf16", 5, 2048, 8192, act="gelu", bias=False),
        # the gradients of a training batch in 32 bits, odd everywhere
        _gated("gated_grad_f32", "backward", "f32", 4_099, 90, 331, act="gelu"),
        # a wide block's training batch, forward
        _gated("gated_keep", "keep", "bf16", 16_384, 1024, 4096, bias=False),
        # and its gradients: the largest case
        _gated("gated_grad", "backward", "bf16", 16_384, 1024, 4096, bias=False),
        # one record online, added to its row
        _linear("linear_record", "forward", "f32", 1, 256, 64, residual=True),
        # batch encoding of YearPrediction's inference share
        _linear("linear_batch", "forward", "bf16", 103_069, 512, 128, act="gelu"),
        # a training batch in 32 bits, odd everywhere
        _linear("linear_keep", "keep", "f32", 20_011, 331, 90, act="silu", residual=True),
        # the gradients of a wide block's second product
        _linear("linear_grad", "backward", "bf16", 16_384, 4096, 1024, scale=0.5),
        # the gradients of a small head: ten trees of depth 4, a block, ten classes
        _clip("clip_small", "new", "310x64:f32,64:f32,64:f32,512x64:f32,512:f32,64x256:f32,64:f32,10x64:f32,10:f32", 0.5),
        # an ordinary step of a head over 500 trees of depth 8, gradients below the limit
        _clip("clip_idle", "in_place", "255500x64:f32,64:f32,64:f32,101x64:f32,101:f32", 4.0),
        # a wide head whose large gradients are in 16 bits, above the limit
        _clip("clip_wide", "new", "250051x128:bf16,128:f32,128:f32,512x128:bf16,512:f32,65536x512:bf16,65536:f32", 0.25),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    """One more case of the same ranges."""
    op = rng.choice(["linear", "linear", "gated", "gated", "clip"])
    if op == "clip":
        shapes, left = [], _log_int(rng, 1_000, MAX_CLIP)
        for _ in range(rng.randint(1, 5)):
            dim = rng.choice([16, 31, 50, 64, 96, 128, 256])
            rows = max(1, min(_log_int(rng, 1, 260_000), left // dim))
            left = max(0, left - rows * dim)
            shapes += ["%dx%d:%s" % (rows, dim, rng.choice(["f32", "bf16"])), "%d:f32" % dim]
        way = rng.choice(["new", "in_place"])
        case = _clip("", way, ",".join(shapes), rng.choice([2.0, 8.0]) if way == "in_place" else rng.choice([0.1, 0.5, 4.0]))
    else:
        dtype, way = rng.choice(["f32", "bf16"]), rng.choice(["forward", "forward", "keep", "backward"])
        rows = _log_int(rng, 1, 64) if way == "forward" and rng.random() < 0.5 else _log_int(rng, 1, 110_000)
        # widths of whole vectors, and any
        dim, outs = _log_int(rng, 8, 4096), _log_int(rng, 8, 8192)
        if rng.random() < 0.6:
            dim, outs = (max(8, n // 16 * 16) for n in (dim, outs))
        each = {"forward": 2, "keep": 2, "backward": 4}[way] * dim * outs * (2 if op == "gated" else 1)
        widest = max(dim, outs * (2 if op == "gated" else 1))
        rows = max(1, min(rows, MAX_FLOPS // (8 if dtype == "f32" else 1) // each, MAX_VALUES // widest))
        act, bias = rng.choice(["relu", "gelu", "silu"]), rng.random() < 0.6
        if op == "gated":
            case = _gated("", way, dtype, rows, dim, outs, act, bias)
        else:
            case = _linear("", way, dtype, rows, dim, outs, rng.choice(["none", "none", act]), bias, rng.random() < 0.5, rng.choice([1.0, 0.5]))
    return {k: v for k, v in case.items() if k != "name"}


# Inputs.

def _tensors(case):
    """(shape, type) of each gradient."""
    return [(tuple(int(n) for n in s.split("x")), DTYPE[t]) for s, t in (part.split(":") for part in case["shapes"].split(","))]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, generator=g, device="cuda") * scale

    state = {"case": case}
    if case["op"] == "clip":
        grads = [normal(*s, scale=1e-3) for s, _ in _tensors(case)]
        for t in grads:  # leaves that no row of the batch reaches
            if t.dim() == 2 and t.shape[0] > 100:
                t[torch.rand(t.shape[0], generator=g, device="cuda") < 0.3] = 0
        state["grads"] = [t.to(d) for t, (_, d) in zip(grads, _tensors(case))]
        state["limit"] = case["limit"] * 1e-3 * math.sqrt(sum(t.numel() for t in grads))
        return state
    dtype, rows, dim, outs = DTYPE[case["dtype"]], case["rows"], case["dim"], case["outs"]
    columns = outs * (2 if case["op"] == "gated" else 1)
    state["x"] = normal(rows, dim).to(dtype)  # a layer norm's rows
    state["weight"] = normal(columns, dim, scale=dim ** -0.5).to(dtype)
    state["bias"] = normal(columns, scale=0.1) if case["bias"] else None
    if case["way"] == "backward":
        state["grad"] = normal(rows, outs, scale=1e-3).to(dtype)
        if case["op"] == "gated" or case["act"] != "none":  # what the forward pass kept
            z = state["x"].float() @ state["weight"].float().T
            state["z"] = (z if state["bias"] is None else z.add_(state["bias"])).to(dtype)
    elif case.get("residual"):
        state["residual"] = normal(rows, outs).to(dtype)
    return state


# The plain forms.

def _act(name, x):
    if name == "silu":
        return x / (1 + torch.exp(-x))
    if name == "gelu":
        return 0.5 * x * (1 + torch.erf(x * math.sqrt(0.5)))
    return x.clamp(min=0) if name == "relu" else x


def _slope(name, x):
    if name == "silu":
        s = 1 / (1 + torch.exp(-x))
        return s * (1 + x * (1 - s))
    if name == "gelu":
        return 0.5 * (1 + torch.erf(x * math.sqrt(0.5))) + x * torch.exp(-0.5 * x * x) / math.sqrt(2 * math.pi)
    return (x > 0).float()


def _plain_product(state):
    z = state["x"].float() @ state["weight"].float().T
    return z if state["bias"] is None else z.add_(state["bias"])


def _plain_grads(state, dz):
    dtype = state["x"].dtype
    out = [(dz @ state["weight"].float()).to(dtype), (dz.T @ state["x"].float()).to(dtype)]
    return out + [dz.sum(0)] if state["bias"] is not None else out


def _plain_linear(state):
    case, dtype = state["case"], state["x"].dtype
    if case["way"] == "backward":
        dz = case["scale"] * state["grad"].float()
        return _plain_grads(state, dz if case["act"] == "none" else dz * _slope(case["act"], state["z"].float()))
    z = _plain_product(state)
    y = case["scale"] * _act(case["act"], z)
    if case["residual"]:
        y = y + state["residual"].float()
    return [y.to(dtype), z.to(dtype)] if case["way"] == "keep" else y.to(dtype)


def _plain_gated(state):
    case, dtype = state["case"], state["x"].dtype
    if case["way"] == "backward":
        grad = state["grad"].float()
        gate, value = state["z"].float().chunk(2, 1)
        return _plain_grads(state, torch.cat([grad * value * _slope(case["act"], gate), grad * _act(case["act"], gate)], 1))
    z = _plain_product(state)
    gate, value = z.chunk(2, 1)
    y = (_act(case["act"], gate) * value).to(dtype)
    return [y, z.to(dtype)] if case["way"] == "keep" else y


def _plain_clip(state):
    norm = torch.stack([g.float().square().sum() for g in state["grads"]]).sum().sqrt()
    factor = (state["limit"] / norm).clamp(max=1)
    new = [(g.float() * factor).to(g.dtype) for g in state["grads"]]
    if state["case"]["way"] == "in_place":
        new = [g.copy_(n) for g, n in zip(state["grads"], new)]
    return norm, new


# The framework's operators.

def _own_linear(pk, state):
    case = state["case"]
    act = None if case["act"] == "none" else case["act"]
    if case["way"] == "backward":
        grads = pk.head_linear_grad(state["grad"], state["x"], state["weight"], state.get("z"), act, case["scale"], bias=case["bias"])
        return [t for t in grads if t is not None]
    return pk.head_linear(state["x"], state["weight"], state["bias"], act, state.get("residual"), case["scale"], keep=case["way"] == "keep")


def _own_gated(pk, state):
    case = state["case"]
    if case["way"] == "backward":
        grads = pk.head_gated_grad(state["grad"], state["x"], state["weight"], state["z"], case["act"], bias=case["bias"])
        return [t for t in grads if t is not None]
    return pk.head_gated(state["x"], state["weight"], state["bias"], case["act"], keep=case["way"] == "keep")


def _own_clip(pk, state):
    return pk.head_clip(state["grads"], state["limit"], in_place=state["case"]["way"] == "in_place")


def run(state):
    op = state["case"]["op"]
    if own:
        import paper_2301_13441_amd as pk
        return {"linear": _own_linear, "gated": _own_gated, "clip": _own_clip}[op](pk, state)
    return {"linear": _plain_linear, "gated": _plain_gated, "clip": _plain_clip}[op](state)


def work(case):
    if case["op"] == "clip":
        values = [math.prod(s) * d.itemsize for s, d in _tensors(case)]
        # the gradients are read for the norm; what is clipped is written too
        return {"bytes": sum(values) * (1 if case["way"] == "in_place" else 2) + 4, "flops": 3 * sum(math.prod(s) for s, _ in _tensors(case))}
    e = DTYPE[case["dtype"]].itemsize
    rows, dim, outs = case["rows"], case["dim"], case["outs"]
    columns = outs * (2 if case["op"] == "gated" else 1)
    product, operands, bias = 2 * rows * dim * columns, e * (rows * dim + columns * dim), 4 * columns * case["bias"]
    if case["way"] == "backward":
        kept = columns if case["op"] == "gated" or case["act"] != "none" else 0
        return {"bytes": 2 * operands + e * rows * (outs + kept) + bias, "flops": 2 * product}
    arrays = outs + (outs if case.get("residual") else 0) + (columns if case["way"] == "keep" else 0)
    return {"bytes": operands + e * rows * arrays + bias, "flops": product}


# The definitions, in 64 bits.

def _act64(name, x):
    if name == "silu":
        return x * torch.sigmoid(x)
    if name == "gelu":
        return x * torch.special.erfc(-x / math.sqrt(2)) / 2
    return torch.relu(x) if name == "relu" else x * 1


def exact(case, seed):
    state, d = prepare(case, seed), torch.float64
    if case["op"] == "clip":
        norm = torch.linalg.vector_norm(torch.cat([g.reshape(-1) for g in state["grads"]], 0).to(d))
        return norm, [g.to(d) * min(1.0, state["limit"] / float(norm)) for g in state["grads"]]
    x, weight = state["x"].to(d), state["weight"].to(d)
    gated = case["op"] == "gated"

    def end(z):
        if gated:
            return _act64(case["act"], z[:, :case["outs"]]) * z[:, case["outs"]:]
        return _act64(case["act"], z) * case["scale"]

    if case["way"] != "backward":
        z = torch.nn.functional.linear(x, weight, None if state["bias"] is None else state["bias"].to(d))
        y = end(z) + (state["residual"].to(d) if case.get("residual") else 0)
        return [y, z] if case["way"] == "keep" else y
    z = state["z"].to(d) if "z" in state else torch.zeros(case["rows"], weight.shape[0], dtype=d, device=x.device)
    z.requires_grad_()
    dz, = torch.autograd.grad(end(z), z, state["grad"].to(d))
    return [torch.mm(dz, weight), torch.mm(dz.t(), x)] + ([dz.sum(0)] if case["bias"] else [])
