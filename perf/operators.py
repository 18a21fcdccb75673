"""The operators of a trainable head over leaf ids, as a list of cases: a forest turns rows into leaf ids, a head has a
vector for every node of every tree, sums a row's vectors, normalises the sum and scores classes with a linear softmax
model.  Four operators, each in both directions:

    "embed"      sum of a row's vectors, or (one tree) a lookup: out[r] = scale * sum_t table[offset[t] + ids[r, t]]
    "norm"       layer norm
    "loss"       softmax cross entropy of a linear model over many classes, logits never kept
    "adamw"      one AdamW step over all tensors of a head, states in 32 bits or in 8

Fields of a case: op; way ("forward", "backward", "step": forward and backward); dtype ("f32", "bf16": of activations, of
the big weights and of their gradients); rows, dim; for "embed" trees, depth (full trees: 2^(depth+1) - 1 nodes each) and
missing (share of the ids that are -1, and of the rows that have no id at all); for "loss" classes, bias, ignored (share of
rows without a target); for "adamw" bits and, separated by commas, the tensors' shapes.

The 8-bit states: blocks of 128 values; a block has a scale byte s, its values are e4m3 codes times 2^(s - 134), and s - 127
is the exponent of the block's largest magnitude.  What is coded is m, and the root of v.  Rounding to a code is up where the
fraction plus a random number in [0, 1) reaches one; the random number is a hash of seed, step, tensor and index.  A root
of v above zero never gets the code of zero, for m divided by that would be without bound.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
BETA1, BETA2, EPS, DECAY, RATE = 0.9, 0.999, 1e-8, 0.01, 1e-3
BLOCK = 128
MAX_TOKENS = 13_192_832          # ids of the largest listed embedding case
MAX_VALUES = 13_192_832 * 128    # and values that it sums
MAX_NORM = 262_147 * 1024
MAX_LOSS = 16_384 * 65_536 * 512
MAX_ADAMW = 66_000_000


def _embed(name, way, dtype, rows, trees, depth, dim, missing=0.0):
    return dict(name=name, op="embed", way=way, dtype=dtype, rows=rows, trees=trees, depth=depth, dim=dim, missing=missing)


def _norm(name, way, dtype, rows, dim):
    return dict(name=name, op="norm", way=way, dtype=dtype, rows=rows, dim=dim)


def _loss(name, way, dtype, rows, dim, classes, bias=True, ignored=0.0):
    return dict(name=name, op="loss", way=way, dtype=dtype, rows=rows, dim=dim, classes=classes, bias=bias, ignored=ignored)


def _adamw(name, dtype, bits, shapes):
    return dict(name=name, op="adamw", way="step", dtype=dtype, bits=bits, shapes=shapes)


def listed():
    return [
        # one record online: the vectors of a forest of 500 trees of depth 8, nothing but latency
        _embed("embed_record", "forward", "f32", 1, 500, 8, 64),
        # batch encoding with 128 deeper trees, YearPrediction's inference share, vectors kept in 16 bits, some trees skipped
        _embed("embed_batch", "forward", "bf16", 103_069, 128, 10, 128, missing=0.1),
        # the gradient of a training batch's vectors: an odd number of rows, 500 trees
        _embed("embed_grad", "backward", "f32", 20_011, 500, 8, 64),
        # one record online
        _norm("norm_record", "forward", "f32", 1, 64),
        # YearPrediction's rows at an odd width, in training
        _norm("norm_batch", "forward", "f32", 515_345, 90),
        # the gradient of a wide head in 16 bits
        _norm("norm_grad", "backward", "bf16", 262_147, 1024),
        # ten classes, a thousand rows: the smallest training step
        _loss("loss_small", "step", "f32", 1_021, 64, 10),
        # twenty thousand classes in 32 bits, odd everywhere, a few rows without a target
        _loss("loss_f32", "step", "f32", 4_099, 128, 20_011, ignored=0.02),
        # many classes, a large batch in 16 bits: the largest training step
        _loss("loss_bf16", "step", "bf16", 16_384, 512, 65_536),
        # the update of a small head: ten trees of depth 4, ten classes
        _adamw("adamw_small", "f32", 32, "310x64,64,64,10x64,10"),
        # the update of a head over 500 trees of depth 8, a hundred classes
        _adamw("adamw_f32", "f32", 32, "255500x64,64,64,101x64,101"),
        # the update of a wide head with states in 8 bits, gradients in 16 and a copy of the weights in 16 bits
        _adamw("adamw_8bit", "bf16", 8, "250051x128,128,128,512x128,512,65536x512,65536"),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    """One more case of the same ranges."""
    op = rng.choice(["embed", "embed", "norm", "loss", "loss", "adamw"])
    dtype = rng.choice(["f32", "bf16"])
    if op == "embed":
        way = rng.choice(["forward", "backward"])
        if rng.random() < 0.3:  # plain lookups
            trees, depth, rows = 1, rng.randint(6, 16), _log_int(rng, 1, 1_000_000)
        else:
            trees, depth, rows = _log_int(rng, 8, 500), rng.randint(4, 10), _log_int(rng, 1, 110_000)
        dim = rng.choice([8, 16, 31, 50, 64, 96, 128, 200, 256])
        rows = max(1, min(rows, MAX_TOKENS // trees, MAX_VALUES // (trees * dim)))
        case = _embed("", way, dtype, rows, trees, depth, dim, rng.choice([0.0, 0.0, 0.1]))
    elif op == "norm":
        dim = _log_int(rng, 8, 2_500)
        case = _norm("", rng.choice(["forward", "backward"]), dtype, min(_log_int(rng, 1, 1_000_000), MAX_NORM // dim), dim)
    elif op == "loss":
        dim, classes = rng.choice([16, 50, 64, 90, 128, 256, 384, 512]), _log_int(rng, 4, 131_072)
        rows = min(_log_int(rng, 1, 20_000), MAX_LOSS // (4 * dim * classes) if dtype == "f32" else MAX_LOSS // (dim * classes))
        case = _loss("", rng.choice(["forward", "step", "step"]), dtype, max(1, rows), dim, classes, rng.random() < 0.7,
                     rng.choice([0.0, 0.05]))
    else:
        shapes, left = [], _log_int(rng, 1_000, MAX_ADAMW)
        for _ in range(rng.randint(1, 5)):
            dim = rng.choice([16, 31, 50, 64, 96, 128, 256])
            rows = max(1, min(_log_int(rng, 1, 260_000), left // dim))
            left = max(0, left - rows * dim)
            shapes += ["%dx%d" % (rows, dim), "%d" % dim]
        case = _adamw("", dtype, rng.choice([8, 32]), ",".join(shapes))
    return {k: v for k, v in case.items() if k != "name"}


# Inputs.

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _leaf_ids(g, rows, trees, depth, missing):
    """Leaf ids of full trees whose splits are uneven, each in its own way; -1 where a tree is skipped."""
    leaf = torch.zeros(rows, trees, dtype=torch.int32, device="cuda")
    for _ in range(depth):
        share = 0.15 + 0.7 * torch.rand(1, trees, generator=g, device="cuda")
        leaf = 2 * leaf + (torch.rand(rows, trees, generator=g, device="cuda") < share).int()
    ids = leaf + ((1 << depth) - 1)
    if missing:
        ids[torch.rand(rows, trees, generator=g, device="cuda") < missing] = -1
        ids[torch.rand(rows, generator=g, device="cuda") < missing / 4] = -1
    return ids.contiguous()


def _targets(g, rows, classes, ignored):
    """Few classes are frequent, most are rare."""
    t = (classes * torch.rand(rows, generator=g, device="cuda") ** 2.5).int().clamp_(max=classes - 1)
    if ignored:
        t[torch.rand(rows, generator=g, device="cuda") < ignored] = -1
    return t


def _shapes(case):
    return [tuple(int(n) for n in s.split("x")) for s in case["shapes"].split(",")]


def prepare(case, seed):
    g = _generator(seed)
    dtype = DTYPE[case["dtype"]]

    def normal(*shape, scale=1.0, offset=0.0):
        return torch.randn(*shape, generator=g, device="cuda") * scale + offset

    state = {"case": case}
    if case["op"] == "embed":
        nodes = (2 << case["depth"]) - 1
        state["ids"] = _leaf_ids(g, case["rows"], case["trees"], case["depth"], case["missing"])
        state["offsets"] = torch.arange(case["trees"], device="cuda", dtype=torch.int64) * nodes
        state["vectors"] = nodes * case["trees"]
        state["scale"] = 1.0 / math.sqrt(case["trees"])
        if case["way"] == "forward":
            state["table"] = normal(state["vectors"], case["dim"], scale=0.1).to(dtype)
        else:
            state["grad"] = normal(case["rows"], case["dim"], scale=1e-3).to(dtype)
    elif case["op"] == "norm":
        rows, dim = case["rows"], case["dim"]
        state["x"] = (normal(rows, dim) * (0.5 + torch.rand(rows, 1, generator=g, device="cuda")) + normal(rows, 1, scale=0.1, offset=0.5)).to(dtype)
        state["weight"], state["bias"] = normal(dim, scale=0.1, offset=1.0), normal(dim, scale=0.1)
        if case["way"] == "backward":
            x = state["x"].float()
            state["mean"] = x.mean(1)
            state["rstd"] = torch.rsqrt((x - state["mean"][:, None]).square().mean(1) + 1e-5)
            state["grad"] = normal(rows, dim, scale=1e-3).to(dtype)
    elif case["op"] == "loss":
        rows, dim, classes = case["rows"], case["dim"], case["classes"]
        state["targets"] = _targets(g, rows, classes, case["ignored"])
        weight = normal(classes, dim, scale=dim ** -0.5)
        state["hidden"] = (normal(rows, dim) + 3 * weight[state["targets"].long().clamp(min=0)]).to(dtype)
        state["weight"] = weight.to(dtype)
        state["bias"] = normal(classes, scale=0.1) if case["bias"] else None
        if case["way"] == "step":
            state["grad_loss"] = torch.full((rows,), 1.0 / rows, device="cuda")
    else:
        shapes = _shapes(case)
        state["params"] = [normal(*s, scale=0.1) for s in shapes]
        grads = [normal(*s, scale=1e-3) for s in shapes]
        for t in grads:  # leaves that no row of the batch reaches
            if t.dim() == 2 and t.shape[0] > 100:
                t[torch.rand(t.shape[0], generator=g, device="cuda") < 0.3] = 0
        state["grads"] = [t.to(dtype) for t in grads]
        m = [normal(*s, scale=3e-4) for s in shapes]
        v = [normal(*s, scale=1e-3).square() + 1e-10 for s in shapes]
        if case["bits"] == 8:
            state["moments"] = [(*_coded(a.reshape(-1), 0.5, False), *_coded(b.reshape(-1).sqrt(), 0.5, True)) for a, b in zip(m, v)]
        else:
            state["moments"] = list(zip(m, v))
        state["copies"] = [t.bfloat16() if t.dim() == 2 else None for t in state["params"]] if case["dtype"] == "bf16" else None
        state["step"], state["seed"] = 1000, seed % 65_521
    return state


# The 8-bit states, on flat tensors.

def _hash(x):
    """A 32-bit hash of 32-bit numbers held in 64 bits."""
    x = ((x ^ (x >> 16)) * 0x7FEB352D) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0x846CA68B) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _key(seed, step, tensor):
    return _hash((_hash((seed + 0x9E3779B9 * step) & 0xFFFFFFFF) + tensor) & 0xFFFFFFFF)


def _randoms(n, key):
    """Two random numbers in [0, 1) for each of n values, multiples of 2^-16."""
    bits = _hash((torch.arange(n, device="cuda") + key) & 0xFFFFFFFF)
    return (bits & 0xFFFF).float() / 65536, (bits >> 16).float() / 65536


def _blocks(x):
    n = x.numel()
    return torch.nn.functional.pad(x, (0, -n % BLOCK)).reshape(-1, BLOCK)


def _coded(x, u, keep):
    """(codes, scale bytes) of x; `keep`: no value above zero gets the code of zero."""
    n = x.numel()
    scale = (torch.frexp(_blocks(x.abs()).amax(1))[1] - 1).clamp(-126, 127)
    scale = torch.where(_blocks(x.abs()).amax(1) > 0, scale + 127, torch.zeros_like(scale))
    back = torch.where(scale > 0, 134 - scale, torch.zeros_like(scale)).repeat_interleave(BLOCK)[:n]
    y = torch.ldexp(x.abs(), back)
    exponent = (torch.frexp(y)[1] - 1).clamp(min=-6)
    whole = torch.floor(torch.ldexp(y, 3 - exponent) + u)  # in steps of the code: 0 to 16
    if keep:
        whole = torch.where((x > 0) & (whole == 0), torch.ones_like(whole), whole)
    code = (8 * (exponent + 6) + whole.int()).clamp(max=126)
    code = torch.where(x < 0, code + 128, code)
    return torch.where(scale.repeat_interleave(BLOCK)[:n] > 0, code, torch.zeros_like(code)).to(torch.uint8), scale.to(torch.uint8)


def _values(code, scale, dtype=torch.float32):
    """The values that codes and scale bytes stand for."""
    code, scale = code.int(), scale.int().repeat_interleave(BLOCK)[:code.numel()]
    exponent = (code >> 3) & 15
    whole = (code & 7) + 8 * (exponent > 0).int()
    y = torch.ldexp(whole.to(dtype), exponent.clamp(min=1) - 10 + scale - 134)
    return torch.where(code > 127, -y, y)


# The plain forms.

def _tokens(state):
    tokens = state["ids"].long() + state["offsets"]
    here = (state["ids"] >= 0) & (tokens < state["vectors"])
    return tokens, here


def _plain_embed(state):
    tokens, here = _tokens(state)
    if state["case"]["way"] == "forward":
        table = state["table"].float()
        rows = table[tokens.clamp(min=0)].mul_(here[..., None])
        return (rows.sum(1) * state["scale"]).to(state["table"].dtype)
    grad = state["grad"].float() * state["scale"]
    row = torch.arange(grad.shape[0], device=grad.device)[:, None].expand_as(tokens)
    out = torch.zeros(state["vectors"], grad.shape[1], device=grad.device)
    return out.index_add_(0, tokens[here], grad[row[here]]).to(state["grad"].dtype)


def _plain_norm(state):
    x = state["x"].float()
    if state["case"]["way"] == "forward":
        mean = x.mean(1)
        centred = x - mean[:, None]
        rstd = torch.rsqrt(centred.square().mean(1) + 1e-5)
        return (centred * rstd[:, None] * state["weight"] + state["bias"]).to(state["x"].dtype), mean, rstd
    grad = state["grad"].float()
    unit = (x - state["mean"][:, None]) * state["rstd"][:, None]
    g = grad * state["weight"]
    dx = state["rstd"][:, None] * (g - g.mean(1, keepdim=True) - unit * (g * unit).mean(1, keepdim=True))
    return dx.to(state["x"].dtype), (grad * unit).sum(0), grad.sum(0)


def _plain_loss(state):
    hidden, weight, target = state["hidden"].float(), state["weight"].float(), state["targets"].long()
    logits = hidden @ weight.T
    if state["bias"] is not None:
        logits += state["bias"]
    most = logits.amax(1)
    p = torch.exp(logits - most[:, None])
    total = p.sum(1)
    log = torch.log(total)
    lse = most + log
    counts = target >= 0
    at = target.clamp(min=0)[:, None]
    loss = torch.where(counts, log + (most - logits.gather(1, at)[:, 0]), torch.zeros_like(lse))
    if state["case"]["way"] == "forward":
        return loss, lse
    g = torch.where(counts, state["grad_loss"], torch.zeros_like(lse))
    p *= (g / total)[:, None]
    p.scatter_add_(1, at, -g[:, None])
    out = [loss, lse, (p @ weight).to(state["hidden"].dtype), (p.T @ hidden).to(state["weight"].dtype)]
    return out + [p.sum(0)] if state["bias"] is not None else out


def _plain_adamw_one(p, grad, moments, copy, step, key):
    g = grad.float()
    eight = len(moments) == 4
    if eight:
        m, v = _values(*moments[:2]).view_as(p), _values(*moments[2:]).square().view_as(p)
    else:
        m, v = moments
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g * g
    p.mul_(1 - RATE * DECAY)
    p.sub_(RATE / (1 - BETA1 ** step) * m / (v.sqrt() / math.sqrt(1 - BETA2 ** step) + EPS))
    if copy is not None:
        copy.copy_(p)
    if eight:
        u, w = _randoms(p.numel(), key)
        coded = (*_coded(m.reshape(-1), u, False), *_coded(v.reshape(-1).sqrt(), w, True))
        [old.copy_(new) for old, new in zip(moments, coded)]
        m, v = _values(*coded[:2]).view_as(p).bfloat16(), _values(*coded[2:]).square().view_as(p).bfloat16()
    else:
        m, v = moments[0].copy_(m), moments[1].copy_(v)
    return p, m, v, copy


def _plain_adamw(state):
    copies = state["copies"] or [None] * len(state["params"])
    return [_plain_adamw_one(p, g, s, c, state["step"], _key(state["seed"], state["step"], k))
            for k, (p, g, s, c) in enumerate(zip(state["params"], state["grads"], state["moments"], copies))]


# The framework's operators.

def _own_embed(pk, state):
    if state["case"]["way"] == "forward":
        return pk.head_embed(state["table"], state["ids"], state["offsets"], state["scale"])
    return pk.head_embed_grad(state["grad"], state["ids"], state["vectors"], state["offsets"], state["scale"])


def _own_norm(pk, state):
    if state["case"]["way"] == "forward":
        return pk.head_layer_norm(state["x"], state["weight"], state["bias"], 1e-5)
    return pk.head_layer_norm_grad(state["grad"], state["x"], state["weight"], state["mean"], state["rstd"])


def _own_loss(pk, state):
    loss, lse = pk.head_cross_entropy(state["hidden"], state["weight"], state["targets"], state["bias"])
    if state["case"]["way"] == "forward":
        return loss, lse
    grads = pk.head_cross_entropy_grad(state["grad_loss"], state["hidden"], state["weight"], state["targets"], lse, state["bias"])
    return [loss, lse, *(t for t in grads if t is not None)]


def _own_adamw(pk, state):
    pk.head_adamw(state["params"], state["grads"], state["moments"], state["step"], RATE, BETA1, BETA2, EPS, DECAY,
                  copies=state["copies"], seed=state["seed"])
    moments = state["moments"] if state["case"]["bits"] == 32 else pk.head_adamw_values(state["moments"], state["params"])
    copies = state["copies"] or [None] * len(state["params"])
    return [(p, m, v, c) for p, (m, v), c in zip(state["params"], moments, copies)]


def run(state):
    op = state["case"]["op"]
    if op == "adamw":
        state["step"] += 1
    if own:
        import paper_2301_13441_amd as pk
        return {"embed": _own_embed, "norm": _own_norm, "loss": _own_loss, "adamw": _own_adamw}[op](pk, state)
    return {"embed": _plain_embed, "norm": _plain_norm, "loss": _plain_loss, "adamw": _plain_adamw}[op](state)


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "embed":
        tokens, vectors = case["rows"] * case["trees"], case["trees"] * ((2 << case["depth"]) - 1)
        read = 4 * tokens + 8 * case["trees"]
        if case["way"] == "forward":  # no more vectors than there are leaves, or ids
            return {"bytes": read + e * case["dim"] * (min(tokens, case["trees"] << case["depth"]) + case["rows"]), "flops": tokens * case["dim"]}
        return {"bytes": read + e * case["dim"] * (vectors + case["rows"]), "flops": tokens * case["dim"]}
    if case["op"] == "norm":
        values = case["rows"] * case["dim"]
        if case["way"] == "forward":
            return {"bytes": 2 * e * values + 8 * case["rows"] + 8 * case["dim"], "flops": 7 * values}
        return {"bytes": 3 * e * values + 8 * case["rows"] + 12 * case["dim"], "flops": 14 * values}
    if case["op"] == "loss":
        rows, dim, classes = case["rows"], case["dim"], case["classes"]
        values = rows * dim + classes * dim
        small = 12 * rows + 4 * classes * case["bias"]
        if case["way"] == "forward":
            return {"bytes": e * values + small, "flops": 2 * rows * classes * dim}
        return {"bytes": 2 * e * values + small + 4 * rows + 4 * classes * case["bias"], "flops": 6 * rows * classes * dim}
    values = sum(math.prod(s) for s in _shapes(case))
    copied = sum(math.prod(s) for s in _shapes(case) if len(s) == 2) if case["dtype"] == "bf16" else 0
    each = 8 + e + (16 if case["bits"] == 32 else 4 + 4 / BLOCK + 4)  # 8 bits: the values come back too, in 16 bits
    return {"bytes": int(each * values) + 2 * copied, "flops": 15 * values}


# The definitions, in 64 bits.

def exact(case, seed):
    state = prepare(case, seed)
    d = torch.float64
    if case["op"] == "embed":
        ids, offsets = state["ids"], state["offsets"].tolist()
        if case["way"] == "forward":
            table = torch.cat([state["table"].to(d), torch.zeros(1, case["dim"], dtype=d, device=ids.device)])  # a last vector of zeros for ids of -1
            out = torch.zeros(case["rows"], case["dim"], dtype=d, device=ids.device)
            for t, offset in enumerate(offsets):
                out += table[torch.where(ids[:, t] < 0, state["vectors"], ids[:, t].long() + offset)]
            return out * state["scale"]
        out = torch.zeros(state["vectors"] + 1, case["dim"], dtype=d, device=ids.device)
        grad = state["grad"].to(d)
        for t, offset in enumerate(offsets):
            out.index_add_(0, torch.where(ids[:, t] < 0, state["vectors"], ids[:, t].long() + offset), grad)
        return out[:-1] * state["scale"]
    if case["op"] == "norm":
        n, dim = case["rows"], case["dim"]
        w, b = state["weight"].to(d), state["bias"].to(d)
        parts, sums = [], torch.zeros(2, dim, dtype=d, device=w.device)
        for lo in range(0, n, 1 << 16):
            x = state["x"][lo:lo + (1 << 16)].to(d)
            if case["way"] == "forward":
                var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
                rstd = 1 / torch.sqrt(var + 1e-5)
                parts.append(((x - mean) * rstd * w + b, mean[:, 0], rstd[:, 0]))
                continue
            mean, rstd = (state[k][lo:lo + (1 << 16)].to(d)[:, None] for k in ("mean", "rstd"))
            g = state["grad"][lo:lo + (1 << 16)].to(d)
            unit = rstd * (x - mean)
            sums += torch.stack([(g * unit).sum(0), g.sum(0)])
            along = (g * w).sum(1, keepdim=True) + unit * (g * w * unit).sum(1, keepdim=True)
            parts.append((rstd * (g * w - along / dim),))
        parts = tuple(torch.cat(p) for p in zip(*parts))
        return parts if case["way"] == "forward" else (parts[0], sums[0], sums[1])
    if case["op"] == "loss":
        n, classes = case["rows"], case["classes"]
        weight = state["weight"].to(d)
        bias = state["bias"].to(d) if case["bias"] else torch.zeros(classes, dtype=d, device=weight.device)
        d_weight, d_bias, losses, lses, d_hidden = torch.zeros_like(weight), torch.zeros_like(bias), [], [], []
        for lo in range(0, n, 2048):
            h, t = state["hidden"][lo:lo + 2048].to(d), state["targets"][lo:lo + 2048].long()
            logits = torch.addmm(bias, h, weight.t())
            lse = torch.logsumexp(logits, 1)
            row = torch.arange(len(t), device=t.device)[t >= 0]
            loss = torch.zeros_like(lse)
            loss[row] = lse[row] - logits[row, t[row]]
            losses.append(loss)
            lses.append(lse)
            if case["way"] == "step":
                p = torch.exp(logits - lse[:, None])
                p[row, t[row]] -= 1
                p *= (state["grad_loss"][lo:lo + 2048].to(d) * (t >= 0))[:, None]
                d_hidden.append(p.mm(weight))
                d_weight.addmm_(p.t(), h)
                d_bias += p.sum(0)
        if case["way"] == "forward":
            return torch.cat(losses), torch.cat(lses)
        return [torch.cat(losses), torch.cat(lses), torch.cat(d_hidden), d_weight] + ([d_bias] if case["bias"] else [])
    step, out = state["step"] + 1, []
    for k, (p, g, s) in enumerate(zip(state["params"], state["grads"], state["moments"])):
        p, g = p.to(d), g.to(d)
        m, v = (_values(*s[:2], d).view_as(p), _values(*s[2:], d).view_as(p) ** 2) if len(s) == 4 else (s[0].to(d), s[1].to(d))
        m, v = m + (1 - BETA1) * (g - m), v + (1 - BETA2) * (g ** 2 - v)
        p = p - RATE * (DECAY * p + m / (1 - BETA1 ** step) / ((v / (1 - BETA2 ** step)) ** 0.5 + EPS))
        if len(s) == 4:
            u, w = _randoms(p.numel(), _key(state["seed"], step, k))
            m = _values(*_coded(m.reshape(-1), u.to(d), False), d).view_as(p)
            v = _values(*_coded(v.reshape(-1).sqrt(), w.to(d), True), d).view_as(p) ** 2
        out.append((p, m, v, p if state["copies"] and state["copies"][k] is not None else None))
    return out
