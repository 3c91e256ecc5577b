"""What a trunk of gated blocks needs around and after them: the norm before a block (`norm`, `norm_grad`); what joins a block's
result to the residual stream, its norm, gate and scale, with the next block's norm (`join`, `join_grad`); updates of
matrices made orthogonal by Newton-Schulz products (`orthogonalise`), and the step that takes them (`muon`).

With `own` false `run` computes an operator in elementary torch operations, in 32 bits; with `own` true it makes the
calls of `paper_2210_07768_amd.train`.  A case is

    op             norm, norm_grad, join, join_grad, orthogonalise, muon
    norm*, join*   records, dim, dtype of the block's side, stream (dtype of the residual stream: the same or float32), vectors
                   (dtype of weights and scales: the same or float32), kind (rms, layer), pad (elements between rows of the
                   stream beyond its columns)
    join*          gate (none, row: one a record, full: one an element), act (sigmoid, none), scale (vector or number), post
                   (the block's result is normed), then (the next block's norm is taken too)
    orthogonalise  matrices ("rows x columns x count" of each shape), dtype (of the matrices), result (of the results), steps
    muon           matrices, param and grad dtypes, copy (a bfloat16 copy of the weights is written too), nesterov, steps
"""
import math
import random

import torch

own = False

EPS = 1e-6
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
TINY = 1e-7                               # beside a matrix's norm
LR, MOMENTUM, DECAY, GRAD_SCALE = 2e-3, 0.95, 0.01, 0.5


def listed():
    def norm(name, records, dim, dtype, op="norm", stream=None, vectors="float32", kind="rms", pad=0):
        return {"name": name, "op": op, "records": records, "dim": dim, "dtype": dtype, "stream": stream or dtype, "vectors": vectors, "kind": kind, "pad": pad}

    def join(name, records, dim, dtype, op="join", gate="full", act="sigmoid", scale="vector", post=True, then=True, **more):
        return {**norm(name, records, dim, dtype, op, **more), "gate": gate, "act": act, "scale": scale, "post": post, "then": then}

    def orthogonalise(name, matrices, dtype, result, steps=5):
        return {"name": name, "op": "orthogonalise", "matrices": matrices, "dtype": dtype, "result": result, "steps": steps}

    def muon(name, matrices, param, grad, copy=False, nesterov=True, steps=5):
        return {"name": name, "op": "muon", "matrices": matrices, "param": param, "grad": grad, "copy": copy, "nesterov": nesterov, "steps": steps}

    return [
        # one record of a serving loop: 164 slots of 16, before the first block
        norm("norm_request", 1, 2_624, "bfloat16"),
        # a large batch of the widest workload
        norm("norm_wide", 65_536, 2_624, "bfloat16"),
        # the gradient for the smallest workload's batch, 24 slots of 16 with 32-bit weights
        norm("norm_grad_small", 4_096, 384, "float32", op="norm_grad", kind="layer"),
        # and at a width that is a multiple of nothing, rows of it cut out of wider ones
        norm("norm_grad_odd", 16_384, 411, "float16", op="norm_grad", kind="layer", pad=3),
        # one record behind a block of the list-heavy workload (96 slots of 16)
        join("join_request", 1, 1_536, "bfloat16"),
        # a large batch of the widest workload, its residual stream in 32 bits
        join("join_wide", 65_536, 2_624, "bfloat16", stream="float32"),
        # the gradient where a record has one gate, and the scale is a number
        join("join_grad_odd", 1_000, 411, "float16", op="join_grad", gate="row", scale="number", kind="layer", vectors="float16"),
        # a step's batch of the widest workload
        join("join_grad_wide", 16_384, 2_624, "bfloat16", op="join_grad"),
        # one matrix of a very small model, 32-bit results
        orthogonalise("orthogonalise_small", "128x96x1", "float32", "float32"),
        # the two matrices of the widest workload's block
        orthogonalise("orthogonalise_wide", "4096x2624x2", "bfloat16", "bfloat16"),
        # a trunk of six blocks behind the smallest workload's rows: 32-bit weights, with the copies that its products read
        muon("muon_trunk", "1024x384x12,384x1024x6", "float32", "float32", copy=True),
        # one block of the widest workload and the matrix back to the stream
        muon("muon_wide", "4096x2624x2,2624x4096x1", "bfloat16", "bfloat16"),
    ]


MOST_ELEMENTS = 65_536 * 2_624


def _products(matrices, steps):
    """Multiplications and additions of the Newton-Schulz steps; of a symmetric product the half that is needed."""
    total = 0
    for rows, columns in matrices:
        m, n = min(rows, columns), max(rows, columns)
        total += steps * (m * (m + 1) * n + m * (m + 1) * m + 2 * m * m * n)
    return total


def _log(rng, low, high):
    n = round(low * (high / low) ** rng.random())
    return max(low, min(high, n))


def draw(rng):
    op = rng.choice(["norm", "norm_grad", "join", "join_grad", "orthogonalise", "muon"])
    if op.startswith(("norm", "join")):
        while True:
            records, dim = _log(rng, 1, 65_536), _log(rng, 1, 16_384)
            if rng.random() < 0.6:  # (widths are slots x dim more often than not)
                dim = -(-dim // 16) * 16
            dtype = rng.choice(["bfloat16", "bfloat16", "float16", "float32"])
            case = {"op": op, "records": records, "dim": dim, "dtype": dtype, "stream": rng.choice([dtype, "float32"]), "vectors": rng.choice([dtype, "float32"]),
                    "kind": rng.choice(["rms", "layer"]), "pad": rng.choice([0, 0, 8, rng.randint(1, 40)])}
            if op.startswith("join"):
                case |= {"gate": rng.choice(["none", "row", "full", "full"]), "act": rng.choice(["sigmoid", "sigmoid", "none"]), "scale": rng.choice(["vector", "number"]),
                         "post": rng.random() < 0.7, "then": rng.random() < 0.7}
            if records * (dim + case["pad"]) <= MOST_ELEMENTS // {"norm": 1, "norm_grad": 2, "join": 1, "join_grad": 4}[op]:
                return case
    most = _products(_shapes("4096x2624x2"), 5) // 2
    while True:
        shapes = []
        for _ in range(rng.randint(1, 4)):
            rows, columns = _log(rng, 1, 4_096), _log(rng, 1, 4_096)
            if rng.random() < 0.6:
                rows, columns = -(-rows // 16) * 16, -(-columns // 16) * 16
            shapes.append("%dx%dx%d" % (rows, columns, rng.randint(1, 6)))
        case = {"op": op, "matrices": ",".join(shapes), "steps": rng.choice([5, 5, 5, 3, 6])}
        if _products(_shapes(case["matrices"]), case["steps"]) > most or len(_shapes(case["matrices"])) > 16:
            continue
        if op == "orthogonalise":
            dtype = rng.choice(["bfloat16", "bfloat16", "float16", "float32"])
            return case | {"dtype": dtype, "result": rng.choice([dtype, "bfloat16"])}
        param = rng.choice(["float32", "float32", "bfloat16", "float16"])
        return case | {"param": param, "grad": param if param != "float32" else rng.choice(["float32", "bfloat16"]), "copy": param == "float32" and rng.random() < 0.5,
                       "nesterov": rng.random() < 0.7}


# ------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 2 + 1)
    return g


def _dtype(name):
    return {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}[name]


def _shapes(text):
    """[(rows, columns)] of "rows x columns x count, ..."."""
    shapes = []
    for part in text.split(","):
        rows, columns, count = (int(n) for n in part.split("x"))
        shapes += [(rows, columns)] * count
    return shapes


def _gradient(g, rows, columns, size):
    """A gradient as a block's matrices get it: a sum over directions of which few are large."""
    n = min(rows, columns, 512)
    r = lambda a, b: torch.randn(a, b, device="cuda", generator=g)  # noqa: E731
    strength = torch.arange(1, n + 1, device="cuda").float().pow(-0.7)
    few = torch.mm(r(rows, n) * strength, r(n, columns)) / strength.square().sum().sqrt()
    return (few + 0.1 * r(rows, columns)) * size


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case}
    if case["op"].startswith(("norm", "join")):
        n, d = case["records"], case["dim"]
        dtype, stream, vectors = _dtype(case["dtype"]), _dtype(case["stream"]), _dtype(case["vectors"])
        r = lambda *shape: torch.randn(*shape, device="cuda", generator=g)  # noqa: E731
        size = torch.exp(0.5 * r(n, 1))  # (records are not of one size, and columns have means of their own)
        s["x"] = (r(n, d + case["pad"]).mul_(size).add_(0.2 * r(d + case["pad"]))).to(stream)[:, :d]
        s["weight"] = (1 + 0.2 * r(d)).to(vectors)
        if case["op"].startswith("norm"):
            if case["op"] == "norm_grad":
                s["dy"] = r(n, d).to(dtype)
            return s
        s["y"] = (r(n, d).mul_(torch.exp(0.5 * r(n, 1))).add_(0.2 * r(d))).to(dtype)
        s["gate"] = None if case["gate"] == "none" else (r(n, 1 if case["gate"] == "row" else d) + 0.5).to(dtype)
        s["scale"] = (0.3 + 0.05 * r(d)).to(vectors) if case["scale"] == "vector" else 0.25
        if not case["post"]:
            s["weight"] = None
        s["next_weight"] = (1 + 0.2 * r(d)).to(vectors) if case["then"] else None
        if case["op"] == "join_grad":
            s["dout"] = r(n, d).to(stream)
            s["dnext"] = r(n, d).to(dtype) if case["then"] else None
        return s
    shapes = _shapes(case["matrices"])
    if case["op"] == "orthogonalise":
        s["matrices"] = [_gradient(g, a, b, 1e-3).to(_dtype(case["dtype"])) for a, b in shapes]
        return s
    r = lambda a, b, size: torch.randn(a, b, device="cuda", generator=g) * size  # noqa: E731
    s["param"] = [r(a, b, 1 / math.sqrt(b)).to(_dtype(case["param"])) for a, b in shapes]
    s["grad"] = [_gradient(g, a, b, 2e-3).to(_dtype(case["grad"])) for a, b in shapes]
    s["momentum"] = [_gradient(g, a, b, 5e-3) for a, b in shapes]
    if case["copy"]:
        s["copy"] = [torch.zeros(a, b, device="cuda", dtype=torch.bfloat16) for a, b in shapes]
    return s


# ------------------------------------------------------------------ plain forms
def _normed(x, kind):
    """Rows of x at unit size, and what they were divided by."""
    x = x - x.mean(1, keepdim=True) if kind == "layer" else x
    root = (x.square().mean(1, keepdim=True) + EPS).sqrt()
    return x / root, root


def _norm_slope(p, unit, root, kind):
    """The gradient of _normed's rows, given that of its result."""
    p = p - p.mean(1, keepdim=True) if kind == "layer" else p
    return (p - unit * (p * unit).mean(1, keepdim=True)) / root


def _norm(s):
    return (_normed(s["x"].float(), s["case"]["kind"])[0] * s["weight"].float()).to(_dtype(s["case"]["dtype"]))


def _norm_grad(s):
    kind = s["case"]["kind"]
    unit, root = _normed(s["x"].float(), kind)
    dy = s["dy"].float()
    return {"dx": _norm_slope(dy * s["weight"].float(), unit, root, kind).to(s["x"].dtype), "dweight": (dy * unit).sum(0).to(s["weight"].dtype)}


def _parts(s):
    """Of a join in 32 bits: the block's rows, normed where they are, with what they were divided by; the gate; the scale."""
    case = s["case"]
    unit, root = _normed(s["y"].float(), case["kind"]) if case["post"] else (s["y"].float(), None)
    gate = 1.0 if s["gate"] is None else torch.sigmoid(s["gate"].float()) if case["act"] == "sigmoid" else s["gate"].float()
    scale = s["scale"] if case["scale"] == "number" else s["scale"].float()
    return unit, root, gate, scale, s["weight"].float() if case["post"] else 1.0


def _join(s):
    case = s["case"]
    unit, _, gate, scale, weight = _parts(s)
    out = s["x"].float() + scale * gate * unit * weight
    if not case["then"]:
        return {"out": out.to(s["x"].dtype)}
    return {"out": out.to(s["x"].dtype), "next": (_normed(out, case["kind"])[0] * s["next_weight"].float()).to(s["y"].dtype)}


def _join_grad(s):
    case = s["case"]
    kind, r = case["kind"], {}
    unit, root, gate, scale, weight = _parts(s)
    d = s["dout"].float()
    if case["then"]:
        after, after_root = _normed(s["x"].float() + scale * gate * unit * weight, kind)
        dnext = s["dnext"].float()
        r["dnext_weight"] = (dnext * after).sum(0).to(s["next_weight"].dtype)
        d = d + _norm_slope(dnext * s["next_weight"].float(), after, after_root, kind)
    r["dx"] = d.to(s["x"].dtype)
    through = d * gate * unit
    if case["post"]:
        r["dweight"] = (through.sum(0) * scale).to(s["weight"].dtype)
    if case["scale"] == "vector":
        r["dscale"] = (through.sum(0) * weight).to(s["scale"].dtype)
    if s["gate"] is not None:
        slope = d * scale * unit * weight
        slope = slope.sum(1, keepdim=True) if case["gate"] == "row" else slope
        r["dgate"] = (slope * gate * (1 - gate) if case["act"] == "sigmoid" else slope).to(s["gate"].dtype)
    p = d * scale * gate * weight
    r["dy"] = (_norm_slope(p, unit, root, kind) if case["post"] else p).to(s["y"].dtype)
    return r


def _orthogonal(u, steps):
    x = u.t() if u.shape[0] > u.shape[1] else u
    x = x / (x.double().square().sum().sqrt() + TINY).float()
    a, b, c = COEFFICIENTS
    for _ in range(steps):
        gram = x @ x.t()
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.t() if u.shape[0] > u.shape[1] else x


def _orthogonalise(s):
    return [_orthogonal(u.float(), s["case"]["steps"]).to(_dtype(s["case"]["result"]), memory_format=torch.contiguous_format) for u in s["matrices"]]


def _factor(shape):
    """So that a step's elements are as large as those of an Adam step: a fifth of the learning rate."""
    return 0.2 * math.sqrt(max(shape))


def _muon_one(s, i):
    case, p, m = s["case"], s["param"][i], s["momentum"][i]
    g = s["grad"][i].float() * GRAD_SCALE
    m.mul_(MOMENTUM).add_(g)
    u = _orthogonal(g + MOMENTUM * m if case["nesterov"] else m, case["steps"])
    new = p.float() * (1 - LR * DECAY) - u * (LR * _factor(p.shape))
    p.copy_(new)
    if case["copy"]:
        s["copy"][i].copy_(new)


def _muon(s):
    [_muon_one(s, i) for i in range(len(s["param"]))]
    return {k: s[k] for k in ("param", "momentum", "copy") if k in s}


PLAIN = {"norm": _norm, "norm_grad": _norm_grad, "join": _join, "join_grad": _join_grad, "orthogonalise": _orthogonalise, "muon": _muon}


# ------------------------------------------------------------------ the framework's operators
def _own(s):
    from paper_2210_07768_amd import train as T

    case = s["case"]
    if case["op"] == "norm":
        return T.norm(s["x"], s["weight"], kind=case["kind"], eps=EPS, dtype=_dtype(case["dtype"]))
    if case["op"] == "norm_grad":
        dx, dweight = T.norm_backward(s["dy"], s["x"], s["weight"], kind=case["kind"], eps=EPS)
        return {"dx": dx, "dweight": dweight}
    if case["op"] == "join":
        got = T.join(s["x"], s["y"], s["weight"], s["gate"], s["scale"], s["next_weight"], post=case["post"], then=case["then"], gate_act=case["act"], kind=case["kind"], eps=EPS)
        return {"out": got[0], "next": got[1]} if case["then"] else {"out": got}
    if case["op"] == "join_grad":
        got = T.join_backward(s["dout"], s["dnext"], s["x"], s["y"], s["weight"], s["gate"], s["scale"], s["next_weight"], post=case["post"], then=case["then"],
                              gate_act=case["act"], kind=case["kind"], eps=EPS)
        return {k: v for k, v in got._asdict().items() if v is not None}
    if case["op"] == "orthogonalise":
        return T.orthogonalise(s["matrices"], steps=case["steps"], coefficients=COEFFICIENTS, eps=TINY, dtype=_dtype(case["result"]))
    T.muon(s["param"], s["grad"], s["momentum"], s.get("copy"), lr=LR, momentum=MOMENTUM, nesterov=case["nesterov"], weight_decay=DECAY, grad_scale=GRAD_SCALE, adjust="rms",
           steps=case["steps"], coefficients=COEFFICIENTS, eps=TINY)
    return {k: s[k] for k in ("param", "momentum", "copy") if k in s}


def run(state):
    return _own(state) if own else PLAIN[state["case"]["op"]](state)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    size = {"float32": 4, "bfloat16": 2, "float16": 2}
    if case["op"].startswith(("norm", "join")):
        n, d, e, x, v = case["records"], case["dim"], size[case["dtype"]], size[case["stream"]], size[case["vectors"]]
        if case["op"] == "norm":
            return {"bytes": n * d * (x + e) + d * v, "flops": 5 * n * d}
        if case["op"] == "norm_grad":
            return {"bytes": n * d * (2 * x + e) + 2 * d * v, "flops": 12 * n * d}
        gate = e * {"none": 0, "row": n, "full": n * d}[case["gate"]]
        vectors = d * v * (int(case["post"]) + (case["scale"] == "vector") + int(case["then"]))
        then = int(case["then"])
        if case["op"] == "join":
            return {"bytes": n * d * (2 * x + e + then * e) + gate + vectors, "flops": 16 * n * d}
        return {"bytes": n * d * (3 * x + 2 * e + then * e) + 2 * gate + 2 * vectors, "flops": 40 * n * d}
    shapes = _shapes(case["matrices"])
    n, flops = sum(a * b for a, b in shapes), _products(shapes, case["steps"])
    if case["op"] == "orthogonalise":
        return {"bytes": n * (size[case["dtype"]] + size[case["result"]]), "flops": flops}
    return {"bytes": n * (2 * size[case["param"]] + size[case["grad"]] + 8 + (2 if case["copy"] else 0)), "flops": flops}


# ------------------------------------------------------------------ the definitions, in 64 bits
def _exact_unit(x, kind):
    """(unit rows, 1 / root) by second moments."""
    mean = x.sum(1, keepdim=True) / x.shape[1] if kind == "layer" else torch.zeros((), dtype=torch.float64, device="cuda")
    inverse = torch.rsqrt(((x - mean) ** 2).sum(1, keepdim=True) / x.shape[1] + EPS)
    return (x - mean) * inverse, inverse


def _exact_back(p, unit, inverse, kind):
    d = p.shape[1]
    along = unit * ((unit * p).sum(1, keepdim=True) / d)
    return inverse * (p - along - (p.sum(1, keepdim=True) / d if kind == "layer" else 0.0))


def _exact_norm(case, s):
    unit, inverse = _exact_unit(s["x"].double(), case["kind"])
    if case["op"] == "norm":
        return s["weight"].double() * unit
    dy = s["dy"].double()
    return {"dx": _exact_back(s["weight"].double() * dy, unit, inverse, case["kind"]), "dweight": torch.einsum("rc,rc->c", dy, unit)}


def _exact_join(case, s):
    kind, one = case["kind"], torch.ones((), dtype=torch.float64, device="cuda")
    y = s["y"].double()
    unit, inverse = _exact_unit(y, kind) if case["post"] else (y, one)
    weight = s["weight"].double() if case["post"] else one
    scale = s["scale"].double() if case["scale"] == "vector" else one * s["scale"]
    z = None if s["gate"] is None else s["gate"].double()
    gate = one if z is None else 1 / (1 + torch.exp(-z)) if case["act"] == "sigmoid" else z
    out = torch.addcmul(s["x"].double(), unit * weight, gate * scale)
    if case["then"]:
        after, after_inverse = _exact_unit(out, kind)
    if case["op"] == "join":
        return {"out": out, **({"next": s["next_weight"].double() * after} if case["then"] else {})}
    r, d = {}, s["dout"].double()
    if case["then"]:
        dnext = s["dnext"].double()
        r["dnext_weight"] = torch.einsum("rc,rc->c", dnext, after)
        d = d + _exact_back(s["next_weight"].double() * dnext, after, after_inverse, kind)
        del after, dnext
    r["dx"] = d
    if case["post"]:
        r["dweight"] = torch.einsum("rc,rc->c", d, unit * gate * scale)
    if case["scale"] == "vector":
        r["dscale"] = torch.einsum("rc,rc->c", d, unit * gate * weight)
    if z is not None:
        slope = d * (unit * (scale * weight))
        slope = slope.sum(1, keepdim=True) if case["gate"] == "row" else slope
        r["dgate"] = slope * torch.exp(-z) / (1 + torch.exp(-z)) ** 2 if case["act"] == "sigmoid" else slope
    p = d * (gate * (scale * weight))
    r["dy"] = _exact_back(p, unit, inverse, kind) if case["post"] else p
    return r


def _exact_orthogonal(u, steps):
    """X q(X^T X) on the narrow side, q(G) = aI + G(bI + cG)."""
    tall = u.shape[0] >= u.shape[1]
    x = (u if tall else u.t().contiguous()) / (torch.linalg.vector_norm(u) + TINY)
    a, b, c = COEFFICIENTS
    eye = torch.eye(x.shape[1], dtype=torch.float64, device="cuda")
    for _ in range(steps):
        gram = torch.mm(x.t(), x)
        x = torch.mm(x, a * eye + torch.mm(gram, b * eye + c * gram))
    return x if tall else x.t().contiguous()


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"].startswith("norm"):
        return _exact_norm(case, s)
    if case["op"].startswith("join"):
        return _exact_join(case, s)
    if case["op"] == "orthogonalise":
        return [_exact_orthogonal(u.double(), case["steps"]) for u in s["matrices"]]
    out = {"param": [], "momentum": []} | ({"copy": []} if case["copy"] else {})
    for p, g, m in zip(s["param"], s["grad"], s["momentum"]):
        g = GRAD_SCALE * g.double()
        m = g + MOMENTUM * m.double()
        u = _exact_orthogonal(g + MOMENTUM * m if case["nesterov"] else m, case["steps"])
        p = p.double() - LR * (DECAY * p.double() + _factor(p.shape) * u)
        out["param"].append(p)
        out["momentum"].append(m)
        if case["copy"]:
            out["copy"].append(p)
    return out
