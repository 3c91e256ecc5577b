"""What a trainer does with the signs that extraction leaves in device memory: slots of 64-bit signs become rows of a
table, pooled per record (`embed`), and the table's gradient comes back the same way (`embed_grad`); the pooled rows go
through a gated feed-forward block (`gated`, `gated_grad`); weights and tables take an AdamW step, all tensors at once,
with states in 32 or in 8 bits (`adamw`).

With `own` false `run` computes an operator in elementary torch operations, in 32 bits; with `own` true it makes the
calls of `paper_2210_07768_amd.train`.  A case is

    op        embed, embed_grad, gated, gated_grad, adamw
    embed*    records, single (slots with one sign a record), ragged (slots with a list a record: 1 + Poisson(mean_items)
              items in every other one of them, Poisson(mean_items), so sometimes none, in the others), vocab (distinct
              tokens of a slot, Zipf-ranked), rows and dim of the table, dtype of table and gradient, mean or sum
    gated*    records, inputs, hidden, dtype, act, pad (elements between the rows of x beyond its columns)
    adamw     tensors, of smallest to largest elements; param and grad dtypes, copy (a bfloat16 copy of the weights is
              written too), bits of a state, step
"""
import math
import random

import torch

own = False

U64 = 0xFFFFFFFFFFFFFFFF
BLOCK = 32  # elements that share a scale in 8-bit states


def listed():
    def embed(name, records, single, ragged, rows, dim, dtype, mean=False, mean_items=3.0, vocab=10_000_000, op="embed"):
        return {"name": name, "op": op, "records": records, "single": single, "ragged": ragged, "mean_items": mean_items,
                "vocab": vocab, "rows": rows, "dim": dim, "dtype": dtype, "mean": mean}

    def gated(name, records, inputs, hidden, dtype, act="silu", pad=0, op="gated"):
        return {"name": name, "op": op, "records": records, "inputs": inputs, "hidden": hidden, "dtype": dtype, "act": act, "pad": pad}

    def adamw(name, tensors, smallest, largest, param, grad, bits, copy, step):
        return {"name": name, "op": "adamw", "tensors": tensors, "smallest": smallest, "largest": largest, "param": param,
                "grad": grad, "bits": bits, "copy": copy, "step": step}

    return [
        # one record of a serving loop: the 16 fields and 8 crosses of the repository's smallest workload
        embed("embed_request", 1, 24, 0, 100_003, 16, "float32", vocab=100_000),
        # a step's batch of the list-heavy workload: 48 lists, 16 single fields and 32 crosses, mean pooling
        embed("embed_lists", 16_384, 16, 80, 2_000_003, 16, "bfloat16", mean=True),
        # a large batch of the widest workload (88 + 8 single fields, 60 single crosses, 4 lists and 4 crosses with them)
        embed("embed_wide", 65_536, 156, 8, 10_000_000, 16, "bfloat16", mean_items=5.0, vocab=100_000_000),
        # the table's gradient for the smallest workload's batch
        embed("embed_grad_small", 4_096, 24, 0, 100_003, 16, "float32", vocab=100_000, op="embed_grad"),
        # and for the wide workload's: twelve million signs, hot rows among them
        embed("embed_grad_wide", 65_536, 156, 8, 10_000_000, 16, "bfloat16", mean_items=5.0, vocab=100_000_000, op="embed_grad"),
        # one record through the block that follows the list-heavy workload's pooled rows (96 slots of 16)
        gated("gated_request", 1, 1_536, 4_096, "bfloat16"),
        # a large batch of the wide workload (164 slots of 16) through its block
        gated("gated_wide", 65_536, 2_624, 4_096, "bfloat16"),
        # the gradient at sizes that are a multiple of nothing, with half precision's types
        gated("gated_grad_odd", 1_000, 411, 773, "float16", act="gelu", pad=3, op="gated_grad"),
        # a step of the smallest workload's block with 32-bit weights
        gated("gated_grad_single", 4_096, 384, 1_024, "float32", op="gated_grad"),
        # a step's batch of the wide workload
        gated("gated_grad_wide", 16_384, 2_624, 4_096, "bfloat16", op="gated_grad"),
        # the dense part of a small model: many tensors of a few elements to some hundred thousand
        adamw("adamw_dense", 48, 1, 400_000, "float32", "float32", 32, False, 10),
        # a table of ten million rows of 16 and its model, states in 8 bits
        adamw("adamw_table", 8, 1_001, 160_000_000, "float32", "bfloat16", 8, True, 1000),
    ]


MOST_PRODUCT = 65_536 * 2_624 * 4_096   # records x inputs x hidden of the largest listed block; a gradient is a third of it
MOST_SIGNS = 65_536 * 200
MOST_ELEMENTS = 160_000_000
ODD_ONE_OUT = 3072                      # a size that no case of this repository has


def _log(rng, low, high):
    n = round(low * (high / low) ** rng.random())
    return max(low, min(high, n))


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "gated", "gated_grad", "adamw"])
    if op.startswith("embed"):
        while True:
            records, single, ragged = _log(rng, 1, 65_536), rng.randint(0, 156), rng.choice([0, rng.randint(1, 8), rng.randint(1, 80)])
            items, dim, rows = round(rng.uniform(0.0, 6.0), 2), rng.choice([1, 4, 8, 12, 16, 16, 17, 24, 32, 50, 64, 128]), _log(rng, 100, 10_000_000)
            slots = single + ragged
            signs = records * (single + ragged * (items + 0.5))
            fits = 1 <= slots and signs * dim <= MOST_SIGNS * 16 and signs <= MOST_SIGNS and records * slots * dim <= MOST_SIGNS * 16 and rows * dim <= MOST_ELEMENTS
            if fits and ODD_ONE_OUT not in (slots * dim, records, rows):
                return {"op": op, "records": records, "single": single, "ragged": ragged, "mean_items": items, "vocab": _log(rng, 1000, 100_000_000),
                        "rows": rows, "dim": dim, "dtype": rng.choice(["float32", "bfloat16", "float16"]), "mean": rng.random() < 0.4}
    if op.startswith("gated"):
        while True:
            records, inputs, hidden = _log(rng, 1, 65_536), _log(rng, 8, 4_096), _log(rng, 16, 8_192)
            if rng.random() < 0.6:  # (widths are slots x dim and round numbers more often than not)
                inputs, hidden = -(-inputs // 16) * 16, -(-hidden // 64) * 64
            dtype = rng.choice(["bfloat16", "bfloat16", "float16", "float32"])
            most = MOST_PRODUCT // (3 if op == "gated_grad" else 1) // (8 if dtype == "float32" else 1)
            if records * inputs * hidden <= most and ODD_ONE_OUT not in (records, inputs, hidden):
                return {"op": op, "records": records, "inputs": inputs, "hidden": hidden, "dtype": dtype,
                        "act": rng.choice(["silu", "gelu", "relu", "sigmoid"]), "pad": rng.choice([0, 0, 0, 8, rng.randint(1, 40)])}
    param = rng.choice(["float32", "float32", "bfloat16", "float16"])
    while True:
        case = {"op": op, "tensors": _log(rng, 1, 200), "smallest": _log(rng, 1, 5000), "largest": _log(rng, 5000, 100_000_000), "param": param,
                "grad": param if param != "float32" else rng.choice(["float32", "bfloat16", "float16"]), "bits": rng.choice([32, 8]),
                "copy": param == "float32" and rng.random() < 0.3, "step": rng.randint(1, 10_000)}
        if sum(_sizes(case)) <= MOST_ELEMENTS and ODD_ONE_OUT not in _sizes(case):
            return case


# ------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 2 + 1)
    return g


def _dtype(name):
    return {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}[name]


def _signed(x):
    """A 64-bit constant as torch's signed integers have it."""
    x &= U64
    return x - (1 << 64) if x >> 63 else x


def _shr(x, n):
    """Logical shift to the right of 64-bit integers."""
    return (x >> n) & ((1 << (64 - n)) - 1)


def _mix64(x):
    x = (x ^ _shr(x, 30)) * _signed(0xBF58476D1CE4E5B9)
    x = (x ^ _shr(x, 27)) * _signed(0x94D049BB133111EB)
    return x ^ _shr(x, 31)


def _mix64_int(x):
    x &= U64
    x = ((x ^ (x >> 30)) * 0xBF58476D1CE4E5B9) & U64
    x = ((x ^ (x >> 27)) * 0x94D049BB133111EB) & U64
    return x ^ (x >> 31)


def _slots(case, g):
    """[(values, offsets or None)], as extraction leaves them: signs in record order, offsets for lists."""
    n, slots = case["records"], []

    def signs(count, salt):  # ranks with probability ~ 1 / rank, then 64 mixed bits
        u = torch.rand(count, device="cuda", generator=g, dtype=torch.float64)
        return _mix64(torch.floor(float(case["vocab"]) ** u).to(torch.int64) + salt)

    k = case["single"]
    flat = signs(k * n, 0).view(k, n)
    flat = _mix64(flat + torch.arange(1, k + 1, device="cuda").view(-1, 1))
    slots += [(flat[i], None) for i in range(k)]
    k = case["ragged"]
    if k:
        lens = torch.poisson(torch.full((k, n), float(case["mean_items"]), device="cuda"), generator=g).to(torch.int64)
        lens[::2] += 1
        offsets = torch.zeros(k, n + 1, dtype=torch.int64, device="cuda")
        offsets[:, 1:] = torch.cumsum(lens, 1)
        totals = offsets[:, -1].tolist()
        flat = signs(sum(totals), 1 << 40)
        salt = torch.repeat_interleave(torch.arange(1000, 1000 + k, device="cuda"), offsets[:, -1])
        flat = _mix64(flat + salt)
        at = 0
        for i in range(k):
            slots.append((flat[at:at + totals[i]], offsets[i]))
            at += totals[i]
    return slots


def _sizes(case):
    """Elements of the tensors: the smallest, the largest, and others spread between them."""
    rng = random.Random("%d %d %d" % (case["tensors"], case["smallest"], case["largest"]))
    low, high = case["smallest"], case["largest"]
    return [high] + [low] * (case["tensors"] > 1) + [_log(rng, low, max(low, high // 8)) for _ in range(case["tensors"] - 2)]


def _cut(flat, sizes, every=1):
    """Views of a flat buffer, one for each size, that begin at multiples of 16 elements."""
    views, at = [], 0
    for n in sizes:
        n = -(-n // every)
        views.append(flat[at:at + n])
        at += -(-n // 16) * 16
    return views


def _room(sizes, every=1):
    return sum(-(-(-(-n // every)) // 16) * 16 for n in sizes)


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case}
    if case["op"].startswith("embed"):
        dtype = _dtype(case["dtype"])
        s["slots"] = _slots(case, g)
        if case["op"] == "embed":
            s["table"] = (torch.randn(case["rows"], case["dim"], device="cuda", generator=g, dtype=torch.float32) * 0.05).to(dtype)
        else:
            s["dout"] = torch.randn(case["records"], case["single"] + case["ragged"], case["dim"], device="cuda", generator=g, dtype=torch.float32).to(dtype)
    elif case["op"].startswith("gated"):
        dtype, m, k, n = _dtype(case["dtype"]), case["records"], case["inputs"], case["hidden"]
        r = lambda a, b, scale: (torch.randn(a, b, device="cuda", generator=g, dtype=torch.float32) * scale).to(dtype)  # noqa: E731
        s["x"] = r(m, k + case["pad"], 1.0)[:, :k]
        s["w_gate"], s["w_up"] = r(n, k, 1 / math.sqrt(k)), r(n, k, 1 / math.sqrt(k))
        if case["op"] == "gated_grad":
            s["dh"] = r(m, n, 1.0)
    else:
        sizes, room = _sizes(case), _room(_sizes(case))
        r = lambda n, scale: torch.randn(n, device="cuda", generator=g, dtype=torch.float32) * scale  # noqa: E731
        s["param"] = r(room, 0.05).to(_dtype(case["param"]))
        s["grad"] = r(room, 0.02).to(_dtype(case["grad"]))
        m, v = r(room, 0.005), r(room, 0.01).square()
        if case["bits"] == 8:
            scales = _room(sizes, BLOCK)
            half = torch.full((1,), 32768, dtype=torch.int64, device="cuda")
            for name, x in (("m", m), ("v", v.sqrt())):
                codes = torch.zeros(room, dtype=torch.uint8, device="cuda")
                scale = torch.ones(scales, dtype=torch.uint8, device="cuda")
                for c, sc, one in zip(_cut(codes, sizes), _cut(scale, sizes, BLOCK), _cut(x, sizes)):
                    a, b = _encode(one, half)
                    c.copy_(a)
                    sc.copy_(b)
                s[name], s[name + "_scale"] = codes.view(torch.float8_e4m3fn), scale.view(torch.float8_e8m0fnu)
        else:
            s["m"], s["v"] = m, v
        if case["copy"]:
            s["copy"] = torch.zeros(room, dtype=torch.bfloat16, device="cuda")
        s["views"] = {k: _cut(x, sizes, BLOCK if k.endswith("scale") else 1) for k, x in s.items() if isinstance(x, torch.Tensor)}
        s["seed"] = int(seed) % (1 << 31)
    return s


LR, BETA1, BETA2, EPS, DECAY, GRAD_SCALE = 1e-3, 0.9, 0.999, 1e-8, 0.01, 0.5


# ------------------------------------------------------------------ plain forms
def _rows(values, rows):
    """floor(mix64(sign) x rows / 2^64)."""
    x = _mix64(values)
    high, low = _shr(x, 32), x & 0xFFFFFFFF
    return (high * rows + ((low * rows) >> 32)) >> 32


def _flat(slots, n):
    """All signs of all slots, the (slot, record) that each belongs to, and how many each of those has."""
    values = torch.cat([v for v, _ in slots])
    lens = torch.cat([torch.ones_like(v) if o is None else o[1:] - o[:-1] for v, o in slots])
    return values, torch.repeat_interleave(torch.arange(lens.numel(), device=lens.device), lens, output_size=values.numel()), lens


def _embed(s):
    case = s["case"]
    values, bag, lens = _flat(s["slots"], case["records"])
    out = torch.zeros(lens.numel(), case["dim"], device="cuda")
    out.index_add_(0, bag, s["table"][_rows(values, case["rows"])].float())
    if case["mean"]:
        out = out / lens.clamp(min=1).unsqueeze(1)
    return out.view(len(s["slots"]), case["records"], case["dim"]).transpose(0, 1).to(s["table"].dtype, memory_format=torch.contiguous_format)


def _embed_grad(s):
    case = s["case"]
    values, bag, lens = _flat(s["slots"], case["records"])
    d = s["dout"].transpose(0, 1).reshape(lens.numel(), case["dim"]).float()
    if case["mean"]:
        d = d / lens.clamp(min=1).unsqueeze(1)
    out = torch.zeros(case["rows"], case["dim"], device="cuda")
    return out.index_add_(0, _rows(values, case["rows"]), d[bag]).to(s["dout"].dtype)


def _phi(a):
    return 0.5 * (1 + torch.erf(a * math.sqrt(0.5)))


def _act(a, act):
    if act == "silu":
        return a * torch.sigmoid(a)
    if act == "gelu":
        return a * _phi(a)
    return a.clamp(min=0) if act == "relu" else torch.sigmoid(a)


def _act_grad(a, act):
    if act == "silu":
        t = torch.sigmoid(a)
        return t * (1 + a * (1 - t))
    if act == "gelu":
        return _phi(a) + a * torch.exp(-0.5 * a * a) * (1 / math.sqrt(2 * math.pi))
    if act == "relu":
        return (a > 0).to(a.dtype)
    t = torch.sigmoid(a)
    return t * (1 - t)


def _gated(s):
    x, wg, wu = s["x"].float(), s["w_gate"].float(), s["w_up"].float()
    return (_act(x @ wg.t(), s["case"]["act"]) * (x @ wu.t())).to(s["x"].dtype)


def _gated_grad(s):
    x, wg, wu, dh, act = s["x"].float(), s["w_gate"].float(), s["w_up"].float(), s["dh"].float(), s["case"]["act"]
    a, u = x @ wg.t(), x @ wu.t()
    du = dh * _act(a, act)
    da = dh * u * _act_grad(a, act)
    return {"dx": (da @ wg + du @ wu).to(s["x"].dtype), "dw_gate": (da.t() @ x).to(s["x"].dtype), "dw_up": (du.t() @ x).to(s["x"].dtype)}


def _blocks(x):
    return torch.nn.functional.pad(x, (0, -x.numel() % BLOCK)).view(-1, BLOCK)


def _decode(codes, scale):
    return (_blocks(codes.float()) * scale.float().unsqueeze(1)).view(-1)[:codes.numel()]


def _encode(x, random16):
    """x in 8 bits (4 of exponent, 3 of mantissa) and a power of two for every 32 elements, which puts the largest of
    them into [128, 256); rounded up where the 16 random bits, as a fraction, say so."""
    b = _blocks(x)
    e = (b.abs().amax(1).view(torch.int32) >> 23) & 255
    scale = torch.where(e == 255, 255, (e - 7).clamp(min=1))
    y = (b * ((254 - scale.clamp(max=247)) << 23).view(torch.float32).unsqueeze(1)).view(-1)[:x.numel()]
    a = y.abs()
    ee = (((a.view(torch.int32) >> 23) & 255) - 127).clamp(min=-6)
    t = a * ((130 - ee) << 23).view(torch.float32)
    q = torch.floor(t + random16.float() * (1 / 65536))
    code = torch.where(q == q, q, 0).to(torch.int32) + ((ee + 6) << 3) + ((y < 0).to(torch.int32) << 7)
    bad = (scale == 255).unsqueeze(1).expand(-1, BLOCK).reshape(-1)[:x.numel()]
    return torch.where(bad, 127, code).to(torch.uint8), scale.to(torch.uint8)


def _adamw_one(s, t):
    """One tensor's step, in place."""
    case, x = s["case"], {k: v[t] for k, v in s["views"].items()}
    n, step = x["param"].numel(), case["step"]
    p, g = x["param"].float(), x["grad"].float() * GRAD_SCALE
    eight = case["bits"] == 8
    m, v = (_decode(x["m"], x["m_scale"]), _decode(x["v"], x["v_scale"]).square()) if eight else (x["m"], x["v"])
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + (g * g) * (1 - BETA2)
    root = v.sqrt()
    p = p * (1 - LR * DECAY) - (m / (root * (1 / math.sqrt(1 - BETA2 ** step)) + EPS)) * (LR / (1 - BETA1 ** step))
    x["param"].copy_(p)
    if case["copy"]:
        x["copy"].copy_(p)
    if eight:
        at = torch.arange(n, device="cuda")
        bits = _mix64((at >> 1) + _signed(_mix64_int(_mix64_int(s["seed"] + step) + t))) >> ((at & 1) << 5)
        for name, value, shift in (("m", m, 0), ("v", root, 16)):
            codes, scale = _encode(value, (bits >> shift) & 0xFFFF)
            x[name].view(torch.uint8).copy_(codes)
            x[name + "_scale"].view(torch.uint8).copy_(scale)
    else:
        x["m"].copy_(m)
        x["v"].copy_(v)


def _adamw(s):
    [_adamw_one(s, t) for t in range(s["case"]["tensors"])]
    return {k: s[k] for k in s["views"] if k != "grad"}


PLAIN = {"embed": _embed, "embed_grad": _embed_grad, "gated": _gated, "gated_grad": _gated_grad, "adamw": _adamw}


# ------------------------------------------------------------------ the framework's operators
def _own(s):
    from paper_2210_07768_amd import train as T

    case = s["case"]
    if case["op"] == "embed":
        return T.embed([T.Signs(v, o) for v, o in s["slots"]], s["table"], case["records"], mean=case["mean"])
    if case["op"] == "embed_grad":
        return T.embed_backward(s["dout"], [T.Signs(v, o) for v, o in s["slots"]], case["rows"], mean=case["mean"])
    if case["op"] == "gated":
        return T.gated(s["x"], s["w_gate"], s["w_up"], act=case["act"])
    if case["op"] == "gated_grad":
        dx, dw_gate, dw_up = T.gated_backward(s["dh"], s["x"], s["w_gate"], s["w_up"], act=case["act"])
        return {"dx": dx, "dw_gate": dw_gate, "dw_up": dw_up}
    x = s["views"]
    T.adamw(x["param"], x["grad"], x["m"], x["v"], x.get("m_scale"), x.get("v_scale"), x.get("copy"), step=case["step"], lr=LR, betas=(BETA1, BETA2),
            eps=EPS, weight_decay=DECAY, grad_scale=GRAD_SCALE, seed=s["seed"])
    return {k: s[k] for k in x if k != "grad"}


def run(state):
    return _own(state) if own else PLAIN[state["case"]["op"]](state)


# ------------------------------------------------------------------ what a pass cannot do without
def _distinct(count, vocab):
    """Expected distinct tokens among `count` of a slot, with probability ~ 1 / rank over `vocab` ranks."""
    if count <= 0:
        return 0.0
    steps, total, h = 400, 0.0, math.log(vocab + 1)
    for i in range(steps):
        low, high = math.exp(h * i / steps), math.exp(h * (i + 1) / steps)
        p = 1 / (h * 0.5 * (low + high))
        total += (high - low) * -math.expm1(-count * p)
    return min(total, count)


def work(case):
    size = {"float32": 4, "bfloat16": 2, "float16": 2}
    if case["op"].startswith("embed"):
        n, e = case["records"], size[case["dtype"]]
        items = case["mean_items"] + 0.5
        signs = n * (case["single"] + case["ragged"] * items)
        inputs = 8 * signs + 8 * (n + 1) * case["ragged"]
        pooled = n * (case["single"] + case["ragged"]) * case["dim"] * e
        if case["op"] == "embed_grad":
            return {"bytes": inputs + pooled + case["rows"] * case["dim"] * e, "flops": signs * case["dim"]}
        tokens = case["single"] * _distinct(n, case["vocab"]) + case["ragged"] * _distinct(n * items, case["vocab"])
        touched = case["rows"] * -math.expm1(-tokens / case["rows"])
        return {"bytes": inputs + touched * case["dim"] * e + pooled, "flops": signs * case["dim"]}
    if case["op"].startswith("gated"):
        m, k, n, e = case["records"], case["inputs"], case["hidden"], size[case["dtype"]]
        if case["op"] == "gated":
            return {"bytes": e * (m * k + 2 * n * k + m * n), "flops": 4 * m * k * n}
        return {"bytes": e * (2 * m * k + 4 * n * k + m * n), "flops": 12 * m * k * n}
    sizes = _sizes(case)
    n, blocks = sum(sizes), sum(-(-x // BLOCK) for x in sizes)
    state = 16 * n if case["bits"] == 32 else 4 * n + 4 * blocks
    return {"bytes": n * (2 * size[case["param"]] + size[case["grad"]] + (2 if case["copy"] else 0)) + state, "flops": 15 * n}


# ------------------------------------------------------------------ the definitions, in 64 bits
def _exact_rows(values, rows):
    """The rows of signs by numpy's unsigned integers."""
    import numpy as np

    x = values.cpu().numpy().view(np.uint64)
    x = (x ^ (x >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
    x = (x ^ (x >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
    x = x ^ (x >> np.uint64(31))
    v = np.uint64(rows)
    carry = ((x & np.uint64(0xFFFFFFFF)) * v) >> np.uint64(32)
    return torch.from_numpy((((x >> np.uint64(32)) * v + carry) >> np.uint64(32)).astype(np.int64)).cuda()


def _exact_embed(case, s):
    n, backward = case["records"], case["op"] == "embed_grad"
    out = torch.zeros((case["rows"], case["dim"]) if backward else (n, len(s["slots"]), case["dim"]), dtype=torch.float64, device="cuda")
    for i, (values, offsets) in enumerate(s["slots"]):
        rows = _exact_rows(values, case["rows"])
        if offsets is None:
            record, share = torch.arange(n, device="cuda"), torch.ones(n, dtype=torch.float64, device="cuda")
        else:
            record = torch.searchsorted(offsets, torch.arange(values.numel(), device="cuda"), right=True) - 1
            share = 1 / (offsets[1:] - offsets[:-1]).double() if case["mean"] else torch.ones(n, dtype=torch.float64, device="cuda")
        if backward:
            out.index_add_(0, rows, s["dout"][:, i].double()[record] * share[record].unsqueeze(1))
        else:
            part = torch.zeros(n, case["dim"], dtype=torch.float64, device="cuda")
            out[:, i] = part.index_add_(0, record, s["table"][rows].double() * share[record].unsqueeze(1))
    return out


def _exact_gated(case, s):
    x, wg, wu = s["x"].double(), s["w_gate"].double(), s["w_up"].double()
    a, u = torch.nn.functional.linear(x, wg), torch.nn.functional.linear(x, wu)
    logistic, bell = 1 / (1 + torch.exp(-a)), torch.exp(a * a / -2) / math.sqrt(2 * math.pi)
    below = torch.special.ndtr(a)
    act = {"silu": a * logistic, "gelu": a * below, "relu": torch.where(a > 0, a, 0.0), "sigmoid": logistic}[case["act"]]
    if case["op"] == "gated":
        return act * u
    slope = {"silu": logistic + a * logistic * (1 - logistic), "gelu": below + a * bell, "relu": torch.where(a > 0, 1.0, 0.0),
             "sigmoid": logistic * (1 - logistic)}[case["act"]]
    dh = s["dh"].double()
    del logistic, bell, below
    da, du = dh * u * slope, dh * act
    return {"dx": torch.mm(da, wg) + torch.mm(du, wu), "dw_gate": torch.mm(da.t(), x), "dw_up": torch.mm(du.t(), x)}


def _exact_adamw(case, s):
    """Weights and states; of states in 8 bits what is rounded to them, in units of the scale, and the scale."""
    sizes, eight = _sizes(case), case["bits"] == 8
    out = {k: v.double().clone() for k, v in s.items() if isinstance(v, torch.Tensor) and k != "grad"}
    views = {k: _cut(v, sizes, BLOCK if k.endswith("scale") else 1) for k, v in out.items()}
    for t, grad in enumerate(_cut(s["grad"], sizes)):
        x = {k: v[t] for k, v in views.items()}
        n, g = grad.numel(), grad.double() * GRAD_SCALE
        wide = lambda scale: scale.repeat_interleave(BLOCK)[:n]  # noqa: E731
        m, v = (x["m"] * wide(x["m_scale"]), (x["v"] * wide(x["v_scale"])) ** 2) if eight else (x["m"].clone(), x["v"].clone())
        m, v = BETA1 * m + (1 - BETA1) * g, BETA2 * v + (1 - BETA2) * g ** 2
        mean, spread = m / (1 - BETA1 ** case["step"]), v / (1 - BETA2 ** case["step"])
        x["param"].copy_(x["param"] - LR * DECAY * x["param"] - LR * mean / (spread.sqrt() + EPS))
        if case["copy"]:
            x["copy"].copy_(x["param"])
        if eight:
            for name, y in (("m", m), ("v", v.sqrt())):
                top = torch.nn.functional.pad(y.abs(), (0, -n % BLOCK)).view(-1, BLOCK).amax(1)
                scale = torch.exp2((torch.floor(torch.log2(top)) - 7).clamp(min=-126))
                x[name + "_scale"].copy_(scale)
                x[name].copy_(y / wide(scale))
        else:
            x["m"].copy_(m)
            x["v"].copy_(v)
    return {k: out[k] for k in s["views"] if k != "grad"}


def exact(case, seed):
    s = prepare(case, seed)
    return {"embed": _exact_embed, "gated": _exact_gated, "adamw": _exact_adamw}[case["op"].split("_")[0]](case, s)
