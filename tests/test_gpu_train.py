"""The trainer's operators on the GPU against their definitions in 64 bits.

Tolerances are bounds on the error of what the header promises, worked out per element from the same inputs: a sum of n
terms held in 32 bits is off by at most n 2^-24 times the sum of its terms' magnitudes, whatever its order; a stored result by
half a unit of its type; an activation by its slope times what its argument is off.  States in 8 bits, and all that
decides about them, are compared bit for bit with the same arithmetic in numpy."""
import math

import numpy as np
import pytest
import torch

from paper_2210_07768_amd import binding as B
from paper_2210_07768_amd import train as T

pytestmark = pytest.mark.gpu
U32 = 2.0 ** -24
HALF_UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -133}   # half of the smallest step, and more
TYPES = [torch.float32, torch.float16, torch.bfloat16]


def _close(got, want, bound, what):
    """|got - want| <= bound, plus rounding to got's type."""
    dtype = got.dtype
    got, want, bound = got.double().to(want.device), want.double(), bound.double().to(want.device)
    limit = bound + HALF_UNIT[dtype] * (want.abs() + bound) + TINY[dtype]
    off = (got - want).abs()
    assert torch.isfinite(got).all(), f"{what}: not finite"
    bad = off > limit
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((off / limit).max()):.3g} times the bound"


# ------------------------------------------------------------------ embed
def _rows_of(values, rows):
    x = values.astype(np.uint64)
    with np.errstate(over="ignore"):
        x = (x ^ (x >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        x = (x ^ (x >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
    x = x ^ (x >> np.uint64(31))
    return np.array([(int(v) * rows) >> 64 for v in x], dtype=np.int64)


def _make_slots(rng, n, spec, distinct):
    """spec: a number (fixed arity) or 'list' / 'long' / 'empty' for each slot; signs from a pool of `distinct`."""
    pool = rng.integers(0, 1 << 64, size=distinct, dtype=np.uint64)
    out = []
    for kind in spec:
        if isinstance(kind, int):
            out.append((pool[(rng.random(n * kind) ** 3 * distinct).astype(int)], None, kind))
        else:
            lens = {"list": rng.integers(0, 6, n), "long": np.where(np.arange(n) == n // 2, 5000, rng.integers(0, 2, n)), "empty": np.zeros(n, int)}[kind]
            o = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
            out.append((pool[(rng.random(int(o[-1])) ** 3 * distinct).astype(int)], o, 0))
    return out


def _on_gpu(slots):
    return [T.Signs(torch.from_numpy(v.view(np.int64)).cuda(), None if o is None else torch.from_numpy(o).cuda(), a) for v, o, a in slots]


def _owners(slots, n):
    """Per slot, the record of every sign and the signs of every record."""
    for v, o, a in slots:
        lens = np.full(n, a, np.int64) if o is None else np.diff(o)
        yield np.repeat(np.arange(n), lens), lens


def _embed_want(slots, n, table, mean):
    rows, dim = table.shape
    out, size = np.zeros((n, len(slots), dim)), np.zeros((n, len(slots), dim))
    for i, ((v, _, _), (owner, lens)) in enumerate(zip(slots, _owners(slots, n))):
        t = table[_rows_of(v, rows)]
        np.add.at(out[:, i], owner, t)
        np.add.at(size[:, i], owner, np.abs(t))
        w = 1 / np.maximum(lens, 1)[:, None] if mean else 1.0
        out[:, i] *= w
        size[:, i] *= w * (np.maximum(lens, 1)[:, None] + 2) * U32
    return torch.from_numpy(out), torch.from_numpy(size)


CASES = [  # records, slots, dim, rows, distinct signs
    (1, [1], 1, 1, 3), (1, [1, 1, 1], 16, 1000, 50), (5, ["empty", 1, "empty"], 8, 10, 4), (33, [1, "list", 3, "list"], 16, 300, 1000),
    (64, ["list"] * 65, 4, 77, 500), (129, [1] * 130, 2, 1001, 3000), (257, ["long", 2], 33, 100, 90), (100, [1, "list"], 300, 64, 1000),
    (1000, [1, "list", 1], 24, 5, 40), (3000, ["list", "long", 1, 1], 12, 4099, 100_000), (31, [2, "list"], 1030, 50, 60),
    (40, [1, "list"] * 100 + [2], 8, 1009, 3000),
]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("mean", [False, True])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_embed_forward(case, mean, dtype):
    n, spec, dim, rows, distinct = CASES[case]
    rng = np.random.default_rng(case)
    slots = _make_slots(rng, n, spec, distinct)
    table = torch.from_numpy(rng.standard_normal((rows, dim))).to(dtype)
    got = T.embed(_on_gpu(slots), table.cuda(), n, mean=mean)
    assert got.shape == (n, len(spec), dim) and got.dtype == dtype
    want, bound = _embed_want(slots, n, table.double().numpy(), mean)
    _close(got, want, bound, "embed")
    for i, (_, lens) in enumerate(_owners(slots, n)):   # nothing pooled: exactly zero; a single sign: its row, exactly
        assert not got[torch.from_numpy(lens == 0).cuda(), i].any()
        one = np.flatnonzero(lens == 1)
        first = np.concatenate([[0], np.cumsum(lens)])[one]
        assert torch.equal(got[torch.from_numpy(one).cuda(), i].cpu(), table[torch.from_numpy(_rows_of(slots[i][0], rows)[first])])


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("mean", [False, True])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_embed_backward(case, mean, dtype):
    n, spec, dim, rows, distinct = CASES[case]
    rng = np.random.default_rng(100 + case)
    slots = _make_slots(rng, n, spec, distinct)
    dout = torch.from_numpy(rng.standard_normal((n, len(spec), dim))).to(dtype)
    got = T.embed_backward(dout.cuda(), _on_gpu(slots), rows, mean=mean)
    want, size, terms = np.zeros((rows, dim)), np.zeros((rows, dim)), np.zeros((rows, 1))
    d = dout.double().numpy()
    for i, ((v, _, _), (owner, lens)) in enumerate(zip(slots, _owners(slots, n))):
        at, w = _rows_of(v, rows), (1 / np.maximum(lens, 1) if mean else np.ones(n))[owner][:, None]
        np.add.at(want, at, d[owner, i] * w)
        np.add.at(size, at, np.abs(d[owner, i] * w))
        np.add.at(terms, at, 1.0)
    _close(got, torch.from_numpy(want), torch.from_numpy(size * (terms + 4) * U32), "embed_backward")
    assert not got[torch.from_numpy(terms[:, 0] == 0).cuda()].any()
    again = T.embed_backward(dout.cuda(), _on_gpu(slots), rows, mean=mean)
    assert torch.equal(got.view(torch.uint8), again.view(torch.uint8)), "the same inputs give the same bits"


@pytest.mark.parametrize("signs", [31, 32, 33, 63, 64, 65, 1023, 1024, 1025, 4095, 4096, 4097, 70_000])
@pytest.mark.parametrize("rows", [1, 2, 256, 257, 70_000])
def test_embed_backward_runs(signs, rows):
    """One row's terms over many stretches, rows with one term each, and what lies between; sums of whole numbers are exact."""
    rng = np.random.default_rng(signs * 7 + rows)
    v = rng.integers(0, 1 << 64, size=signs, dtype=np.uint64)
    v[: signs // 2] = v[0]
    dout = torch.from_numpy(rng.integers(-8, 9, (signs, 1, 4)).astype(np.float32)).cuda()
    got = T.embed_backward(dout, _on_gpu([(v, None, 1)]), rows)
    want = np.zeros((rows, 4))
    np.add.at(want, _rows_of(v, rows), dout[:, 0].double().cpu().numpy())
    assert np.array_equal(got.double().cpu().numpy(), want)


@pytest.mark.parametrize("distinct", [1, 60, 3000, 1 << 20])
@pytest.mark.parametrize("dim, pad, rows", [(4, 0, 540_000), (1, 2, 300_001), (16, 4, 270_011), (300, 0, 400_000), (300, 5, 540_001)])
def test_embed_backward_many(dim, pad, rows, distinct):
    """More pairs than half the rows, from rows that nearly all have terms to one row that has them all; sums of whole numbers
    are exact, rows without terms are zero, and nothing is written beside them."""
    n = 90_007
    rng = np.random.default_rng(dim + distinct)
    slots = _make_slots(rng, n, [1, 1, 1], distinct)
    g = torch.Generator(device="cuda").manual_seed(distinct)
    dout = torch.randint(-8, 9, (n, 3, dim), device="cuda", generator=g).float()
    room = torch.full((rows, dim + pad), 7.0, device="cuda")
    T.embed_backward(dout, _on_gpu(slots), rows, out=room[:, :dim])
    want = torch.zeros(rows, dim, device="cuda")
    for i, (v, _, _) in enumerate(slots):
        want.index_add_(0, torch.from_numpy(_rows_of(v, rows)).cuda(), dout[:, i])
    assert torch.equal(room[:, :dim], want) and bool((room[:, dim:] == 7.0).all())


def test_embed_strides_and_outputs():
    rng = np.random.default_rng(5)
    slots = _make_slots(rng, 50, [1, "list", 2], 200)
    for pad, off in ((0, 0), (8, 0), (3, 1), (1, 3)):
        base = torch.from_numpy(rng.standard_normal((100, 16 + pad)).astype(np.float32)).cuda()
        table = base[:, :16]
        room = torch.full((50 * (48 + pad) + 8,), 7.0, device="cuda")
        out = room[off:off + 50 * (48 + pad)].view(50, 48 + pad)[:, :48].unflatten(1, (3, 16))
        T.embed(_on_gpu(slots), table, 50, out=out)
        assert torch.equal(out, T.embed(_on_gpu(slots), table.contiguous(), 50))
        assert int((room == 7.0).sum()) >= room.numel() - 50 * 48, "written outside its rows"
        grads = torch.full((100, 16 + pad), 7.0, device="cuda")
        T.embed_backward(out, _on_gpu(slots), 100, out=grads[:, :16])
        assert torch.equal(grads[:, :16], T.embed_backward(out.contiguous(), _on_gpu(slots), 100)) and bool((grads[:, 16:] == 7.0).all())


def test_embed_table_beyond_32_bits():
    """Rows whose elements lie beyond 2^32, and the gradient's."""
    rows, dim, n = 17_000_001, 256, 500
    rng = np.random.default_rng(6)
    slots = _make_slots(rng, n, [1], 5000)
    at = torch.from_numpy(_rows_of(slots[0][0], rows))
    assert int(at.max()) * dim > 1 << 32
    table = torch.zeros(rows, dim, dtype=torch.bfloat16, device="cuda")
    want = torch.randn(n, dim).to(torch.bfloat16)
    table[at.cuda()] = want.cuda()
    assert torch.equal(T.embed(_on_gpu(slots), table, n)[:, 0], table[at.cuda()])
    dout = torch.ones(n, 1, dim, dtype=torch.bfloat16, device="cuda")
    T.embed_backward(dout, _on_gpu(slots), rows, out=table)
    count = torch.zeros(rows).index_add_(0, at, torch.ones(n)).cuda()
    for r0 in range(0, rows, 1 << 21):
        assert torch.equal(table[r0:r0 + (1 << 21)].sum(1, dtype=torch.float32), count[r0:r0 + (1 << 21)] * dim)


@pytest.mark.parametrize("placement, tile_log2", [(0, -1), (1, -1), (1, 2), (1, 0)])
def test_embed_takes_extraction_results(placement, tile_log2):
    """What extraction returns, in record order and in arrival order: every list pools to the same."""
    from paper_2210_07768_amd import workloads as W

    w = W.get(5, 3000)
    raw, off = w.generate()
    d_raw, d_off = torch.from_numpy(raw.copy()).cuda(), torch.from_numpy(off.astype(np.int64)).cuda()
    plan = B.Plan(w.spec)
    res, ws = B.extract_with_retry(plan, d_raw, d_off)
    table = torch.randint(-50, 50, (5003, 8), device="cuda").float()   # (whole numbers: sums do not depend on order)
    want = T.embed(res, table)
    signs = [res.slots[i] for i in res.slot_ids]
    assert torch.equal(want, T.embed(signs, table, res.n_records))
    want_grad = T.embed_backward(want, res, 5003)
    if placement:
        plan.set_option("placement", 1)
        plan.set_option("tile_log2", tile_log2)
        for _ in range(2):
            res = plan.extract(d_raw, d_off)
        assert res.arrival_tile_records
        assert torch.equal(T.embed(res, table), want)
        assert torch.equal(T.embed_backward(want, res, 5003), want_grad)
    plan.close()


def test_embed_special_values_stay_in_their_rows():
    table = torch.zeros(8, 4, device="cuda")
    values = np.arange(1, 200, dtype=np.uint64)
    at = _rows_of(values, 8)
    table[3] = float("nan")
    table[5] = float("inf")
    got = T.embed(_on_gpu([(values, None, 1)]), table, 199)[:, 0]
    assert torch.equal(torch.isnan(got[:, 0]).cpu(), torch.from_numpy(at == 3)) and torch.equal(torch.isinf(got[:, 0]).cpu(), torch.from_numpy(at == 5))
    dout = torch.ones(199, 1, 4, device="cuda")
    dout[np.flatnonzero(at == 2)[0]] = float("nan")
    grad = T.embed_backward(dout, _on_gpu([(values, None, 1)]), 8)
    assert torch.isnan(grad[2]).all() and torch.isfinite(grad[[0, 1, 3, 4, 5, 6, 7]]).all()


def test_embed_nothing():
    table = torch.ones(10, 4, device="cuda")
    assert T.embed([], table, 3).shape == (3, 0, 4)
    none = T.Signs(torch.zeros(0, dtype=torch.int64, device="cuda"))
    assert T.embed([none], table, 0).shape == (0, 1, 4)
    assert not T.embed_backward(torch.zeros(0, 1, 4, device="cuda"), [none], 10).any()
    assert not T.embed_backward(torch.zeros(3, 0, 4, device="cuda"), [], 10).any()


# ------------------------------------------------------------------ gated
def _act64(a, act):
    s, phi = torch.sigmoid(a), torch.special.ndtr(a)
    if act == "silu":
        return a * s, s * (1 + a * (1 - s))
    if act == "gelu":
        return a * phi, phi + a * torch.exp(-a * a / 2) / math.sqrt(2 * math.pi)
    return (a.clamp(min=0), (a > 0).double()) if act == "relu" else (s, s * (1 - s))


SLOPE, BEND = {"silu": 1.1, "gelu": 1.13, "relu": 1.0, "sigmoid": 0.25}, {"silu": 0.5, "gelu": 0.8, "relu": 0.0, "sigmoid": 0.1}
# an activation's own arithmetic: a few operations with results up to the larger of 1 and its argument
OWN = 16 * U32


def _projections(x, wg, wu):
    k = x.shape[1]
    a, u = x @ wg.T, x @ wu.T
    return a, u, (k + 1) * U32 * (x.abs() @ wg.abs().T), (k + 1) * U32 * (x.abs() @ wu.abs().T)


def _inputs(m, k, n, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    return (r(m, k) * scale).to(dtype), (r(n, k) / math.sqrt(k)).to(dtype), (r(n, k) / math.sqrt(k)).to(dtype), r(m, n).to(dtype)


def _check_forward(got, x, wg, wu, act, where="cpu"):
    x, wg, wu = (t.double().to(where) for t in (x, wg, wu))
    a, u, ea, eu = _projections(x, wg, wu)
    f, _ = _act64(a, act)
    ef = SLOPE[act] * ea + OWN * a.abs().clamp(min=1)
    _close(got, f * u, ef * u.abs() + f.abs() * eu + ef * eu, "gated")


def _check_backward(got, dh, x, wg, wu, act, where="cpu"):
    dtype, half = x.dtype, HALF_UNIT[x.dtype]
    x, wg, wu, dh = (t.double().to(where) for t in (x, wg, wu, dh))
    a, u, ea, eu = _projections(x, wg, wu)
    f, s = _act64(a, act)
    ef, es = SLOPE[act] * ea + OWN * a.abs().clamp(min=1), BEND[act] * ea + OWN * a.abs().clamp(min=1)
    if act == "relu":
        es = es + (a.abs() <= ea)   # the slope jumps where the argument's sign is in doubt
    da, du = dh * u * s, dh * f
    eda = (1 + half) * dh.abs() * (u.abs() * es + s.abs() * eu + es * eu) + (half + 3 * U32) * da.abs() + TINY[dtype]
    edu = (1 + half) * dh.abs() * ef + (half + 3 * U32) * du.abs() + TINY[dtype]
    m, n = dh.shape
    dx, dwg, dwu = got
    A, G, U, DA, DU = x.abs(), wg.abs(), wu.abs(), da.abs() + eda, du.abs() + edu
    if dx is not None:
        _close(dx, da @ wg + du @ wu, eda @ G + edu @ U + (2 * n + 2) * U32 * (DA @ G + DU @ U), "dx")
    if dwg is not None:
        _close(dwg, da.T @ x, eda.T @ A + (m + 2) * U32 * (DA.T @ A), "dw_gate")
        _close(dwu, du.T @ x, edu.T @ A + (m + 2) * U32 * (DU.T @ A), "dw_up")


SHAPES = [(1, 1, 1), (1, 8, 16), (1, 264, 520), (2, 7, 5), (3, 64, 64), (15, 40, 33), (16, 128, 96), (17, 65, 129), (31, 256, 200), (64, 72, 64), (65, 63, 130), (100, 411, 77),
          (128, 512, 128), (129, 136, 257), (255, 33, 72), (256, 64, 256), (257, 200, 130), (300, 1000, 24), (520, 96, 264), (1030, 48, 40)]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_gated_forward(shape, dtype):
    m, k, n = shape
    act = sorted(T.ACTS)[(m + k + n) % 4]
    x, wg, wu, _ = _inputs(m, k, n, dtype, m + k + n)
    got = T.gated(x.cuda(), wg.cuda(), wu.cuda(), act=act)
    assert got.shape == (m, n) and got.dtype == dtype
    _check_forward(got, x, wg, wu, act)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_gated_backward(shape, dtype):
    m, k, n = shape
    act = sorted(T.ACTS)[(m + k + n + 1) % 4]
    x, wg, wu, dh = _inputs(m, k, n, dtype, m * k + n)
    got = T.gated_backward(dh.cuda(), x.cuda(), wg.cuda(), wu.cuda(), act=act)
    _check_backward(got, dh, x, wg, wu, act)
    again = T.gated_backward(dh.cuda(), x.cuda(), wg.cuda(), wu.cuda(), act=act)
    for a, b in zip(got, again):
        assert torch.equal(a, b), "the same inputs give the same bits"


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("shape", [(1030, 40, 2100), (2100, 72, 4100), (70, 2056, 1030), (4200, 4100, 40), (33, 4104, 2050), (20_000, 24, 40), (40, 24, 9000), (513, 1100, 1027)], ids=str)
def test_gated_large(shape, dtype):
    """Sizes at which tiles are larger, and at which the depth of a product is shared out."""
    m, k, n = shape
    x, wg, wu, dh = _inputs(m, k, n, dtype, m + 3 * n)
    _check_forward(T.gated(x.cuda(), wg.cuda(), wu.cuda()), x, wg, wu, "silu")
    _check_backward(T.gated_backward(dh.cuda(), x.cuda(), wg.cuda(), wu.cuda()), dh, x, wg, wu, "silu")


# Together these take each of the four products (h, the slopes, dx, the weights' gradients) through tiles of each size, whole
# and with their depth shared out, in 16 and in 32 bits.
TILINGS = {torch.bfloat16: [(24, 1450, 2732), (19, 3156, 331), (889, 1102, 3585), (3450, 35, 21), (4660, 1665, 23), (4308, 463, 20), (193, 2901, 3786), (48, 38, 1327),
                            (3457, 21, 1294), (3870, 20, 262), (947, 901, 4142), (139, 1490, 27), (772, 21, 1225), (30, 26, 394)],
           torch.float16: [(10_936, 997, 730), (1166, 3232, 2505), (16_396, 958, 500)],
           torch.float32: [(18, 1678, 3734), (2139, 694, 1500), (21, 1507, 2504), (1375, 590, 877), (1254, 88, 21), (4684, 2684, 21), (1227, 1717, 983), (3619, 2118, 23),
                           (196, 4176, 735), (85, 323, 21), (30, 26, 394), (1835, 22, 3601), (4152, 1960, 236), (912, 27, 3812), (616, 1539, 814), (52, 744, 57)]}


@pytest.mark.parametrize("dtype, shape", [(d, s) for d in TILINGS for s in TILINGS[d]], ids=str)
def test_gated_tilings(dtype, shape):
    m, k, n = shape
    x, wg, wu, dh = (t.cuda() for t in _inputs(m, k, n, dtype, m + 3 * n))
    act = sorted(T.ACTS)[m % 4]
    _check_forward(T.gated(x, wg, wu, act=act), x, wg, wu, act, where="cuda")
    got = T.gated_backward(dh, x, wg, wu, act=act)
    _check_backward(got, dh, x, wg, wu, act, where="cuda")
    for a, b in zip(got, T.gated_backward(dh, x, wg, wu, act=act)):
        assert torch.equal(a, b), "the same inputs give the same bits"


@pytest.mark.parametrize("act", sorted(T.ACTS))
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_gated_activations(act, dtype):
    """Every activation over arguments from tiny to large."""
    x, wg, wu, dh = _inputs(150, 40, 90, dtype, 3, scale=6.0)
    x[0] *= 1e-6
    x[1] *= 4
    got = T.gated(x.cuda(), wg.cuda(), wu.cuda(), act=act)
    _check_forward(got, x, wg, wu, act)
    _check_backward(T.gated_backward(dh.cuda(), x.cuda(), wg.cuda(), wu.cuda(), act=act), dh, x, wg, wu, act)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("pads", [(8, 16, 8, 24), (1, 0, 0, 0), (0, 3, 5, 1), (0, 0, 0, 7)], ids=str)
def test_gated_strides(pads, dtype):
    """Rows further apart than they are long, at odd places: the same values, and nothing written beside the output."""
    m, k, n = 70, 72, 96
    x, wg, wu, dh = (t.cuda() for t in _inputs(m, k, n, dtype, 9))

    def spread(t, pad):
        room = torch.full((t.shape[0] * (t.shape[1] + pad) + pad,), float("nan"), dtype=dtype, device="cuda")
        view = room[pad:].view(t.shape[0], t.shape[1] + pad)[:, :t.shape[1]]
        view.copy_(t)
        return view

    X, G, U, D = (spread(t, p) for t, p in zip((x, wg, wu, dh), pads))
    out = torch.full((m, n + pads[3]), 7.0, dtype=dtype, device="cuda")
    T.gated(X, G, U, out=out[:, :n])
    assert bool((out[:, n:] == 7.0).all())
    _check_forward(out[:, :n], x, wg, wu, "silu")
    _check_backward(T.gated_backward(D, X, G, U), dh, x, wg, wu, "silu")


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_gated_special_values_stay_in_their_rows(dtype):
    """A record or a weight row that is not finite spoils what is computed from it, and nothing else."""
    m, k, n = 70, 40, 50
    x, wg, wu, dh = (t.cuda() for t in _inputs(m, k, n, dtype, 4))
    clean = T.gated(x, wg, wu)
    x[13, 39] = float("nan")
    wg[49, 0] = float("inf")
    got = T.gated(x, wg, wu)
    assert torch.isnan(got[13]).all() and not torch.isfinite(got[:, 49]).all()
    keep = torch.ones(m, n, dtype=torch.bool, device="cuda")
    keep[13] = False
    keep[:, 49] = False
    assert torch.equal(got[keep], clean[keep])
    dx, dwg, dwu = T.gated_backward(dh[:, :49].contiguous(), x, wg[:49], wu[:49])
    assert torch.isnan(dx[13]).all() and torch.isfinite(dx[:13]).all() and torch.isfinite(dx[14:]).all()
    assert torch.isnan(dwg).all() and torch.isnan(dwu).all()   # every sum over records has the spoiled one in it


def test_gated_parts_of_the_gradient():
    x, wg, wu, dh = (t.cuda() for t in _inputs(90, 56, 72, torch.bfloat16, 8))
    dx, dwg, dwu = T.gated_backward(dh, x, wg, wu)
    only, a, b = T.gated_backward(dh, x, wg, wu, need_dw=False)
    assert torch.equal(only, dx) and a is None and b is None
    none, a, b = T.gated_backward(dh, x, wg, wu, need_dx=False)
    assert none is None and torch.equal(a, dwg) and torch.equal(b, dwu)


def test_gated_nothing():
    w = torch.ones(5, 6, device="cuda")
    x = torch.ones(0, 6, device="cuda")
    assert T.gated(x, w, w).shape == (0, 5)
    dx, dwg, dwu = T.gated_backward(torch.ones(0, 5, device="cuda"), x, w, w)
    assert dx.shape == (0, 6) and not dwg.any() and not dwu.any()


@pytest.mark.parametrize("act", ["silu", "gelu", "sigmoid"])
def test_gated_gradient_against_differences(act):
    """Central differences of the definition in 64 bits: their error is below step^2 times a third derivative (far below
    1e-5 here) and the gradient's own 32-bit error is far below that too."""
    x, wg, wu, dh = _inputs(9, 11, 13, torch.float32, 21)
    f = lambda x, g, u: float((_act64(x @ g.T, act)[0] * (x @ u.T) * dh.double()).sum())  # noqa: E731
    got = T.gated_backward(dh.cuda(), x.cuda(), wg.cuda(), wu.cuda(), act=act)
    g, h = torch.Generator().manual_seed(1), 1e-4
    ins = [x.double(), wg.double(), wu.double()]
    for i in range(3):
        for _ in range(5):
            way = torch.randn(ins[i].shape, generator=g, dtype=torch.float64)
            up, down = ([t + s * h * way if j == i else t for j, t in enumerate(ins)] for s in (1, -1))
            want = (f(*up) - f(*down)) / (2 * h)
            assert abs(float((got[i].double().cpu() * way).sum()) - want) < 1e-4 * max(1.0, abs(want))


def test_operators_in_autograd_and_on_other_streams():
    x, wg, wu, dh = (t.cuda() for t in _inputs(40, 24, 32, torch.bfloat16, 2))
    slots = _on_gpu(_make_slots(np.random.default_rng(0), 40, [1, "list", 1], 30))
    table = torch.randn(50, 8, device="cuda").to(torch.bfloat16).requires_grad_()
    wg.requires_grad_()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        pooled = T.embed(slots, table, 40)
        h = T.gated(pooled.flatten(1), wg, wu)
        h.backward(dh)
    s.synchronize()
    flat = T.embed(slots, table.detach(), 40).flatten(1)
    dx, dwg, _ = T.gated_backward(dh, flat, wg.detach(), wu)
    assert torch.equal(wg.grad, dwg) and wu.grad is None
    assert torch.equal(table.grad, T.embed_backward(dx.unflatten(1, (3, 8)), slots, 50))


def test_operators_in_a_graph():
    """Captured once, replayed on other inputs, with eager work between the replays."""
    rng = np.random.default_rng(1)
    slots = _on_gpu(_make_slots(rng, 200, [1, 1, "list"], 400))
    table, wg, wu = torch.randn(300, 16, device="cuda"), torch.randn(64, 48, device="cuda") / 7, torch.randn(64, 48, device="cuda") / 7
    dh = torch.randn(200, 64, device="cuda")
    state = [torch.zeros_like(t) for t in (table, wg, wu)], [torch.zeros_like(t) for t in (table, wg, wu)]

    def step(params, m, v):
        x = T.embed(slots, params[0], 200).flatten(1)
        dx, a, b = T.gated_backward(dh, x, params[1], params[2])
        T.adamw(params, [T.embed_backward(dx.unflatten(1, (3, 16)), slots, 300), a, b], m, v, step=3)
        return T.gated(x, params[1], params[2])

    eager = [t.clone() for t in (table, wg, wu)], *[[t.clone() for t in s] for s in state]
    mine = [t.clone() for t in (table, wg, wu)], *[[t.clone() for t in s] for s in state]
    warm = [t.clone() for t in (table, wg, wu)], *[[t.clone() for t in s] for s in state]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step(*warm)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h = step(*mine)
    for _ in range(4):
        graph.replay()
        want = step(*eager)
        torch.cuda.synchronize()
        assert torch.equal(h, want)
        for a, b in zip(mine, eager):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


# ------------------------------------------------------------------ AdamW
def _mix(x):
    x &= (1 << 64) - 1
    x = ((x ^ (x >> 30)) * 0xBF58476D1CE4E5B9) & ((1 << 64) - 1)
    x = ((x ^ (x >> 27)) * 0x94D049BB133111EB) & ((1 << 64) - 1)
    return x ^ (x >> 31)


E4M3 = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()


def _decode(codes, scale):
    with np.errstate(over="ignore", invalid="ignore"):
        return E4M3[codes] * np.repeat(np.ldexp(np.float32(1), scale.astype(int) - 127).astype(np.float32), 32)[:codes.size]


def _encode(x, random16):
    """Codes and scales by comparing with the values that codes stand for: the one below, or the one above it where the
    distance to the one below, as a share of the step and cut to 2^-16, and the random share together reach one."""
    n = x.size
    top = np.abs(np.pad(x, (0, -n % 32))).reshape(-1, 32).max(1)
    scale = np.where(np.isfinite(top), np.maximum(np.frexp(top)[1] - 1 - 7 + 127, 1), 255).astype(int)
    scale = np.where(top == 0, 1, scale)
    steps = E4M3[:127]
    y = x.astype(np.float64) / np.ldexp(1.0, np.repeat(np.where(scale == 255, 127, scale), 32)[:n] - 127)
    a = np.abs(np.where(np.isfinite(y), y, 0))
    low = np.searchsorted(steps, a, side="right") - 1
    share = (a - steps[low]) / (steps[np.minimum(low + 1, 126)] - steps[low])
    code = low + (share + random16 / 65536.0 >= 1) + np.where(y < 0, 128, 0)
    return np.where(np.repeat(scale, 32)[:n] == 255, 127, code).astype(np.uint8), scale.astype(np.uint8)


HYPER = dict(lr=2e-3, betas=(0.9, 0.99), eps=1e-6, weight_decay=0.1)


def _step64(p, g, m, v, step, grad_scale, lr, betas, eps, weight_decay):
    g = g * grad_scale
    m, v = betas[0] * m + (1 - betas[0]) * g, betas[1] * v + (1 - betas[1]) * g * g
    return p - lr * weight_decay * p - lr * (m / (1 - betas[0] ** step)) / (np.sqrt(v / (1 - betas[1] ** step)) + eps), m, v


SIZES = [1, 2, 7, 8, 9, 31, 32, 33, 63, 65, 2047, 2048, 2049, 0, 10_000, 4096 + 17]


@pytest.mark.parametrize("grad", TYPES, ids=str)
@pytest.mark.parametrize("param", TYPES, ids=str)
def test_adamw_32_bit_states(param, grad):
    """Three steps over tensors of many sizes (more than one launch takes), against the formulas in 64 bits, and copies."""
    g = torch.Generator().manual_seed(4)
    sizes = SIZES * 9
    p = [torch.randn(n, generator=g).to(param) for n in sizes]
    gpu = [t.clone().cuda() for t in p]
    m, v = [torch.zeros(n, device="cuda") for n in sizes], [torch.zeros(n, device="cuda") for n in sizes]
    copies = [torch.zeros(n, dtype=torch.bfloat16, device="cuda") for n in sizes] if param == torch.float32 else None
    for step in range(1, 4):
        grads = [(torch.randn(n, generator=g) * 10.0 ** (step - 2)).to(grad) for n in sizes]
        before = [(a.cpu().double().numpy(), b.cpu().double().numpy(), c.cpu().double().numpy()) for a, b, c in zip(gpu, m, v)]
        T.adamw(gpu, [t.cuda() for t in grads], m, v, copies=copies, step=step, grad_scale=0.5, **HYPER)
        for i, n in enumerate(sizes):
            wp, wm, wv = _step64(before[i][0], grads[i].double().numpy(), before[i][1], before[i][2], step, 0.5, **HYPER)
            # (four roundings of m and six of v, none larger than their larger term; of p: three, and a quotient's ten)
            small = torch.from_numpy(np.abs(before[i][1]) + np.abs(0.5 * grads[i].double().numpy()))
            move = torch.from_numpy(np.abs(wp - before[i][0]) + np.abs(before[i][0]) * HYPER["lr"] * HYPER["weight_decay"])
            quotient = 16 * U32 + 4 * U32 * small.numpy() / np.maximum(np.abs(wm), 1e-300)
            _close(m[i], torch.from_numpy(wm), 4 * U32 * small, f"m of {n}")
            _close(v[i], torch.from_numpy(wv), 6 * U32 * torch.from_numpy(np.abs(wv)), f"v of {n}")
            _close(gpu[i], torch.from_numpy(wp), 3 * U32 * torch.from_numpy(np.abs(before[i][0])) + move * torch.from_numpy(quotient), f"weights of {n}")
            if copies is not None:
                assert torch.equal(copies[i], gpu[i].to(torch.bfloat16))


@pytest.mark.parametrize("grad", TYPES, ids=str)
@pytest.mark.parametrize("param", TYPES, ids=str)
def test_adamw_8_bit_states(param, grad):
    """Codes and scales bit for bit, weights to the last bits, over steps that start from nothing."""
    rng = np.random.default_rng(11)
    b1, b2 = HYPER["betas"]
    f = np.float32
    sizes, seed = SIZES, (1 << 63) + 12345
    gpu = [torch.from_numpy(rng.standard_normal(n).astype(f)).to(param).cuda() for n in sizes]
    m, v = ([torch.zeros(n, dtype=torch.uint8, device="cuda") for n in sizes] for _ in range(2))
    ms, vs = ([torch.zeros(-(-n // 32), dtype=torch.uint8, device="cuda") for n in sizes] for _ in range(2))
    for step in range(1, 4):
        grads = [torch.from_numpy((rng.standard_normal(n) * 10.0 ** rng.integers(-6, 1, n)).astype(f)).to(grad) for n in sizes]
        before = [[t[i].cpu().numpy() if t is not gpu else t[i].cpu().double().numpy() for t in (gpu, m, v, ms, vs)] for i in range(len(sizes))]
        T.adamw(gpu, [t.cuda() for t in grads], [t.view(torch.float8_e4m3fn) for t in m], v, ms, [t.view(torch.float8_e8m0fnu) for t in vs], step=step, seed=seed, **HYPER)
        for i, n in enumerate(sizes):
            if not n:
                continue
            p, cm, cv, sm, sv = before[i]
            g = grads[i].float().numpy()
            m0, r0 = _decode(cm, sm), _decode(cv, sv)
            m1 = m0 * f(b1) + g * f(1 - b1)
            v1 = (r0 * r0) * f(b2) + (g * g) * f(1 - b2)
            bits = np.array([_mix(_mix(_mix(seed + step) + i) + k) for k in range((n + 1) // 2)], dtype=np.uint64)
            bits = np.repeat(bits, 2)[:n] >> ((np.arange(n, dtype=np.uint64) & np.uint64(1)) << np.uint64(5))
            for x, shift, code, scale in ((m1, 0, m, ms), (np.sqrt(v1), 16, v, vs)):
                want, want_scale = _encode(x, ((bits >> np.uint64(shift)) & np.uint64(0xFFFF)).astype(np.float64))
                assert np.array_equal(scale[i].cpu().numpy(), want_scale), f"scales of {n}"
                assert np.array_equal(code[i].cpu().numpy(), want), f"codes of {n}"
            wp, _, _ = _step64(p, g.astype(np.float64), m0.astype(np.float64), (r0 * r0).astype(np.float64), step, 1.0, **HYPER)
            move = np.abs(wp - p) + np.abs(p) * HYPER["lr"] * HYPER["weight_decay"]
            quotient = 16 * U32 + 4 * U32 * (np.abs(m0) + np.abs(g)) / np.maximum(np.abs(m1).astype(np.float64), 1e-300)
            _close(gpu[i], torch.from_numpy(wp), torch.from_numpy(3 * U32 * np.abs(p) + move * quotient), f"weights of {n}")


def test_adamw_8_bit_rounding_is_fair():
    """A state that decays by less than a step of its code still decays on average: 4,096 copies of one element, 200 steps
    without gradient; the mean's expected deviation is a step of 1/16 over sqrt(4,096), times sqrt(200), below 2 %."""
    n, b1 = 32 * 4096, 0.999
    m = torch.zeros(n, device="cuda")
    m.view(-1, 32)[:, 0], m.view(-1, 32)[:, 1] = 200.0, 100.0
    codes, zero = m.to(torch.float8_e4m3fn), torch.zeros(n, dtype=torch.uint8, device="cuda")
    scale, zs = torch.full((n // 32,), 127, dtype=torch.uint8, device="cuda"), torch.zeros(n // 32, dtype=torch.uint8, device="cuda")
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    first = codes.float().view(-1, 32)[:, :2].mean(0)
    for step in range(1, 201):
        T.adamw([p], [g], [codes], [zero], [scale], [zs], step=step, betas=(b1, 0.99), eps=1.0, seed=9)
    now = (codes.float() * scale.view(torch.float8_e8m0fnu).float().repeat_interleave(32)).view(-1, 32)[:, :2].mean(0)
    assert torch.allclose(now / first, torch.full((2,), b1 ** 200, device="cuda"), rtol=0.06)


def test_adamw_not_finite():
    """A gradient that is not finite spoils its element (32 bits), or its block's states (8 bits), and nothing else."""
    n = 100
    p, g = torch.ones(n, device="cuda"), torch.ones(n, device="cuda")
    g[40] = float("nan")
    m, v = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    T.adamw([p], [g], [m], [v], step=1)
    assert torch.isnan(p).nonzero().flatten().tolist() == [40] and torch.isnan(m).nonzero().flatten().tolist() == [40]
    p = torch.ones(n, device="cuda")
    cm, cv = (torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2))
    sm, sv = (torch.zeros(4, dtype=torch.uint8, device="cuda") for _ in range(2))
    T.adamw([p], [g], [cm], [cv], [sm], [sv], step=1)
    assert torch.isnan(p).nonzero().flatten().tolist() == [40]
    assert (sm == 255).tolist() == [False, True, False, False] and (sv == 255).tolist() == [False, True, False, False]
    T.adamw([p], [torch.ones(n, device="cuda")], [cm], [cv], [sm], [sv], step=2)
    assert torch.isnan(p).nonzero().flatten().tolist() == list(range(32, 64))


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("off", [0, 1, 3])
def test_adamw_places(bits, off):
    """Tensors that begin anywhere: the same bits, and nothing written outside them."""
    n, kind = 1000, torch.uint8 if bits == 8 else torch.float32
    g = torch.Generator(device="cuda").manual_seed(0)
    p0, grad = torch.randn(n, device="cuda", generator=g), torch.randn(n, device="cuda", generator=g)
    outs = []
    for o in (0, off):
        rooms = [torch.zeros(n + 8, device="cuda"), torch.zeros(n + 8, dtype=kind, device="cuda"), torch.zeros(n + 8, dtype=kind, device="cuda")]
        scales = [torch.zeros(40, dtype=torch.uint8, device="cuda") for _ in range(2)] if bits == 8 else [None, None]
        p, m, v = (r[o:o + n] for r in rooms)
        p.copy_(p0)
        G = torch.zeros(n + 8, device="cuda")[o:o + n]
        G.copy_(grad)
        cut = [None if s is None else [s[o:o + 32]] for s in scales]
        for step in (1, 2):
            T.adamw([p], [G], [m], [v], *cut, step=step, seed=5)
        for r in rooms:
            assert not r[:o].any() and not r[o + n:].any()
        outs.append([p.clone(), m.clone(), v.clone()])
    assert all(torch.equal(a, b) for a, b in zip(*outs))


@pytest.mark.parametrize("bits", [8, 32])
def test_adamw_class(bits):
    """Weights without a gradient stay, types are grouped, a state that is saved and loaded goes on the same way."""
    make = lambda: [torch.full((37,), 0.5, device="cuda"), torch.full((3, 5), 0.25, device="cuda").to(torch.bfloat16), torch.ones(4, device="cuda")]  # noqa: E731
    a, b = make(), make()
    one = T.AdamW(a, lr=0.1, bits=bits, seed=3)
    grads = lambda k: [torch.full((37,), 0.1 * k, device="cuda"), torch.full((3, 5), -0.2, device="cuda").to(torch.bfloat16), None]  # noqa: E731
    one.step(grads(1))
    saved = {k: [t.clone() for t in x] if isinstance(x, list) else x for k, x in one.state_dict().items()}
    for x, y in zip(a, b):
        y.copy_(x)
    one.step(grads(2))
    two = T.AdamW(b, lr=0.1, bits=bits)
    two.load_state_dict(saved)
    two.step(grads(2))
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    assert torch.equal(a[2], torch.ones(4, device="cuda")) and bool((a[0] < 0.5).all()) and bool((a[1] > 0.25).all())
    w = torch.nn.Parameter(torch.ones(5, device="cuda"))
    three = T.AdamW([w], bits=bits)
    (w * 2).sum().backward()
    three.step()
    assert bool((w < 1).all())
    three.zero_grad()
    assert w.grad is None
