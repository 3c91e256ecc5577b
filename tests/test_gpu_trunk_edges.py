"""Orthogonalised matrices, Muon, norms and joins where a call's edges lie: lists of several kinds, every tile of the products, what overlaps.

Tolerances are what the header promises: products of both parts are off like products in 32 bits (held to twice what the same formula in torch's
32 bits is off), products of first parts by 1.6e-3 of the result's size; what is stored adds half a unit of its type."""
import math

import pytest
import torch

from paper_2210_07768_amd import binding as B
from paper_2210_07768_amd import train as T

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
HALF_UNIT = {F32: 2.0 ** -24, F16: 2.0 ** -11, BF16: 2.0 ** -8}


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _r(g, *shape, dtype=F32, size=1.0, shift=0.0):
    return (torch.randn(*shape, device="cuda", generator=g) * size + shift).to(dtype)


def _decaying(g, rows, columns, dtype=F32):
    n = min(rows, columns)
    s = torch.arange(1, n + 1, device="cuda").float().pow(-0.7)
    return ((_r(g, rows, n) * s) @ _r(g, n, columns) + 0.1 * _r(g, rows, columns)).to(dtype)


def _iterated(u, dtype, steps=5, eps=1e-7):
    """The formula in `dtype`, the norm in 64 bits."""
    tall = u.shape[0] > u.shape[1]
    x = u.double().t().contiguous() if tall else u.double()
    x = (x / (x.norm() + eps)).to(dtype)
    a, b, c = T.NEWTON_SCHULZ
    for _ in range(steps):
        gram = torch.mm(x, x.t().contiguous())
        x = a * x + torch.mm(b * gram + c * torch.mm(gram, gram), x)
    return x.t() if tall else x


def _goal(u, exact, dtype, steps=5):
    """(the result in 64 bits, how far in the norm a result stored in `dtype` may be from it)"""
    want = _iterated(u, torch.float64, steps)
    off = 2 * float((_iterated(u, F32, steps).double() - want).norm()) if exact else 1.6e-3 * float(want.norm())
    return want, off + HALF_UNIT[dtype] * (float(want.norm()) + off)


def _near(got, want, off, what):
    far = float((got.double() - want).norm())
    assert torch.isfinite(got).all() and far <= off, f"{what}: {far:.3g} off, {off:.3g} allowed"


# ------------------------------------------------------------------ lists
def test_lists_of_several_kinds():
    """More matrices of either kind of products than a launch holds, and of those that a workgroup holds, in turn."""
    g = _gen(60)
    shapes = [(64, 700), (257, 260), (20, 30), (270, 257)] * 33
    given = [_decaying(g, r, c, BF16) for r, c in shapes]
    got = T.orthogonalise(given)
    start = [torch.zeros(s, device="cuda", dtype=BF16) for s in shapes]
    p, m = [t.clone() for t in start], [torch.zeros(s, device="cuda") for s in shapes]
    T.muon(p, given, m, lr=1.0, momentum=0.5, nesterov=False, weight_decay=0.0, adjust="none")   # (0 - O(gradient))
    for u, o, w, x in zip(given, got, p, m):
        want, off = _goal(u, min(u.shape) <= 256, BF16)
        _near(o, want, off, tuple(u.shape))
        _near(-w, want, off, f"weights {tuple(u.shape)}")
        assert torch.equal(x, u.float())


# ------------------------------------------------------------------ products of both parts, and of first parts
def _made(kind, rows, columns):
    g = _gen(rows + columns)
    if kind == "decaying":
        return _decaying(g, rows, columns)
    if kind == "normal":
        return _r(g, rows, columns)
    if kind == "one direction":
        return _r(g, rows, 1) @ _r(g, 1, columns) + 1e-3 * _r(g, rows, columns)
    if kind == "most rows zero":
        return _r(g, rows, columns) * (torch.arange(rows, device="cuda") % 5 == 0)[:, None]
    u = torch.zeros(rows, columns, device="cuda")   # "unit 319": 319 equal singular values
    u.diagonal()[:int(kind.split()[1])] = 1.0
    return u


@pytest.mark.parametrize("kind, rows, columns", [("decaying", 1000, 400), ("normal", 300, 400), ("one direction", 400, 1000), ("most rows zero", 257, 257), ("unit 319", 319, 319), ("unit 3", 300, 600),
                                                 ("unit 2", 700, 260)])
def test_results_are_rounded_once_unless_asked(kind, rows, columns):
    """Left to itself `orthogonalise` gives 32-bit accuracy, rounded to the result's type; half precision is the caller's to ask for.  (Products of first
    parts of unit matrices are off by more than bfloat16's half unit, 2^-8: their roundings are all the same.)"""
    u = _made(kind, rows, columns)
    want, off = _goal(u, True, F32)
    floor = 2.0 ** -21 * float(want.norm())   # (where 32 bits make no mistake at all: two parts have 22 bits)
    single = T.orthogonalise(u)
    _near(single, want, off + 15 * floor, kind)   # (three products a step)
    assert not torch.equal(single, T.orthogonalise(u, exact=False))
    for dtype in (F16, BF16):
        got = T.orthogonalise(u, dtype=dtype)
        assert torch.equal(got, single.to(dtype))
        assert torch.equal(got, T.orthogonalise(u, dtype=dtype, exact=True))


@pytest.mark.parametrize("kind, rows, columns, most", [("decaying", 1000, 400, 1.6e-3), ("normal", 300, 400, 1.6e-3), ("one direction", 400, 1000, 2.8e-3), ("most rows zero", 257, 257, 2.8e-3),
                                                       ("unit 319", 319, 319, 27e-3), ("unit 2", 700, 260, 27e-3)])
def test_products_of_first_parts(kind, rows, columns, most):
    """As far off as the header says, before the result is rounded."""
    u = _made(kind, rows, columns)
    want = _iterated(u, torch.float64)
    _near(T.orthogonalise(u, exact=False), want, most * float(want.norm()), kind)


# ------------------------------------------------------------------ results beside and over what they are made of
def test_results_in_the_same_buffer():
    """Columns beside an input's are no part of it; a matrix's own result may lie over it anyhow, as all of it is read before."""
    g = _gen(61)
    for n, d in ((37, 24), (300, 270)):
        both = _r(g, n, 3 * d)
        a, b, c = (both[:, i * d:(i + 1) * d] for i in range(3))
        w = _r(g, d, shift=1.0)
        want = T.norm(a.contiguous(), w)
        assert torch.equal(T.norm(a, w, out=c), want) and torch.equal(c, want)
        want = T.join(a.contiguous(), b.contiguous(), w)
        assert torch.equal(T.join(a, b, w, out=c), want) and torch.equal(c, want)
        want = T.orthogonalise([t.contiguous() for t in (a, b, c)])
        T.orthogonalise([a, b, c], out=[a, b, c])
        assert all(torch.equal(t, o) for t, o in zip((a, b, c), want))
        rows = _r(g, n + 3, d)
        want = T.orthogonalise(rows[:n].clone())
        T.orthogonalise(rows[:n], out=rows[3:])
        assert torch.equal(rows[3:], want)


def test_shifted_results_are_refused():
    g = _gen(62)
    rows, w = _r(g, 5000, 64), _r(g, 64, shift=1.0)
    flat = torch.zeros(4 * 48 * 40, device="cuda")
    p = [flat[i * 1920 - (i == 1):][:1920].view(48, 40) for i in range(2)]
    grads, m = [_r(g, 48, 40) for _ in range(2)], [torch.zeros(48, 40, device="cuda") for _ in range(2)]
    before = rows.clone()
    for call in (lambda: T.norm(rows[:-1], w, out=rows[1:]), lambda: T.norm(rows[1:], w, out=rows[:-1]), lambda: T.join(rows[:100], rows[100:200], w, out=rows[150:250]),
                 lambda: T.join(rows[:100], rows[100:200], w, next_weight=w, out=rows[300:400], out_next=rows[399:499]), lambda: T.muon(p, grads, m),
                 lambda: T.orthogonalise([rows[:50], rows[50:100]], out=[rows[40:90], rows[200:250]])):
        with pytest.raises(B.FbxError) as e:
            call()
        assert e.value.status == B.E_ARG and "overlaps" in str(e.value)
    assert torch.equal(rows, before) and not flat.any() and not any(t.any() for t in m)


# ------------------------------------------------------------------ Muon's lists
def test_muon_steps_all_lists_or_none():
    """Weights of two types are two calls; what only the library refuses of the second (3e38 times 0.2 sqrt(64)) leaves the first one's alone."""
    w = [torch.ones(1, 1, device="cuda"), torch.ones(64, 64, device="cuda", dtype=BF16)]
    opt = T.Muon(w, lr=3e38)
    grads = [torch.ones_like(t) for t in w]
    with pytest.raises(B.FbxError) as e:
        opt.step(grads)
    assert "factor" in str(e.value)
    assert all((t == 1).all() for t in w) and not any(m.any() for m in opt.m) and opt.step_count == 0
    opt.step(grads, lr=1.0)
    assert all((t != 1).any() for t in w) and all(m.all() for m in opt.m) and opt.step_count == 1


# ------------------------------------------------------------------ every tile of the products
LISTS = {"tiles of 64": [(400, 300), (300, 400)], "tiles of 128": [(513, 520)] * 16 + [(520, 513)] * 16, "A and B in tiles of 256": [(700, 701)] * 16 + [(715, 699)] * 16,
         "X in tiles of 256": [(1050, 701)] * 8 + [(700, 1050)] * 8}   # (as the library's rule has it; with both parts the last list's A is in tiles of 64)


@pytest.mark.parametrize("exact", [True, False])
@pytest.mark.parametrize("name", list(LISTS))
def test_every_tile(name, exact):
    """Results against 64 bits; into weights of each type, with copies: what the results themselves give, rounded a few times in 32 bits and once to
    the weights' type."""
    g = _gen(70)
    shapes = LISTS[name]
    given = [_decaying(g, r, c) for r, c in shapes]
    got = T.orthogonalise(given, exact=exact)
    for i, (u, o) in enumerate(zip(given, got)):
        want, off = _goal(u, exact, F32)
        _near(o, want, off, (name, i))
    assert all(torch.equal(a, b) for a, b in zip(got, T.orthogonalise(given, exact=exact)))   # the same inputs, the same bits
    lr, decay = 0.05, 0.1
    for kind in (F32, F16, BF16):
        p = [_r(g, *s, size=0.05, dtype=kind) for s in shapes]
        before, m = [t.double() for t in p], [torch.zeros(s, device="cuda") for s in shapes]
        copies = [torch.zeros(s, dtype=BF16, device="cuda") for s in shapes] if kind == F32 else None
        T.muon(p, given, m, copies, lr=lr, momentum=0.9, nesterov=False, weight_decay=decay, exact=exact)
        for i, (s, w, b, o) in enumerate(zip(shapes, p, before, got)):
            step = lr * 0.2 * math.sqrt(max(s))
            want = b * (1 - lr * decay) - step * o.double()
            terms = 4 * HALF_UNIT[F32] * (b.abs() + step * o.double().abs())   # (the two factors, the product and the difference)
            limit = terms + HALF_UNIT[kind] * (want.abs() + terms) + 2.0 ** -25
            assert ((w.double() - want).abs() <= limit).all(), (name, kind, i)
            assert torch.equal(m[i], given[i])
            if copies is not None:
                assert ((copies[i].double() - want).abs() <= terms + HALF_UNIT[BF16] * (want.abs() + terms) + 2.0 ** -133).all(), (name, i)


@pytest.mark.parametrize("shape", [(300, 400), (520, 270)])
@pytest.mark.parametrize("exact", [True, False])
def test_extremes_of_larger_matrices(exact, shape):
    """Zeros, one number, what is not finite, and sizes near the ends of 32 bits, in the launches that larger matrices go through."""
    g = _gen(71)
    zero, one, nan, inf, usual = torch.zeros(shape, device="cuda"), torch.zeros(shape, device="cuda"), *(_r(g, *shape) for _ in range(3))
    one[shape[0] - 1, 5] = -2.5
    nan[2, 2], inf[-1, -1] = float("nan"), float("-inf")
    tiny, huge = usual * 2.0 ** -110, usual * 2.0 ** 120
    got = T.orthogonalise([zero, one, nan, inf, tiny, huge, usual], eps=1e-30, exact=exact)
    assert not got[0].any() and torch.isnan(got[2]).all() and torch.isnan(got[3]).all()
    most = 1.6e-3 if not exact else 2.0 ** -17   # (one number: 15 products, 2^-21 each)
    alone = _iterated(one, torch.float64)
    assert (got[1] != 0).sum() == 1 and abs(float(got[1][-1, 5] - alone[-1, 5])) <= most * abs(float(alone[-1, 5]))
    want, off = _goal(usual, exact, F32)
    for i in (5, 6):
        _near(got[i], want, off, i)
    assert torch.equal(got[5], got[6])   # (a power of two apart)
    near = _iterated(tiny, torch.float64, eps=1e-30)
    _near(got[4], near, 2 * off, "tiny")


@pytest.mark.parametrize("param", [F32, F16, BF16])
def test_what_muon_is_left_to(param):
    """Without the caller's word products are of both parts, but for bfloat16 weights of more than 256 rows and columns."""
    g = _gen(72)
    shapes = [(256, 600), (600, 256), (257, 257), (20, 30)]
    grads = [_decaying(g, *s) for s in shapes]

    def step(**how):
        p = [torch.zeros(s, dtype=param, device="cuda") for s in shapes]
        T.muon(p, grads, [torch.zeros(s, device="cuda") for s in shapes], lr=1.0, adjust="none", **how)
        return p

    left, both, first = step(), step(exact=True), step(exact=False)
    for i in range(4):
        assert not torch.equal(both[i], first[i]) or i == 3
        alone = [torch.zeros(shapes[i], dtype=param, device="cuda")]
        T.muon(alone, [grads[i]], [torch.zeros(shapes[i], device="cuda")], lr=1.0, adjust="none", exact=param != BF16 or i != 2)
        assert torch.equal(left[i], alone[0]), i
