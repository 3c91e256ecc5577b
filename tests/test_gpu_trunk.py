"""Norms, joins and their gradients, orthogonalised updates and Muon on the GPU against their definitions in 64 bits.

Tolerances of the norms and joins are running error bounds: `Num` carries every value of the formula in 64 bits beside a bound on what the
same formula is off in 32 bits, each operation adding half a unit (U32) of its result.  A row's sum is of lanes' sums of at
most 16 terms, six halvings and at most 16 wavefronts: with min(n, 64) additions behind any of its terms at most, half a unit
each.  A column's sum has no order here: as many as it has terms.  What is stored adds half a unit of its type.

Of orthogonalised matrices: a step's own error is bounded element by element with the products of magnitudes (`_step_bound`); steps behind it
multiply an error's norm by the largest slope of their polynomial at most.  A result of products in half precision is held to what
its documentation promises."""
import math
import threading

import pytest
import torch

from paper_2210_07768_amd import binding as B
from paper_2210_07768_amd import train as T

pytestmark = pytest.mark.gpu
U32 = 2.0 ** -24
HALF_UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -133}
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
PAIRS = [(F32, F32), (F16, F16), (BF16, BF16), (F32, F16), (F32, BF16)]   # types of the stream and of the block


def _close(got, want, bound, what):
    dtype = got.dtype
    got, want, bound = got.double(), want.double(), bound.double()
    limit = bound + HALF_UNIT[dtype] * (want.abs() + bound) + TINY[dtype]
    off = (got - want).abs()
    assert got.shape == want.shape, what
    assert torch.isfinite(got).all(), f"{what}: not finite"
    bad = off > limit
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((off / limit).max()):.3g} times the bound"


class Num:
    """A value in 64 bits, and a bound on the error of what 32 bits make of it."""

    def __init__(self, v, e=None):
        self.v = v.double() if isinstance(v, torch.Tensor) else torch.tensor(float(v), dtype=torch.float64, device="cuda")
        self.e = torch.zeros_like(self.v) if e is None else e

    @staticmethod
    def of(x):
        return x if isinstance(x, Num) else Num(x)

    def _rounded(self, v, e):
        return Num(v, e + U32 * (v.abs() + e) + TINY[F32])

    def __add__(self, o):
        o = Num.of(o)
        return self._rounded(self.v + o.v, self.e + o.e)

    def __sub__(self, o):
        o = Num.of(o)
        return self._rounded(self.v - o.v, self.e + o.e)

    def __mul__(self, o):
        o = Num.of(o)
        return self._rounded(self.v * o.v, self.v.abs() * o.e + self.e * o.v.abs() + self.e * o.e)

    __rmul__ = __mul__

    def sum(self, dim, keepdim=False):
        n = self.v.shape[dim]
        additions = min(n, 64) if dim == 1 else n + 64
        return Num(self.v.sum(dim, keepdim=keepdim), self.e.sum(dim, keepdim=keepdim) + additions * U32 * (self.v.abs() + self.e).sum(dim, keepdim=keepdim) + TINY[F32])

    def mean(self):
        return self.sum(1, keepdim=True) * Num(1.0 / self.v.shape[1], torch.tensor(U32 / self.v.shape[1], dtype=torch.float64, device="cuda"))

    def inverse_root(self):
        """1 / sqrt, both rounded; of a value whose least is above 0."""
        low = (self.v - self.e).clamp(min=self.v * 1e-3)
        v = self.v.rsqrt()
        e = low.rsqrt() - v
        return Num(v, e + 3 * U32 * (v + e))

    def sigmoid(self):
        """By the hardware's exponential and reciprocal: a unit each, and |z| units for the rounding of its argument."""
        v = torch.sigmoid(self.v)
        return Num(v, self.e * 0.25 + v * (1 - v) * 2 * U32 * (self.v.abs() + 2) + 4 * U32 * v + 2.0 ** -126)


def _norm_num(v, kind, eps):
    if kind == "layer":
        v = v - v.mean()
    inverse = ((v * v).mean() + Num(eps, torch.tensor(U32 * eps, dtype=torch.float64, device="cuda"))).inverse_root()
    return v * inverse, inverse


def _back_num(p, unit, inverse, kind):
    along = unit * (p * unit).mean()
    return ((p - p.mean()) - along) * inverse if kind == "layer" else (p - along) * inverse


def _r(g, *shape, dtype=F32, size=1.0, shift=0.0):
    return (torch.randn(*shape, device="cuda", generator=g) * size + shift).to(dtype)


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _pad(t, pad):
    """The same rows, `pad` elements further apart."""
    wide = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), dtype=t.dtype, device=t.device)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


# (records, dim): a row of fewer, as many and more elements than a lane, a wavefront and a workgroup hold; odd ones; few and many rows
SHAPES = [(1, 1), (3, 2), (70, 5), (1000, 8), (513, 9), (37, 17), (129, 63), (64, 64), (300, 100), (1, 128), (65, 257), (40, 411), (17, 512), (9, 513), (2, 1000), (33, 1536), (20, 2049),
          (5, 2624), (7, 4097), (3, 8192), (2, 8193), (2, 16384)]


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("types", PAIRS, ids=str)
def test_norm_and_gradient(types, kind):
    stream, block = types
    for i, (n, d) in enumerate(SHAPES):
        g = _gen(1000 + i)
        vectors = [block, F32][i % 2]
        x, w, dy = _pad(_r(g, n, d, dtype=stream, shift=0.5), i % 3), _r(g, d, dtype=vectors, size=0.3, shift=1.0), _pad(_r(g, n, d, dtype=block), i % 4)
        eps = [1e-6, 1e-3][i % 2]
        unit, inverse = _norm_num(Num(x), kind, eps)
        want = unit * Num(w)
        got = T.norm(x, w, kind=kind, eps=eps, dtype=block)
        assert got.dtype == block
        _close(got, want.v, want.e, f"norm {n} x {d}")
        into = _pad(torch.zeros(n, d, dtype=block, device="cuda"), 1 + i % 3)
        assert T.norm(x, w, kind=kind, eps=eps, dtype=block, out=into) is into and torch.equal(into, got)
        assert torch.isnan(into._base if into._base is not None else into)[:, d:].all()   # beyond the rows: as it was
        dx, dw = T.norm_backward(dy, x, w, kind=kind, eps=eps)
        assert dx.dtype == stream and dw.dtype == vectors
        want = _back_num(Num(dy) * Num(w), unit, inverse, kind)
        _close(dx, want.v, want.e, f"dx {n} x {d}")
        want = (Num(dy) * unit).sum(0)
        _close(dw, want.v, want.e, f"dweight {n} x {d}")
        bare = T.norm(x, None, kind=kind, eps=eps, dtype=block)
        _close(bare, unit.v, unit.e, f"norm without weights {n} x {d}")
        only = T.norm_backward(dy, x, w, kind=kind, eps=eps, need_dx=False)
        assert only[0] is None and torch.equal(only[1], dw)
        only = T.norm_backward(dy, x, w, kind=kind, eps=eps, need_dw=False)
        assert only[1] is None and torch.equal(only[0], dx)


def _join_num(x, y, weight, gate, scale, next_weight, post, then, gate_act, kind, eps):
    r = {}
    r["unit"], r["inverse"] = _norm_num(Num(y), kind, eps) if post else (Num(y), None)
    scale = Num(scale) if isinstance(scale, torch.Tensor) else Num(scale, torch.tensor(U32 * abs(scale), dtype=torch.float64, device="cuda"))
    r["scale"], r["weight"] = scale, Num(1.0) if weight is None else Num(weight)
    r["both"] = r["scale"] * r["weight"]
    r["gate"] = Num(1.0) if gate is None else Num(gate).sigmoid() if gate_act == "sigmoid" else Num(gate)
    r["out"] = Num(x) + r["gate"] * r["both"] * r["unit"]
    if then:
        r["after"], r["after_inverse"] = _norm_num(r["out"], kind, eps)
        r["next"] = r["after"] * (Num(1.0) if next_weight is None else Num(next_weight))
    return r


def _join_back_num(r, dout, dnext, gate, next_weight, post, gate_act, kind):
    d = Num(dout) if dout is not None else None
    w = {}
    if dnext is not None:
        q = Num(dnext) * (Num(1.0) if next_weight is None else Num(next_weight))
        back = _back_num(q, r["after"], r["after_inverse"], kind)
        w["dnext_weight"] = (Num(dnext) * r["after"]).sum(0)
        d = back if d is None else d + back
    w["dx"] = d
    through = d * r["unit"]
    sums = (through * r["gate"]).sum(0)
    w["dweight"], w["dscale"] = sums * r["scale"], sums * r["weight"]
    if gate is not None:
        slope = through * r["both"]
        slope = slope.sum(1, keepdim=True) if gate.shape[1] == 1 else slope
        w["dgate"] = slope * (r["gate"] * (Num(1.0) - r["gate"])) if gate_act == "sigmoid" else slope
    p = d * (r["both"] * r["gate"])
    w["dy"] = _back_num(p, r["unit"], r["inverse"], kind) if post else p
    return w


FORMS = [dict(gate="full", act="sigmoid", scale=True, post=True, then=True), dict(gate="row", act="sigmoid", scale=False, post=True, then=True),
         dict(gate="full", act="none", scale=False, post=False, then=True), dict(gate=None, act="none", scale=True, post=True, then=False),
         dict(gate="row", act="none", scale=True, post=False, then=True), dict(gate=None, act="sigmoid", scale=False, post=False, then=False),
         dict(gate="row", act="sigmoid", scale=True, post=True, then=False)]


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("types", PAIRS, ids=str)
def test_join_and_gradient(types, kind):
    stream, block = types
    for i, (n, d) in enumerate(SHAPES):
        form = FORMS[i % len(FORMS)]
        g = _gen(2000 + i)
        vectors = [F32, block][i % 2]
        x, y = _pad(_r(g, n, d, dtype=stream, shift=0.3), i % 2), _pad(_r(g, n, d, dtype=block, size=2.0, shift=0.2), i % 3)
        weight = _r(g, d, dtype=vectors, size=0.3, shift=1.0) if form["post"] and i % 5 else None
        gate = None if form["gate"] is None else _pad(_r(g, n, 1 if form["gate"] == "row" else d, dtype=block, size=2.0), i % 4)
        scale = _r(g, d, dtype=vectors, size=0.1, shift=0.3) if form["scale"] else 0.7
        next_weight = _r(g, d, dtype=vectors, size=0.3, shift=1.0) if form["then"] and i % 4 else None
        how = dict(post=form["post"], then=form["then"], gate_act=form["act"], kind=kind, eps=[1e-6, 1e-4][i % 2])
        r = _join_num(x, y, weight, gate, scale, next_weight, **how)
        got = T.join(x, y, weight, gate, scale, next_weight, **how)
        out, nxt = got if form["then"] else (got, None)
        assert out.dtype == stream
        _close(out, r["out"].v, r["out"].e, f"out {n} x {d} {form}")
        if nxt is not None:
            assert nxt.dtype == block
            _close(nxt, r["next"].v, r["next"].e, f"next {n} x {d} {form}")
        into = [_pad(torch.zeros(n, d, dtype=t, device="cuda"), 1 + i % 3) for t in (stream, block)[:1 + form["then"]]]
        T.join(x, y, weight, gate, scale, next_weight, **how, out=into[0], out_next=into[1] if form["then"] else None)
        assert torch.equal(into[0], out) and (nxt is None or torch.equal(into[1], nxt))
        assert all(torch.isnan(t._base)[:, d:].all() for t in into)
        dout = _pad(_r(g, n, d, dtype=stream), i % 2) if not form["then"] or i % 3 else None
        dnext = _pad(_r(g, n, d, dtype=block), i % 3) if form["then"] else None
        given = (dout, dnext, x, y, weight, gate, scale, next_weight)
        back = T.join_backward(*given, **how)
        want = _join_back_num(r, dout, dnext, gate, next_weight, form["post"], form["act"], kind)
        there = {"dx": x, "dy": y, "dweight": weight, "dgate": gate, "dscale": scale if form["scale"] else None, "dnext_weight": next_weight}
        for name, like in there.items():
            value = getattr(back, name)
            assert (value is None) == (like is None), name
            if value is not None:
                assert value.dtype == like.dtype and value.shape == like.shape
                _close(value, want[name].v, want[name].e, f"{name} {n} x {d} {form}")
                alone = getattr(T.join_backward(*given, **how, need=[name[1:]]), name)
                assert torch.equal(alone, value), name
        assert all(v is None for v in T.join_backward(*given, **how, need=[]))


@pytest.mark.parametrize("n, d", [(5000, 24), (3001, 411), (2000, 2624)])
def test_many_records(n, d):
    """More rows than the workgroups take at a time, so that each takes several."""
    g = _gen(7)
    x, y, gate = _r(g, n, d, dtype=F32), _r(g, n, d, dtype=BF16), _r(g, n, d, dtype=BF16)
    w, scale, w2 = (_r(g, d, size=0.2, shift=1.0) for _ in range(3))
    how = dict(post=True, then=True, gate_act="sigmoid", kind="rms", eps=1e-6)
    dout, dnext = _r(g, n, d), _r(g, n, d, dtype=BF16)
    r = _join_num(x, y, w, gate, scale, w2, **how)
    out, nxt = T.join(x, y, w, gate, scale, w2, **how)
    _close(out, r["out"].v, r["out"].e, "out")
    _close(nxt, r["next"].v, r["next"].e, "next")
    want = _join_back_num(r, dout, dnext, gate, w2, True, "sigmoid", "rms")
    back = T.join_backward(dout, dnext, x, y, w, gate, scale, w2, **how)
    for name, value in back._asdict().items():
        _close(value, want[name].v, want[name].e, name)
    again = T.join_backward(dout, dnext, x, y, w, gate, scale, w2, **how)
    assert all(torch.equal(a, b) for a, b in zip(back, again))   # the same inputs, the same bits


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_gradients_against_differences(kind):
    """Of the formula in 64 bits, along a direction: (f(h) - f(-h)) / 2h is off by h^2 / 6 times the third derivative (a few units
    here: 1e-7 of the sum of magnitudes) and the gradient by its own rounding."""
    g = _gen(11)
    n, d, eps, h = 7, 45, 1e-3, 1e-4
    t = {"x": _r(g, n, d), "y": _r(g, n, d), "weight": _r(g, d, shift=1.0), "gate": _r(g, n, 1), "scale": _r(g, d), "next_weight": _r(g, d)}
    dout, dnext = _r(g, n, d), _r(g, n, d)

    def f(**v):
        v = {k: x.double() for k, x in v.items()}
        unit = lambda a: (a - (a.mean(1, keepdim=True) if kind == "layer" else 0)) / ((a - (a.mean(1, keepdim=True) if kind == "layer" else 0)).square().mean(1, keepdim=True) + eps).sqrt()  # noqa: E731
        out = v["x"] + v["scale"] * torch.sigmoid(v["gate"]) * unit(v["y"]) * v["weight"]
        return (out * dout.double()).sum() + (unit(out) * v["next_weight"] * dnext.double()).sum()

    back = T.join_backward(dout, dnext, *(t[k] for k in ("x", "y", "weight", "gate", "scale", "next_weight")), kind=kind, eps=eps)
    for i, name in enumerate(("x", "y", "weight", "gate", "scale", "next_weight")):
        along = torch.randn(t[name].shape, device="cuda", generator=g).double()
        moved = lambda s: f(**{**{k: v.double() for k, v in t.items()}, name: t[name].double() + s * along})  # noqa: E731
        slope, terms = (moved(h) - moved(-h)) / (2 * h), back[i].double() * along
        assert abs(float(terms.sum() - slope)) < 1e-5 * float(terms.abs().sum()) + 1e-4, name


def test_autograd():
    g = _gen(12)
    n, d = 50, 72
    x, y, gate = (_r(g, n, d, dtype=BF16).requires_grad_() for _ in range(3))
    w, scale, w2, w0 = (_r(g, d, shift=1.0).requires_grad_() for _ in range(4))
    k1, k2 = _r(g, n, d), _r(g, n, d)
    first = T.norm(x, w0, kind="layer", eps=1e-5)
    out, nxt = T.join(x, y, w, gate, scale, w2, kind="layer", eps=1e-5)
    (out.float() * k1 + nxt.float() * k2).sum().backward(retain_graph=True)
    back = T.join_backward(k1.to(BF16), k2.to(BF16), x.detach(), y.detach(), w.detach(), gate.detach(), scale.detach(), w2.detach(), kind="layer", eps=1e-5)
    for t, want in zip((x, y, w, gate, scale, w2), back):
        assert torch.equal(t.grad, want)
    x.grad = None
    first.sum().backward()   # (a sum's gradient is one element seen many times)
    dx, dw = T.norm_backward(torch.ones(n, d, dtype=BF16, device="cuda"), x.detach(), w0.detach(), kind="layer", eps=1e-5)
    assert torch.equal(x.grad, dx) and torch.equal(w0.grad, dw)
    # only one of the two results is used; only some inputs ask
    for used in (0, 1):
        a = y.detach().requires_grad_()
        got = T.join(x.detach(), a, w.detach(), None, 0.5, w2.detach())
        got[used].float().sum().backward()
        ones = torch.ones(n, d, dtype=BF16, device="cuda")
        want = T.join_backward(None if used else ones, ones if used else None, x.detach(), a.detach(), w.detach(), None, 0.5, w2.detach(), need=["y"])
        assert torch.equal(a.grad, want.dy) and want.dx is None
    with torch.no_grad():
        assert not T.norm(x, w0).requires_grad and not T.join(x, y, w).requires_grad
    with pytest.raises(B.FbxError):
        T.norm(x, w0, out=torch.zeros(n, d, dtype=BF16, device="cuda"))
    with pytest.raises(B.FbxError):
        T.join(x, y, w, out=torch.zeros(n, d, dtype=BF16, device="cuda"))


def test_rows_keep_to_themselves():
    """What is not finite stays in its row (and in the columns' sums); a row of zeros is one of zeros."""
    g = _gen(13)
    n, d = 6, 300
    x, y, w = _r(g, n, d), _r(g, n, d), _r(g, d, shift=1.0)
    clean = T.join(x, y, w, None, 1.0, w)
    x2, y2 = x.clone(), y.clone()
    x2[1, 7], y2[2, 299], y2[4, 0] = float("nan"), float("inf"), float("-inf")
    out, nxt = T.join(x2, y2, w, None, 1.0, w)
    for r in (0, 3, 5):
        assert torch.equal(out[r], clean[0][r]) and torch.equal(nxt[r], clean[1][r])
    assert torch.isnan(out[1]).sum() == 1 and torch.isnan(nxt[1]).all() and torch.isnan(out[2, 299]) and torch.isnan(out[4, 0])
    dx = T.norm_backward(y, x2, w)[0]
    assert torch.isnan(dx[1]).all() and torch.equal(dx[[0, 2, 3, 4, 5]], T.norm_backward(y, x, w)[0][[0, 2, 3, 4, 5]])
    zero = torch.zeros(n, d, device="cuda")
    for kind in ("rms", "layer"):
        assert not T.norm(zero, w, kind=kind).any()
        assert torch.equal(T.join(x, zero, w, None, 1.0, kind=kind), x)
        flat = T.norm_backward(y, zero, None, kind=kind)[0].double()   # unit is 0: the slope is 1 / sqrt(eps), less the mean
        want = (y.double() - (y.double().mean(1, keepdim=True) if kind == "layer" else 0)) * 1e3
        assert ((flat - want).abs() <= 1e3 * 70 * U32 * (y.double().abs() + y.double().abs().mean(1, keepdim=True))).all()
    big = torch.full((2, d), 3e4, device="cuda", dtype=F16)
    assert torch.equal(T.norm(big, None), torch.ones_like(big)) and not T.norm(big, None, kind="layer").any()


def test_no_records():
    x, w = torch.zeros(0, 40, device="cuda"), torch.ones(40, device="cuda")
    assert T.norm(x, w).shape == (0, 40)
    dx, dw = T.norm_backward(x, x, w)
    assert dx.shape == (0, 40) and not dw.any()
    out, nxt = T.join(x, x, w, x[:, :1], w, w)
    assert out.shape == nxt.shape == (0, 40)
    back = T.join_backward(x, x, x, x, w, x[:, :1], w, w)
    assert back.dgate.shape == (0, 1) and not any(v.any() for v in (back.dweight, back.dscale, back.dnext_weight))


def test_a_table_of_rows_beyond_32_bits():
    """Rows whose elements lie further apart than 32 bits reach."""
    d, far = 64, (1 << 31) + 24
    whole = torch.zeros(far + d, dtype=BF16, device="cuda")
    x = torch.as_strided(whole, (2, d), (far, 1))
    x.copy_(_r(_gen(14), 2, d, dtype=BF16))
    near = x.contiguous()
    assert torch.equal(T.norm(x), T.norm(near))
    assert torch.equal(T.join(x, x, None, x, 0.5), T.join(near, near, None, near, 0.5))
    T.norm(near, out=x)
    assert torch.equal(x, T.norm(near))


def test_results_over_inputs():
    """Where a result may lie over its input it is the same, and elsewhere it is refused."""
    g = _gen(15)
    for d in (5, 60, 411, 2624, 9001):
        x, w = _r(g, 37, d, dtype=BF16), _r(g, d, shift=1.0)
        want = T.norm(x, w, kind="layer")
        assert T.norm(x, w, kind="layer", out=x) is x and torch.equal(x, want)
    u = [_decaying(g, 30, 50), _decaying(g, 300, 200)]
    want = T.orthogonalise(u)
    T.orthogonalise(u, out=u)
    assert all(torch.equal(a, b) for a, b in zip(u, want))
    x, y, z = (_r(g, 4, 24) for _ in range(3))
    for call in (lambda: T.join(x, y, None, z, out=x), lambda: T.join(x, y, None, z, out=y), lambda: T.join(x, y, None, z, then=True, out_next=z),
                 lambda: T.join(x, y, then=True, out=z, out_next=z), lambda: T.orthogonalise([x, y], out=[y, x])):
        with pytest.raises(B.FbxError):
            call()


# ------------------------------------------------------------------ orthogonalised matrices
C = T.NEWTON_SCHULZ


def _ortho64(u, steps, coefficients=C, eps=1e-7):
    x = u.double()
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    x = x / (x.norm() + eps)
    a, b, c = coefficients
    for _ in range(steps):
        gram = torch.mm(x, x.t().contiguous())
        x = a * x + torch.mm(b * gram + c * torch.mm(gram, gram), x)
    return x.t() if tall else x


def _step_bound(x, ex, part, coefficients=C):
    """One step on an x that is off by ex, element by element: what it is off afterwards.  part: what a factor's parts leave out (2^-11 of a
    first part, 2^-21 of two); a held value is off by 2^-22 of itself, or the smallest step of f16 (2^-24) at a scale of 2^12 at least."""
    a, b, c = (abs(v) for v in coefficients)
    small = 2.0 ** -36
    product = lambda p, q, ep, eq: ep @ q + p @ eq + ep @ eq + (2 * part + (3 * p.shape[1] + 8) * U32) * (p @ q)  # noqa: E731
    m = x.abs()
    mt, et = m.t().contiguous(), ex.t().contiguous()
    gram, eg = m @ mt, product(m, mt, ex, et)
    eg = eg * (1 + part) + part * gram + small
    g2, eg2 = gram @ gram, product(gram, gram, eg, eg)
    poly = b * gram + c * g2 + a * torch.eye(len(gram), dtype=torch.float64, device="cuda")   # (a X is part of the product with X)
    ep = (b * eg + c * eg2) * (1 + 4 * U32) + (part + 8 * U32) * poly + small
    return product(poly, m, ep, ex) + 2.0 ** -21 * (poly @ m) + small


def _decaying(g, rows, columns, dtype=F32):
    n = min(rows, columns)
    s = torch.arange(1, n + 1, device="cuda").float().pow(-0.7)
    return ((_r(g, rows, n) * s) @ _r(g, n, columns) + 0.1 * _r(g, rows, columns)).to(dtype)


SIDES = [(1, 1), (1, 50), (50, 1), (2, 3), (63, 64), (64, 65), (65, 63), (100, 100), (129, 200), (200, 129), (64, 1000), (257, 300), (700, 130)]


@pytest.mark.parametrize("exact", [True, False])
@pytest.mark.parametrize("steps", [1, 2])
def test_orthogonalise_few_steps(steps, exact):
    g = _gen(20)
    given = [_decaying(g, r, c) for r, c in SIDES]
    got = T.orthogonalise([_pad(u, i % 3) for i, u in enumerate(given)], steps=steps, exact=exact)
    for u, o in zip(given, got):
        assert o.dtype == F32 and o.shape == u.shape
        x = u.double() if u.shape[0] <= u.shape[1] else u.double().t().contiguous()
        x = x / (x.norm() + 1e-7)
        ex = (2.0 ** -22 + 4 * U32) * x.abs() + 2.0 ** -36
        for _ in range(steps):
            ex = _step_bound(x, ex, 2.0 ** -21 if exact else 2.0 ** -11)
            x = _ortho64_step(x)
        want = x if u.shape[0] <= u.shape[1] else x.t()
        _close(o, want, ex if u.shape[0] <= u.shape[1] else ex.t(), f"{tuple(u.shape)} {steps} steps")


def _ortho64_step(x, coefficients=C):
    a, b, c = coefficients
    gram = torch.mm(x, x.t().contiguous())
    return a * x + torch.mm(b * gram + c * torch.mm(gram, gram), x)


@pytest.mark.parametrize("shape", [(16, 16), (20, 33), (96, 128), (128, 128), (64, 500), (31, 1000), (300, 200)])
def test_both_parts_are_those_of_one_number(shape):
    """An element's second part is what its first leaves; where the two were rounded from values a bit apart (one in some thousands, a unit of
    the first part) two steps are 4e-6 to 2e-5 off.  In the norm every one of eight roundings a step (X, A and B held, and a
    sum of each; each product's two factors) leaves 2^-22 at most, and two steps twice that: 3.8e-6."""
    for seed in range(12):
        u = _decaying(_gen(100 + seed), *shape)
        want = _ortho64(u, 2)
        off = float((T.orthogonalise(u, steps=2, exact=True).double() - want).norm() / want.norm())
        assert off <= 2 * 8 * 2.0 ** -22, (seed, off)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_orthogonalise(dtype):
    """Five steps.  A step's own error, in the norm, is that of its bound; every later step multiplies it by the polynomial's largest
    slope at most: max |a + 3 b s^2 + 5 c s^4| for s up to 1.25, which singular values stay below."""
    a, b, c = C
    s = torch.linspace(0, 1.25, 4001, dtype=torch.float64)
    slope = float((a + 3 * b * s ** 2 + 5 * c * s ** 4).abs().max())
    g = _gen(21)
    given = [_decaying(g, r, k, dtype) for r, k in SIDES]
    got = T.orthogonalise(given, dtype=F32)
    rounded = T.orthogonalise(given)
    for u, o, q in zip(given, got, rounded):
        x = u.double() if u.shape[0] <= u.shape[1] else u.double().t().contiguous()
        x = x / (x.norm() + 1e-7)
        off = float(((2.0 ** -22 + 4 * U32) * x.abs() + 2.0 ** -36).norm())
        for _ in range(5):
            off = off * slope * 1.01 + float(_step_bound(x, torch.zeros_like(x), 2.0 ** -21).norm())
            x = _ortho64_step(x)
        want = x if u.shape[0] <= u.shape[1] else x.t()
        assert float((o.double() - want).norm()) <= off + U32 * float(want.norm()), u.shape
        assert float((q.double() - want).norm()) <= max(off, 4e-3 * float(want.norm()) if dtype == BF16 else 0.0) + HALF_UNIT[dtype] * float(want.norm()), u.shape


@pytest.mark.parametrize("rows, columns, count", [(1024, 384, 9), (300, 2000, 2), (1500, 1400, 1), (2624, 4096, 1)])
def test_orthogonalise_large(rows, columns, count):
    """The sizes where tiles of 64, 128 and 256 are taken.  Products of 32-bit accuracy and in half precision, against 64 bits, in the
    norm: the first off by at most 1e-4 (what 32 bits leave, 2^-22 and a growth of 4 a step: 5e-5, and sums of thousands of terms), the
    second by the 4e-3 that is promised for results in bfloat16."""
    g = _gen(22)
    given = [_decaying(g, rows, columns) for _ in range(count)]
    for exact, dtype, most in ((True, F32, 1e-4), (False, BF16, 4e-3), (None, BF16, 4e-3)):
        got = T.orthogonalise(given, dtype=dtype, exact=exact)
        for u, o in zip(given, got):
            want = _ortho64(u, 5)
            assert float((o.double() - want).norm()) <= most * float(want.norm())
        assert all(torch.equal(p, q) for p, q in zip(got, T.orthogonalise(given, dtype=dtype, exact=exact)))   # the same bits


def test_orthogonalise_singular_values():
    """What the iteration is for: singular values that were not tiny end in [0.65, 1.25]."""
    g = _gen(23)
    u = _r(g, 200, 500, dtype=BF16)
    s = torch.linalg.svdvals(T.orthogonalise(u).double().cpu())
    assert 0.65 < float(s.min()) and float(s.max()) < 1.25


def test_orthogonalise_low_rank():
    """A few large directions and little noise: the noise's singular values grow 485 times, and rounding may not stand in for them."""
    g = _gen(24)
    u = _r(g, 384, 8) @ _r(g, 8, 1024) + 0.01 * _r(g, 384, 1024)
    want = _ortho64(u, 5)
    for exact in (True, False):
        o = T.orthogonalise(u, exact=exact, dtype=BF16)
        assert float((o.double() - want).norm()) <= 4e-3 * float(want.norm())


def test_orthogonalise_extremes():
    zero, one = torch.zeros(30, 40, device="cuda"), torch.zeros(30, 40, device="cuda")
    one[3, 5] = 2.5
    nan, inf = _r(_gen(25), 30, 40), _r(_gen(25), 30, 40)
    nan[2, 2], inf[29, 39] = float("nan"), float("inf")
    tiny, huge = _r(_gen(26), 30, 40) * 1e-30, _r(_gen(26), 30, 40) * 1e30
    got = T.orthogonalise([zero, one, nan, inf, tiny, huge], eps=1e-30)
    assert not got[0].any()
    want = _ortho64(one, 5)
    assert ((got[1].double() - want).abs() <= 1e-5).all() and not got[1].bool().sum() > 1
    assert torch.isnan(got[2]).all() and torch.isnan(got[3]).all()
    plain = _ortho64(_r(_gen(26), 30, 40), 5, eps=0.0)
    assert float((got[5].double() - plain).norm()) <= 1e-4 * float(plain.norm())
    assert float((got[4].double() - _ortho64(tiny, 5, eps=1e-30)).norm()) <= 1e-4 * float(plain.norm())
    many = torch.ones(65, 66, device="cuda", dtype=F16) * 6e4   # one direction
    assert float((T.orthogonalise(many, dtype=F32).double() - _ortho64(many, 5)).norm()) <= 1e-4
    empty = T.orthogonalise([torch.zeros(0, 5, device="cuda"), torch.zeros(5, 0, device="cuda")])
    assert [tuple(e.shape) for e in empty] == [(0, 5), (5, 0)]


def test_orthogonalise_coefficients_and_results():
    g = _gen(27)
    u = _decaying(g, 90, 120)
    schedule = [(3.4445, -4.7750, 2.0315), (2.0, -1.5, 0.5), (1.875, -1.25, 0.375)]
    x = u.double() / (u.double().norm() + 1e-7)
    for c in schedule:
        x = _ortho64_step(x, c)
    got = T.orthogonalise(u, steps=3, coefficients=schedule)
    assert float((got.double() - x).norm()) <= 1e-4 * float(x.norm())
    into = _pad(torch.zeros(120, 90, device="cuda", dtype=F16), 5)
    assert T.orthogonalise(u.t().contiguous(), steps=3, coefficients=schedule, dtype=F16, out=into) is into
    assert float((into.double() - x.t()).norm()) <= (1e-4 + 2.0 ** -11) * float(x.norm()) and torch.isnan(into._base[:, 90:]).all()
    with pytest.raises(B.FbxError):
        T.orthogonalise([u, u], out=[torch.zeros_like(u)] * 2)


def test_orthogonalise_more_matrices_than_a_launch_holds():
    g = _gen(28)
    given = [_decaying(g, 20 + i, 33) for i in range(70)]
    got = T.orthogonalise(given)
    assert all(torch.equal(o, T.orthogonalise(u)) for u, o in zip(given, got))


# ------------------------------------------------------------------ Muon
@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("param, grad, copy", [(F32, F32, BF16), (F32, BF16, F16), (F32, F16, None), (BF16, BF16, None), (F16, F32, None), (BF16, F32, None)])
def test_muon(param, grad, copy, nesterov):
    g = _gen(30)
    shapes = [(1, 7), (7, 1), (33, 65), (130, 70), (64, 192), (400, 300)]
    p, d = [_r(g, *s, dtype=param, size=0.2) for s in shapes], [_decaying(g, *s, grad) for s in shapes]
    m = [_decaying(g, *s) for s in shapes]
    copies = None if copy is None else [torch.zeros(s, dtype=copy, device="cuda") for s in shapes]
    p0, m0 = [t.clone() for t in p], [t.clone() for t in m]
    lr, momentum, decay, scale = 0.05, 0.9, 0.1, 0.5
    T.muon(p, d, m, copies, lr=lr, momentum=momentum, nesterov=nesterov, weight_decay=decay, grad_scale=scale)
    for i, s in enumerate(shapes):
        gs = d[i].float() * scale
        want_m = m0[i] * momentum + gs                     # (in 32 bits, each operation rounded: the same bits)
        assert torch.equal(m[i], want_m), s
        u = gs.double() + want_m.double() * float(torch.tensor(momentum, dtype=F32)) if nesterov else want_m.double()
        o = _ortho64(u, 5)
        step = lr * 0.2 * math.sqrt(max(s))
        want = p0[i].double() * (1 - lr * decay) - step * o
        # elements of o off by what the orthogonalised matrix may be (`test_orthogonalise`): 1e-4 of its norm, 4e-3 with bf16 weights
        off = step * (4e-3 if param == BF16 else 1e-4) * o.norm() + 4 * U32 * (p0[i].double().abs() + step * o.abs())
        _close(p[i], want, off.expand(s), f"weights {s}")
        if copies is not None:
            _close(copies[i], want, off.expand(s), f"copy {s}")


def test_muon_class():
    g = _gen(31)
    shapes = [(40, 60), (60, 40), (33, 33)]
    start = [_r(g, *s) for s in shapes]
    a, b = ([w.clone().requires_grad_() for w in start] for _ in range(2))
    copies = [torch.zeros(s, dtype=BF16, device="cuda") for s in shapes]
    one, other = T.Muon(a, lr=0.01, copies=copies), T.Muon(b, lr=0.01)
    m = [torch.zeros(s, device="cuda") for s in shapes]
    mine = [w.clone() for w in start]
    for k in range(4):
        grads = [_decaying(g, *s) for s in shapes]
        if k == 2:
            other.load_state_dict({key: v for key, v in one.state_dict().items()})
            for x, y in zip(b, a):
                x.data.copy_(y.data)
        skip = 1 if k == 1 else None
        for i, (w, d) in enumerate(zip(a, grads)):
            w.grad = None if i == skip else d.clone()
        one.step(grad_scale=0.5)
        if k >= 2:
            other.step(grads, grad_scale=0.5)
        at = [i for i in range(3) if i != skip]
        T.muon([mine[i] for i in at], [grads[i] for i in at], [m[i] for i in at], lr=0.01, grad_scale=0.5)
        assert all(torch.equal(x, y) for x, y in zip(a, mine)) and all(torch.equal(x, y) for x, y in zip(one.m, m))
        assert all(torch.equal(c, w.to(BF16)) for i, (c, w) in enumerate(zip(copies, a)) if i != skip)
    assert all(torch.equal(x, y) for x, y in zip(a, b)) and one.step_count == 4 and other.step_count == 4
    one.zero_grad()
    assert all(w.grad is None for w in a)


def test_muon_steps_all_or_none_and_notes_changes():
    w = [torch.ones(4, 6, device="cuda"), torch.ones(4, 6, device="cuda", dtype=BF16)]
    opt = T.Muon(w)
    good = [torch.ones(4, 6, device="cuda"), torch.ones(4, 6, device="cuda", dtype=BF16)]
    versions = [t._version for t in (*w, *opt.m)]
    for bad in (torch.ones(4, 5, device="cuda", dtype=BF16), torch.ones(6, 4, device="cuda", dtype=BF16).t()):
        with pytest.raises(B.FbxError):
            opt.step([good[0], bad])
        assert (w[0] == 1).all() and not opt.m[0].any() and opt.step_count == 0
    opt.step(good)
    assert all(t._version > v for t, v in zip((*w, *opt.m), versions))
    assert (w[0] != 1).all() and all(m.all() for m in opt.m)   # (the step is less than half a unit of the bfloat16 weights)


# ------------------------------------------------------------------ all of them as a trunk takes them
class Trunk:
    """Two blocks behind pooled rows: norm -> gated -> a product back -> join (with the next norm) -> ..."""

    def __init__(self, g, width, hidden, dtype=BF16):
        r = lambda a, b: _r(g, a, b, dtype=dtype, size=1 / math.sqrt(b)).requires_grad_()  # noqa: E731
        v = lambda value: torch.full((width,), value, device="cuda").requires_grad_()  # noqa: E731
        self.blocks = [dict(gate=r(hidden, width), up=r(hidden, width), down=r(width, hidden), open=r(width, width), post=v(1.0), scale=v(0.5), next=v(1.0)) for _ in range(2)]
        self.first = v(1.0)
        self.matrices = [b[k] for b in self.blocks for k in ("gate", "up", "down", "open")]
        self.vectors = [self.first] + [b[k] for b in self.blocks for k in ("post", "scale", "next")]

    def __call__(self, x, ops=T):
        h = ops.norm(x, self.first)
        for b in self.blocks:
            y = ops.gated(h, b["gate"], b["up"]) @ b["down"].t()
            x, h = ops.join(x, y, b["post"], h @ b["open"].t(), b["scale"], b["next"])
        return x, h


class Plain:
    """The same in torch's own operations, in the inputs' type's products and 64 bits beside them."""

    @staticmethod
    def norm(x, w):
        x = x.double()
        return x * (x.square().mean(1, keepdim=True) + 1e-6).rsqrt() * w.double()

    @staticmethod
    def gated(h, gate, up):
        return torch.nn.functional.silu(h @ gate.double().t()) * (h @ up.double().t())

    @staticmethod
    def join(x, y, post, z, scale, nxt):
        out = x.double() + scale.double() * torch.sigmoid(z) * Plain.norm(y, post)
        return out, Plain.norm(out, nxt)


def test_trunk_learns_as_in_64_bits():
    """Forward and gradients in float32 against 64 bits, on the CPU, of a chain of 14 operators: 1e-4 of each gradient's norm is 1,700
    half units of 32 bits, for sums of at most 512 terms each that the chain adds up."""
    g = _gen(40)
    x = _r(g, 200, 96)
    trunk = Trunk(g, 96, 128, F32)
    k = _r(g, 200, 96)
    out, h = trunk(x)
    (out * k).sum().backward()
    mine = [t.grad.double().cpu() for t in trunk.matrices + trunk.vectors if t.grad is not None]
    asked = [t for t in trunk.matrices + trunk.vectors if t.grad is not None]
    assert len(asked) == len(trunk.matrices) + len(trunk.vectors) - 1   # (the last norm's weights lead nowhere)
    host = Trunk(_gen(41), 96, 128, F32)
    for b, c in zip(host.blocks, trunk.blocks):
        for key in b:
            b[key] = c[key].detach().double().cpu().requires_grad_()
    host.first = trunk.first.detach().double().cpu().requires_grad_()
    blocks = host.blocks
    a, hh = x.double().cpu(), Plain.norm(x.cpu(), host.first)
    for b in blocks:
        y = Plain.gated(hh, b["gate"], b["up"]) @ b["down"].t()
        a, hh = Plain.join(a, y, b["post"], hh @ b["open"].t(), b["scale"], b["next"])
    (a * k.double().cpu()).sum().backward()
    assert float((out.detach().double().cpu() - a.detach()).norm()) <= 1e-5 * float(a.detach().norm())
    want = [b[key].grad for b in blocks for key in ("gate", "up", "down", "open")] + [host.first.grad] + [b[key].grad for b in blocks for key in ("post", "scale", "next") if b[key].grad is not None]
    for got, ref in zip(mine, want):
        assert float((got - ref).norm()) <= 1e-4 * float(ref.norm())


def test_training_steps_on_another_stream_and_in_a_graph():
    g = _gen(42)
    x, k = _r(g, 120, 80, dtype=BF16), _r(g, 120, 80)

    def start():
        t = Trunk(_gen(43), 80, 96)
        return t, T.Muon(t.matrices, lr=0.01), T.AdamW(t.vectors, lr=0.01)

    def steps(n):
        trunk, muon, adamw = start()
        for _ in range(n):
            out, h = trunk(x)
            ((out.float() + h.float()) * k).sum().backward()
            muon.step()
            adamw.step()
            muon.zero_grad()
            adamw.zero_grad()
        return [t.detach() for t in trunk.matrices + trunk.vectors] + muon.m

    want = steps(3)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = steps(3)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))

    # captured by hand: forward functions, their gradients and the updates, replayed among eager work
    w = _r(g, 80, shift=1.0)
    d = dict(p=[_r(g, 80, 96), _r(g, 300, 70)], m=[torch.zeros(80, 96, device="cuda"), torch.zeros(300, 70, device="cuda")])
    grads = [_decaying(g, 80, 96), _decaying(g, 300, 70)]

    def work(d):
        h = T.norm(x, w)
        out, nxt = T.join(x, h, w, x, w, w)
        back = T.join_backward(out, nxt, x, h, w, x, w, w)
        dx, dw = T.norm_backward(back.dy, x, w)
        T.muon(d["p"], grads, d["m"])
        return [h, out, nxt, *back, dx, dw, *d["p"], *d["m"], T.orthogonalise(grads[1], dtype=BF16)]

    mine, other = ({key: [t.clone() for t in v] for key, v in d.items()} for _ in range(2))
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        work({key: [t.clone() for t in v] for key, v in d.items()})
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = work(mine)
    for _ in range(4):
        graph.replay()
        eager = work(other)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, eager))


def test_autograd_in_a_graph():
    """Forward and backward through autograd, captured where no eager graph of the leaves is alive, and replayed among eager work on new inputs."""
    g = _gen(45)
    shapes, vectors = [(70, 411), (70, 411), (70, 1)], [(411,)] * 3
    leaves = [_r(g, *shape, dtype=BF16).requires_grad_() for shape in shapes] + [_r(g, *shape, shift=1.0).requires_grad_() for shape in vectors]
    ends = [_r(g, 70, 411, dtype=BF16) for _ in range(2)]

    def work():
        x, y, gate, *w = leaves
        out, nxt = T.join(x, T.norm(y, w[0], kind="layer"), w[1], gate, 0.5, w[2])
        return [out.detach(), nxt.detach(), *torch.autograd.grad([out, nxt], leaves, ends)]

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        work()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = work()
    for i in range(4):
        with torch.no_grad():
            for t in leaves + ends:
                t.mul_(1.0 + 0.25 * i)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in captured]
        assert all(torch.equal(a, b) for a, b in zip(got, work()))


def test_results_over_other_inputs_are_refused():
    """What lies over an input in a way that a row may be written before it is read, or a matrix that is both read and written, is refused."""
    g = _gen(46)
    both = _r(g, 8, 60)
    x, w = both[:4, :24], _r(g, 1, 24)
    shorter = torch.as_strided(both, (4, 24), (30, 1))
    p = [_r(g, 8, 9) for _ in range(3)]
    for call in (lambda: T.norm(x, out=shorter), lambda: T.norm(x.contiguous(), w[0], out=x.contiguous()[:3]), lambda: T.norm(x[:1], w[0], out=w), lambda: T.join(x[:1], x[:1], w[0], out=w),
                 lambda: T.join(x[:1], x[:1], None, None, w[0], out=w), lambda: T.join(x[:1], x[:1], None, None, 0.5, w[0], out_next=w), lambda: T.norm(x, out=x.view(BF16)[:, :24], dtype=BF16),
                 lambda: T.muon([p[0]], [p[0]], [p[1]]), lambda: T.muon([p[0]], [p[1]], [p[1]]), lambda: T.muon([p[0], p[1]], [p[2], p[0]], [torch.zeros(8, 9, device="cuda") for _ in range(2)])):
        before = [t.clone() for t in (both, w, *p)]
        with pytest.raises(B.FbxError) as e:
            call()
        assert e.value.status == B.E_ARG and all(torch.equal(a, b) for a, b in zip(before, (both, w, *p)))
    assert T.norm(x[:1], w[0], out=torch.as_strided(both, (1, 24), (30, 1))) is not None   # (one row: its stride says nothing)


def test_orthogonalise_many_steps():
    """As many steps as there may be, of coefficients that take every singular value to 1: what is left is off by the last steps'
    roundings and by what the first ones left in the directions of the smallest singular value (a 2^-21 of each product, 2 sqrt(rows) of
    them in a norm, over that value, which the steps make 1.875 times larger each: less than 3 times the first)."""
    g = _gen(47)
    for rows, columns in ((48, 80), (200, 320)):
        u = _r(g, rows, columns)
        d = u.double().cpu()
        left, s, right = torch.linalg.svd(d, full_matrices=False)
        want = (left @ right).cuda()
        small = float(s[-1] / d.norm())
        got = T.orthogonalise(u, steps=64, coefficients=(1.875, -1.25, 0.375))
        assert float((got.double() - want).norm()) <= 3 * 8 * 2.0 ** -21 * 2 * rows ** 0.5 / small


def test_two_threads_at_once():
    """Two calls at a time, on streams of their own: neither's results depend on the other."""
    g = _gen(44)
    x, w = _r(g, 500, 700), _r(g, 700, shift=1.0)
    u = [_decaying(g, 100, 150), _decaying(g, 300, 40)]
    want = (*T.join(x, x, w, x, 0.5, w), *T.orthogonalise(u))
    torch.cuda.synchronize()
    got, wrong = [None, None], []

    def work(i):
        try:
            s = torch.cuda.Stream()
            with torch.cuda.stream(s):
                for _ in range(10):
                    got[i] = (*T.join(x, x, w, x, 0.5, w), *T.orthogonalise(u))
            s.synchronize()
        except Exception as e:  # noqa: BLE001
            wrong.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not wrong
    for mine in got:
        assert all(torch.equal(a, b) for a, b in zip(mine, want))
