"""Norms, joins, orthogonalised updates and Muon without a GPU: bad arguments are refused before any work, by the C ABI and by the
Python entry points."""
import ctypes

import pytest
import torch

from paper_2210_07768_amd import binding as B
from paper_2210_07768_amd import train as T

vp, u64, u32, i32, f64 = ctypes.c_void_p, ctypes.c_uint64, ctypes.c_uint32, ctypes.c_int, ctypes.c_double
P = 4096   # an address that no call here reads


class Norm(ctypes.Structure):
    _fields_ = [("records", u64), ("dim", u32), ("kind", i32), ("stream", i32), ("block", i32), ("vectors", i32), ("eps", f64), ("d_x", vp), ("d_weight", vp), ("ld_x", u64)]


class Join(ctypes.Structure):
    _fields_ = [("records", u64), ("dim", u32), ("kind", i32), ("stream", i32), ("block", i32), ("vectors", i32), ("gate_act", i32), ("gate_columns", u32), ("post", i32),
                ("eps", f64), ("scale", f64), ("d_x", vp), ("d_y", vp), ("d_gate", vp), ("d_weight", vp), ("d_scale", vp), ("d_next_weight", vp),
                ("ld_x", u64), ("ld_y", u64), ("ld_gate", u64)]


class Gradients(ctypes.Structure):
    _fields_ = [(n, vp) for n in ("d_dout", "d_dnext", "d_dx", "d_dy", "d_dgate", "d_dweight", "d_dscale", "d_dnext_weight")] + [
        (n, u64) for n in ("ld_dout", "ld_dnext", "ld_dx", "ld_dy", "ld_dgate")]


class OrthoMatrix(ctypes.Structure):
    _fields_ = [("d_u", vp), ("d_out", vp), ("ld_u", u64), ("ld_out", u64), ("rows", u32), ("columns", u32)]


class Ortho(ctypes.Structure):
    _fields_ = [("in_", i32), ("out", i32), ("exact", u32), ("steps", u32), ("coefficients", ctypes.POINTER(f64)), ("eps", f64)]


class MuonMatrix(ctypes.Structure):
    _fields_ = [("d_param", vp), ("d_grad", vp), ("d_m", vp), ("d_copy", vp), ("rows", u32), ("columns", u32), ("factor", f64)]


class Muon(ctypes.Structure):
    _fields_ = [("ortho", Ortho), ("param_dtype", i32), ("grad_dtype", i32), ("copy_dtype", i32), ("nesterov", i32), ("lr", f64), ("momentum", f64), ("weight_decay", f64),
                ("grad_scale", f64)]


def _library():
    L = B.lib()
    p = ctypes.POINTER
    L.fbx_train_last_error.restype = ctypes.c_char_p
    L.fbx_train_last_error.argtypes = []
    L.fbx_norm_forward.argtypes = [p(Norm), vp, u64, vp]
    L.fbx_norm_scratch.argtypes = [p(Norm), p(u64)]
    L.fbx_norm_backward.argtypes = [p(Norm), vp, u64, vp, u64, vp, vp, u64, vp]
    L.fbx_join_forward.argtypes = [p(Join), vp, u64, vp, u64, vp]
    L.fbx_join_scratch.argtypes = [p(Join), p(u64)]
    L.fbx_join_backward.argtypes = [p(Join), p(Gradients), vp, u64, vp]
    L.fbx_ortho_scratch.argtypes = [p(Ortho), p(OrthoMatrix), u32, p(u64)]
    L.fbx_orthogonalise.argtypes = [p(Ortho), p(OrthoMatrix), u32, vp, u64, vp]
    L.fbx_muon_scratch.argtypes = [p(Muon), p(MuonMatrix), u32, p(u64)]
    L.fbx_muon_step.argtypes = [p(Muon), p(MuonMatrix), u32, vp, u64, vp]
    return L


def _why():
    return _library().fbx_train_last_error().decode()


def _made(kind, defaults, change):
    values = {**defaults, **change}
    return kind(**{("in_" if k == "in" else k): v for k, v in values.items()})


NORM = dict(records=8, dim=24, kind=0, stream=0, block=0, vectors=0, eps=1e-6, d_x=P, d_weight=P, ld_x=24)
TYPES = [(dict(stream=3), "dtype"), (dict(block=-1), "dtype"), (dict(vectors=7), "dtype"), (dict(stream=1, block=2), "stream"), (dict(stream=1, block=0), "stream"),
         (dict(vectors=1), "vectors"), (dict(stream=2, block=2, vectors=1), "vectors")]
SIZES = [(dict(dim=0), "dim"), (dict(dim=T.NORM_MOST + 1, ld_x=1 << 20, ld_y=1 << 20), "dim"), (dict(records=1 << 40), "records"), (dict(kind=2), "kind"), (dict(eps=0.0), "eps"),
         (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(eps=float("inf")), "eps"), (dict(eps=1e-60), "eps"), (dict(ld_x=23), "ld_x"), (dict(ld_x=1 << 40), "ld_x"),
         (dict(d_x=None), "d_x"), (dict(d_x=P + 1), "aligned"), (dict(d_weight=P + 2), "aligned")]


@pytest.mark.parametrize("change, why", TYPES + [(c, w) for c, w in SIZES])
def test_norm_refuses(change, why):
    L, h = _library(), _made(Norm, NORM, {k: v for k, v in change.items() if k != "ld_y"})
    assert L.fbx_norm_forward(h, P, 1 << 21, None) == B.E_ARG and why in _why()
    assert L.fbx_norm_backward(h, P, 1 << 21, P, 1 << 21, P, P, 1 << 40, None) == B.E_ARG and why in _why()


def test_norm_refuses_results_and_scratch():
    L, need, h = _library(), u64(), _made(Norm, NORM, {})
    assert L.fbx_norm_forward(None, P, 24, None) == B.E_ARG
    assert L.fbx_norm_forward(h, None, 24, None) == B.E_ARG and "d_out" in _why()
    assert L.fbx_norm_forward(h, P, 23, None) == B.E_ARG and "ld_out" in _why()
    assert L.fbx_norm_forward(_made(Norm, NORM, dict(records=0)), None, 24, None) == B.OK   # nothing to do
    assert L.fbx_norm_scratch(h, None) == B.E_ARG
    assert L.fbx_norm_scratch(h, ctypes.byref(need)) == B.OK and need.value > 0
    back = lambda dy=P, ld=24, dx=P, ld_dx=24, dw=P, scratch=P, size=need.value: L.fbx_norm_backward(h, dy, ld, dx, ld_dx, dw, scratch, size, None)  # noqa: E731
    assert back(dy=None) == B.E_ARG and back(ld=23) == B.E_ARG and back(ld_dx=23) == B.E_ARG and back(dw=P + 2) == B.E_ARG
    assert back(scratch=None) == B.E_ARG and back(scratch=P + 8) == B.E_ARG and back(size=need.value - 1) == B.E_NOMEM
    assert back(dx=None, dw=None, scratch=None, size=0) == B.OK   # nothing is asked for


JOIN = dict(records=8, dim=24, kind=1, stream=0, block=0, vectors=0, gate_act=1, gate_columns=24, post=1, eps=1e-6, scale=1.0, d_x=P, d_y=P, d_gate=P, d_weight=P, d_scale=P,
            d_next_weight=P, ld_x=24, ld_y=24, ld_gate=24)
GRADIENTS = dict(d_dout=P, d_dnext=P, d_dx=P, d_dy=P, d_dgate=P, d_dweight=P, d_dscale=P, d_dnext_weight=P, ld_dout=24, ld_dnext=24, ld_dx=24, ld_dy=24, ld_dgate=24)


@pytest.mark.parametrize("change, why", TYPES + SIZES + [
    (dict(gate_act=2), "gate_act"), (dict(gate_columns=2), "gate_columns"), (dict(gate_columns=0), "gate_columns"), (dict(ld_gate=23), "ld_gate"), (dict(d_gate=P + 1), "aligned"),
    (dict(ld_y=23), "ld_y"), (dict(d_y=None), "d_y"), (dict(d_y=P + 2), "aligned"), (dict(post=0), "post"), (dict(scale=float("nan")), "scale"), (dict(scale=1e300), "scale"),
    (dict(d_scale=P + 2), "aligned"), (dict(d_next_weight=P + 1), "aligned")])
def test_join_refuses(change, why):
    L, h = _library(), _made(Join, JOIN, change)
    assert L.fbx_join_forward(h, P, 1 << 21, P, 1 << 21, None) == B.E_ARG and why in _why()
    wide = {k: 1 << 21 for k in GRADIENTS if k.startswith("ld")}
    assert L.fbx_join_backward(h, _made(Gradients, GRADIENTS, wide), P, 1 << 40, None) == B.E_ARG and why in _why()


def test_join_refuses_results_and_scratch():
    L, need, h = _library(), u64(), _made(Join, JOIN, {})
    assert L.fbx_join_forward(None, P, 24, None, 0, None) == B.E_ARG
    assert L.fbx_join_forward(h, None, 24, None, 0, None) == B.E_ARG and "d_out" in _why()
    assert L.fbx_join_forward(h, P, 23, None, 0, None) == B.E_ARG and "ld_out" in _why()
    assert L.fbx_join_forward(h, P, 24, P, 23, None) == B.E_ARG and "ld_next" in _why()
    assert L.fbx_join_forward(_made(Join, JOIN, dict(records=0)), None, 24, None, 0, None) == B.OK
    assert L.fbx_join_scratch(h, None) == B.E_ARG
    assert L.fbx_join_scratch(h, ctypes.byref(need)) == B.OK and need.value > 0
    back = lambda scratch=P, size=need.value, h=h, **change: L.fbx_join_backward(h, _made(Gradients, GRADIENTS, change), scratch, size, None)  # noqa: E731
    for k in GRADIENTS:
        if k.startswith("ld"):
            assert back(**{k: 23}) == B.E_ARG and k in _why()
        else:
            assert back(**{k: P + 2}) == B.E_ARG and "aligned" in _why()
    assert back(d_dout=None, d_dnext=None) == B.E_ARG
    assert back(h=_made(Join, JOIN, dict(d_gate=None))) == B.E_ARG and "gate" in _why()
    assert back(scratch=None) == B.E_ARG and back(scratch=P + 8) == B.E_ARG and back(size=need.value - 1) == B.E_NOMEM
    assert L.fbx_join_backward(h, None, P, need.value, None) == B.E_ARG
    assert L.fbx_join_backward(h, Gradients(d_dout=P, ld_dout=24), None, 0, None) == B.OK   # nothing is asked for


C3 = (3.4445, -4.7750, 2.0315)


def _ortho(steps=2, coefficients=C3, **change):
    a = dict(exact=1, eps=1e-7, **{"in": 0, "out": 0})
    a.update(change)
    n = steps if steps and steps < 65 else 1
    return _made(Ortho, a, dict(steps=steps, coefficients=None if coefficients is None else (f64 * (3 * n))(*(coefficients * n))))


MATRIX = dict(d_u=P, d_out=P, ld_u=6, ld_out=6, rows=4, columns=6)


@pytest.mark.parametrize("change, matrix, why", [
    (dict(steps=0), {}, "steps"), (dict(steps=65), {}, "steps"), (dict(coefficients=None), {}, "coefficients"), (dict(coefficients=(1.0, float("nan"), 0.0)), {}, "finite"),
    (dict(coefficients=(4.0, 0.0, 0.0)), {}, "beyond 3"), (dict(coefficients=(1.0, 300.0, 0.0)), {}, "beyond"), (dict(exact=3), {}, "exact"), (dict(eps=0.0), {}, "eps"),
    (dict(eps=float("nan")), {}, "eps"), (dict(out=3), {}, "dtype"), ({"in": -1}, {}, "dtype"), ({}, dict(rows=0), "rows"), ({}, dict(columns=(1 << 16) + 1, ld_u=1 << 17), "rows"),
    ({}, dict(ld_u=5), "stride"), ({}, dict(ld_out=5), "stride"), ({}, dict(ld_out=1 << 40), "stride"), ({}, dict(d_u=None), "NULL"), ({}, dict(d_out=None), "NULL"),
    ({}, dict(d_u=P + 2), "aligned"), ({}, dict(d_out=P + 1), "aligned")])
def test_orthogonalise_refuses(change, matrix, why):
    m = (OrthoMatrix * 2)(_made(OrthoMatrix, MATRIX, {}), _made(OrthoMatrix, MATRIX, matrix))
    assert _library().fbx_orthogonalise(_ortho(**change), m, 2, P, 1 << 40, None) == B.E_ARG and why in _why(), _why()


def test_orthogonalise_refuses_lists_and_scratch():
    L, need, m = _library(), u64(), (OrthoMatrix * 1)(_made(OrthoMatrix, MATRIX, dict(rows=300, columns=400, ld_u=400, ld_out=400)))   # (more than needs no scratch)
    assert L.fbx_orthogonalise(None, m, 1, P, 1 << 40, None) == B.E_ARG
    assert L.fbx_orthogonalise(_ortho(), None, 1, P, 1 << 40, None) == B.E_ARG
    assert L.fbx_orthogonalise(_ortho(), None, 0, None, 0, None) == B.OK   # nothing to do
    assert L.fbx_ortho_scratch(_ortho(), m, 1, None) == B.E_ARG
    assert L.fbx_ortho_scratch(_ortho(), m, 1, ctypes.byref(need)) == B.OK and need.value > 0
    for scratch, size, status in ((None, need.value, B.E_ARG), (P + 8, need.value, B.E_ARG), (P, need.value - 1, B.E_NOMEM)):
        assert L.fbx_orthogonalise(_ortho(), m, 1, scratch, size, None) == status


MUON_MATRIX = dict(d_param=P, d_grad=P, d_m=P, d_copy=None, rows=4, columns=6, factor=1.0)


@pytest.mark.parametrize("change, matrix, why", [
    (dict(param_dtype=3), {}, "dtype"), (dict(grad_dtype=-1), {}, "dtype"), (dict(momentum=1.0), {}, "momentum"), (dict(momentum=-0.1), {}, "momentum"), (dict(lr=float("inf")), {}, "lr"),
    (dict(weight_decay=float("nan")), {}, "lr"), (dict(grad_scale=1e300), {}, "lr"), (dict(ortho=dict(steps=0)), {}, "steps"), ({}, dict(rows=0), "rows"), ({}, dict(d_param=None), "lacks"),
    ({}, dict(d_grad=None), "lacks"), ({}, dict(d_m=None), "lacks"), ({}, dict(d_param=P + 2), "aligned"), ({}, dict(d_m=P + 2), "aligned"), ({}, dict(factor=float("nan")), "factor"),
    ({}, dict(d_copy=P), "either"), (dict(copy_dtype=0), dict(d_copy=P), "copy"), (dict(param_dtype=2), dict(d_copy=P), "copy")])
def test_muon_refuses(change, matrix, why):
    a = dict(param_dtype=0, grad_dtype=0, copy_dtype=2, nesterov=1, lr=1e-3, momentum=0.95, weight_decay=0.0, grad_scale=1.0, ortho={})
    a.update(change)
    h = Muon(**{**a, "ortho": _ortho(**a["ortho"])})
    m = (MuonMatrix * 2)(_made(MuonMatrix, MUON_MATRIX, {}), _made(MuonMatrix, MUON_MATRIX, matrix))
    assert _library().fbx_muon_step(h, m, 2, P, 1 << 40, None) == B.E_ARG and why in _why(), _why()
    assert _library().fbx_muon_step(None, m, 2, P, 1 << 40, None) == B.E_ARG
    assert _library().fbx_muon_scratch(h, m, 2, None) == B.E_ARG


def test_python_entry_points_refuse():
    x, w, d = torch.zeros(4, 6), torch.ones(6), dict(params=[torch.zeros(4, 6)], grads=[torch.zeros(4, 6)], momenta=[torch.zeros(4, 6)])
    norm, join, back, muon = T.norm, T.join, T.join_backward, lambda **k: T.muon(**{**d, **k})
    for call in (lambda: norm(x, w), lambda: norm([1.0]), lambda: norm(x.double()), lambda: norm(x, w.double()), lambda: norm(x, w[:5]), lambda: norm(x, torch.ones(6, 1)), lambda: norm(x[0]),
                 lambda: norm(x, torch.ones(12)[::2]), lambda: norm(x.t()), lambda: norm(x, w, kind="batch"), lambda: norm(x, w, eps=0.0), lambda: norm(x, w, dtype=torch.float64),
                 lambda: norm(x, w, dtype="float16"), lambda: norm(x, w, out=x[:, :5]), lambda: norm(x, w, out=x.half()), lambda: norm(x[:, :0]), lambda: norm(x, None, kind=None),
                 lambda: norm(torch.zeros(1, T.NORM_MOST + 1)), lambda: norm(x, w, dtype=torch.float16, out=x), lambda: T.norm_backward(x[:3], x, w), lambda: T.norm_backward(x, None, w),
                 lambda: join(x, x, w), lambda: join(x, x[:3], w), lambda: join(x.half(), x, w), lambda: join(x.half(), x.bfloat16()), lambda: join(x, x, w, x[:, :2]), lambda: join(x, x, w, x[:3]),
                 lambda: join(x, x, w, x.half()), lambda: join(x, x, w, x, w[:5]), lambda: join(x, x, w, scale=w.half()), lambda: join(x, x, w, next_weight=w, then=False), lambda: join(x, x, w, post=False),
                 lambda: join(x, x, w, gate_act="tanh"), lambda: join(x, x, w, kind=""), lambda: join(x, x, w, out_next=x), lambda: join(x, x, w, scale=float("inf")), lambda: join(x, None),
                 lambda: join(x, x, w, x[:, :1].expand(4, 1)[:1].expand(4, 1)), lambda: back(None, None, x, x, w), lambda: back(x, x, x, x, w), lambda: back(x, None, x, x, w, need=["z"]),
                 lambda: back(x.half(), None, x, x, w), lambda: back(x, x[:2], x, x, w, next_weight=w), lambda: T.orthogonalise(x), lambda: T.orthogonalise(x[0]), lambda: T.orthogonalise([x, x.half()]),
                 lambda: T.orthogonalise(x, steps=0), lambda: T.orthogonalise(x, coefficients=(1, 2)), lambda: T.orthogonalise(x, steps=2, coefficients=[C3]), lambda: T.orthogonalise([None]),
                 lambda: T.orthogonalise(x, out=[x]), lambda: T.orthogonalise([x], out=[]), lambda: T.orthogonalise(x.t()), lambda: T.orthogonalise(x, dtype=torch.int8), lambda: T.orthogonalise(x.requires_grad_()),
                 lambda: T.orthogonalise(torch.zeros(2, (1 << 16) + 1)), lambda: muon(), lambda: muon(grads=[x[:2]]), lambda: muon(grads=[]), lambda: muon(momenta=[x.half()]), lambda: muon(copies=[x.detach()]),
                 lambda: muon(copies=[]), lambda: muon(adjust="max"), lambda: muon(steps=0), lambda: muon(params=[x.detach().t()], grads=[x.detach().t()]), lambda: muon(params=[w], grads=[w], momenta=[w]),
                 lambda: T.muon([x.detach()] * 2, [x.detach()] * 2, [torch.zeros(4, 6) for _ in range(2)]), lambda: T.Muon([x], copies=[]), lambda: T.Muon([w]), lambda: T.Muon([x], adjust=""),
                 lambda: T.Muon([x], coefficients=())):
        with pytest.raises(B.FbxError) as e:
            call()
        assert e.value.status == B.E_ARG
    T.muon([], [], [])
    assert T.orthogonalise([]) == []


def test_forward_mode_is_refused():
    import torch.autograd.forward_ad as fwd

    x, w = torch.zeros(4, 6), torch.ones(6)
    with fwd.dual_level():
        t = fwd.make_dual(x, torch.ones_like(x))
        v = fwd.make_dual(w, torch.ones_like(w))
        for call in (lambda: T.norm(t), lambda: T.norm(x, v), lambda: T.norm_backward(t, x), lambda: T.join(t, x), lambda: T.join(x, t), lambda: T.join(x, x, v), lambda: T.join(x, x, w, t),
                     lambda: T.join(x, x, w, x, v), lambda: T.join(x, x, w, x, w, v), lambda: T.join_backward(t, None, x, x), lambda: T.orthogonalise(t)):
            with pytest.raises(B.FbxError):
                call()


def test_muon_loads_only_states_of_its_weights():
    a, b = T.Muon([torch.zeros(3, 4), torch.zeros(5, 2)]), T.Muon([torch.zeros(3, 4), torch.zeros(5, 2)])
    for m in a.m:
        m.uniform_()
    a.step_count = 7
    b.load_state_dict(a.state_dict())
    assert b.step_count == 7 and all(torch.equal(x, y) and x.data_ptr() != y.data_ptr() for x, y in zip(a.m, b.m))
    for wrong in ([torch.ones(3, 4)], [torch.ones(3, 4), torch.ones(2, 5)], [torch.ones(3, 4), torch.ones(5, 2).half()]):
        with pytest.raises(B.FbxError):
            b.load_state_dict({"step": 9, "m": wrong})
        assert b.step_count == 7 and all(torch.equal(x, y) for x, y in zip(a.m, b.m))


BF16 = 2
LISTS = [[(256, 1024), (257, 257)] * 32, [(256, 1024), (1024, 1024)] * 32, [(256, 4096), (512, 512)] * 24, [(128, 2048), (512, 2048), (512, 512)] * 16, [(300, 200), (1024, 1024), (20, 30)] * 40,
         [(1200, 65536), (256, 65536), (256, 65536), (1100, 65536), (256, 65536)]]


@pytest.mark.skipif(torch.cuda.is_available(), reason="what is not refused would be launched, on addresses that are none")
@pytest.mark.parametrize("exact", [0, 1, 2])
@pytest.mark.parametrize("shapes", LISTS, ids=lambda s: f"{len(s)}x{s[0]}")
def test_scratch_of_lists_of_several_kinds(shapes, exact):
    """What the scratch functions give is enough for lists whose matrices go through products of both kinds, and no byte less is."""
    L, need, n = _library(), u64(), len(shapes)
    lists = ((OrthoMatrix * n)(*[_made(OrthoMatrix, MATRIX, dict(rows=r, columns=c, ld_u=c, ld_out=c)) for r, c in shapes]),
             (MuonMatrix * n)(*[_made(MuonMatrix, MUON_MATRIX, dict(rows=r, columns=c)) for r, c in shapes]))
    h = _ortho(exact=exact, out=BF16)
    muon = Muon(ortho=h, param_dtype=BF16, grad_dtype=BF16, copy_dtype=BF16, nesterov=1, lr=1e-3, momentum=0.95, grad_scale=1.0)
    for a, m, size, call in ((h, lists[0], L.fbx_ortho_scratch, L.fbx_orthogonalise), (muon, lists[1], L.fbx_muon_scratch, L.fbx_muon_step)):
        assert size(a, m, n, ctypes.byref(need)) == B.OK and need.value > 0
        assert call(a, m, n, P, need.value - 1, None) == B.E_NOMEM
        assert call(a, m, n, P, need.value, None) == B.E_HIP   # (there is no GPU to launch it on)


def _refusal(call):
    with pytest.raises(B.FbxError) as e:
        call()
    assert e.value.status == B.E_ARG
    return str(e.value)


def _view(buffer, n, d, stride, at):
    return torch.as_strided(buffer, (n, d), (stride, 1), at)


def test_results_that_overlap_are_refused():
    """Views of one buffer, at random: a result that has an element in common with an input is refused as that, and one that has none (columns
    beside it, say) is not.  (Then for lying on the CPU.)"""
    rng = torch.Generator().manual_seed(3)
    pick = lambda a, b: int(torch.randint(a, b + 1, (1,), generator=rng))  # noqa: E731
    buffer, met, missed = torch.zeros(400), 0, 0
    elements = lambda t: set((torch.arange(t.shape[0])[:, None] * (t.stride(0) if t.shape[0] > 1 else 0) + torch.arange(t.shape[1]) + t.storage_offset()).flatten().tolist())  # noqa: E731
    apart = torch.zeros(400)
    for k in range(3000):
        n, d = pick(1, 9), pick(1, 6)
        strides = [pick(d, 3 * d + 4)] * 2 if k % 3 else [pick(d, 3 * d + 4), pick(d, 3 * d + 4)]
        x, out = (_view(buffer, n, d, s, pick(0, 400 - (n - 1) * s - d) if k % 4 else pick(0, min(12, 400 - (n - 1) * s - d))) for s in strides)
        own = x.storage_offset() == out.storage_offset() and (strides[0] == strides[1] or n == 1)
        meet = bool(elements(x) & elements(out))
        y, z = (_view(apart, n, d, d, at) for at in (0, 200))
        met, missed = met + meet, missed + (not meet)
        said = "GPU" if not meet else "overlaps"
        assert ("GPU" if own else said) in _refusal(lambda: T.norm(x, out=out))
        for call in (lambda: T.join(x, y, out=out), lambda: T.join(y, x, out=out), lambda: T.join(y, z, None, x, then=True, out_next=out), lambda: T.join(y, z, then=True, out=x, out_next=out),
                     lambda: T.orthogonalise([x, y], out=[z, out]), lambda: T.orthogonalise([y, z], out=[x, out])):
            assert said in _refusal(call)
        w = buffer[out.storage_offset():out.storage_offset() + d]
        if x.shape[0] > 1 and elements(x) & set(range(out.storage_offset(), out.storage_offset() + d)):
            assert "overlaps" in _refusal(lambda: T.norm(y, w, out=x)) and "overlaps" in _refusal(lambda: T.join(y, z, None, None, w, out=x))
    assert met > 300 and missed > 300
    assert "GPU" in _refusal(lambda: T.orthogonalise([x, y], out=[x, y]))   # (each over itself)


def test_matrices_that_overlap_are_refused_by_muon():
    """Weights, momenta and copies that share an element with each other or with a gradient; gradients may share theirs."""
    b, half, free = torch.zeros(600), torch.zeros(600, dtype=torch.bfloat16), torch.zeros(600)
    at = lambda t, k, n=4: t[k:k + 5 * n].view(n, 5)  # noqa: E731
    p, g, m, c = [at(b, 0), at(b, 20)], [at(free, 0), at(free, 7)], [at(b, 40), at(b, 60)], [at(half, 0), at(half, 20)]
    muon = lambda **k: _refusal(lambda: T.muon(**{**dict(params=p, grads=g, momenta=m, copies=c), **k}))  # noqa: E731
    assert "GPU" in muon()
    for change, why in ((dict(params=[p[0], at(b, 19)]), "another"), (dict(params=[p[0], at(b, 21)]), "another"), (dict(momenta=[at(b, 39), m[1]]), "another"), (dict(momenta=[m[0], at(b, 59)]), "another"),
                        (dict(params=[at(b, 15, 12), p[1]], grads=[at(free, 0, 12), g[1]], momenta=[at(b, 100, 12), m[1]], copies=None), "another"),
                        (dict(copies=[c[0], at(half, 1)]), "another"), (dict(grads=[at(b, 79), g[1]]), "gradient"), (dict(grads=[g[0], at(b, 10)]), "gradient"),
                        (dict(grads=[g[0], at(half, 39).view(4, 5)]), "one type")):
        assert why in muon(**change), change
    assert "GPU" in muon(grads=[at(b, 80), at(b, 99)])


def test_muon_refuses_states_of_another_shape():
    """A momentum or copy of as many elements, but other rows and columns, would be filled in the weights' order."""
    d = dict(params=[torch.zeros(4, 6)], grads=[torch.zeros(4, 6)], momenta=[torch.zeros(4, 6)], copies=[torch.zeros(4, 6, dtype=torch.float16)])
    for name in ("grads", "momenta", "copies"):
        for shape in ((6, 4), (24,), (1, 4, 6)):
            assert "size" in _refusal(lambda: T.muon(**{**d, name: [d[name][0].reshape(shape)]})), (name, shape)
    assert "GPU" in _refusal(lambda: T.muon(**d))
    w = [torch.zeros(4, 6)]
    assert "size" in _refusal(lambda: T.Muon(w, copies=[d["copies"][0].reshape(6, 4)]).step([torch.zeros(4, 6)]))


MUON_REFUSED = test_muon_refuses.pytestmark[0].args[1]


@pytest.mark.parametrize("change, matrix, why", MUON_REFUSED + [({}, {}, "")])
def test_muon_check_refuses_what_a_step_refuses(change, matrix, why):
    L = _library()
    L.fbx_muon_check.argtypes = [ctypes.POINTER(Muon), ctypes.POINTER(MuonMatrix), u32]
    a = dict(param_dtype=0, grad_dtype=0, copy_dtype=2, nesterov=1, lr=1e-3, momentum=0.95, weight_decay=0.0, grad_scale=1.0, ortho={})
    a.update(change)
    h = Muon(**{**a, "ortho": _ortho(**a["ortho"])})
    m = (MuonMatrix * 2)(_made(MuonMatrix, MUON_MATRIX, {}), _made(MuonMatrix, MUON_MATRIX, matrix))
    if why:
        assert L.fbx_muon_check(h, m, 2) == B.E_ARG and why in _why(), _why()
    else:
        assert L.fbx_muon_check(h, m, 2) == B.OK and L.fbx_muon_check(h, None, 0) == B.OK
    assert L.fbx_muon_check(None, m, 2) == B.E_ARG


def test_muon_checks_a_list_before_another_is_stepped():
    """What is checked of every list before one is stepped holds all that the library refuses: 3e38 times a factor of 1.6 is no number of 32 bits."""
    p = [torch.zeros(64, 64)]
    how = [0.95, True, 0.0, 1.0, -1, [3.4445, -4.7750, 2.0315], 1e-7, True]
    check = lambda lr, factor: _refusal(lambda: T._load().muon(p, [torch.zeros(64, 64)], [torch.zeros(64, 64)], None, [factor], lr, *how))  # noqa: E731
    assert "factor" in check(3e38, 1.6) and "lr" in check(float("inf"), 1.0) and "GPU" in check(3e38, 1.0)
