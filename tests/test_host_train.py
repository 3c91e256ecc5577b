"""The trainer's operators without a GPU: declared symbols are exported, and bad arguments are refused before any work."""
import ctypes
import os
import re
import struct

import pytest
import torch

from paper_2210_07768_amd import binding as B
from paper_2210_07768_amd import train as T

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_library_exports_every_declared_symbol():
    text = open(os.path.join(ROOT, "include", "fbx_train.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    declared = set(re.findall(r"\b(fbx_[a-z_]+)\s*\(", text))
    assert declared == set(T.EXPORTS)
    L = ctypes.CDLL(B.LIB_PATH)
    for name in declared:
        assert hasattr(L, name), name


class GatedArgs(ctypes.Structure):
    _fields_ = [("records", ctypes.c_uint64), ("inputs", ctypes.c_uint32), ("hidden", ctypes.c_uint32), ("dtype", ctypes.c_int), ("act", ctypes.c_int),
                ("d_x", ctypes.c_void_p), ("d_w_gate", ctypes.c_void_p), ("d_w_up", ctypes.c_void_p),
                ("ld_x", ctypes.c_uint64), ("ld_w_gate", ctypes.c_uint64), ("ld_w_up", ctypes.c_uint64)]


class AdamwArgs(ctypes.Structure):
    _fields_ = [("param_dtype", ctypes.c_int), ("grad_dtype", ctypes.c_int), ("copy_dtype", ctypes.c_int), ("state_bits", ctypes.c_uint32),
                ("step", ctypes.c_uint64), ("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double),
                ("weight_decay", ctypes.c_double), ("grad_scale", ctypes.c_double), ("seed", ctypes.c_uint64)]


SLOT = struct.Struct("=IIQQQQ")     # fbx_slot_view
TENSOR = struct.Struct("=8Q")       # fbx_adamw_tensor
_lib = None


def _library():
    """The C ABI as a C program sees it."""
    global _lib
    if _lib is None:
        L = B.lib()
        vp, u64, u32, i32 = ctypes.c_void_p, ctypes.c_uint64, ctypes.c_uint32, ctypes.c_int
        u64p = ctypes.POINTER(u64)
        L.fbx_train_last_error.restype = ctypes.c_char_p
        L.fbx_train_last_error.argtypes = []
        L.fbx_embed_forward.argtypes = [ctypes.c_char_p, u32, u64, u32, vp, u64, u32, u64, i32, i32, vp, u64, vp]
        L.fbx_embed_backward_scratch.argtypes = [ctypes.c_char_p, u32, u64, u64, u32, i32, u64p]
        L.fbx_embed_backward.argtypes = [ctypes.c_char_p, u32, u64, u32, vp, u64, u64, u32, u64, i32, i32, vp, vp, u64, vp]
        L.fbx_gated_scratch.argtypes = [ctypes.POINTER(GatedArgs), i32, u64p]
        L.fbx_gated_forward.argtypes = [ctypes.POINTER(GatedArgs), vp, u64, vp, u64, vp]
        L.fbx_gated_backward.argtypes = [ctypes.POINTER(GatedArgs), vp, u64, vp, u64, vp, u64, vp, u64, vp, u64, vp]
        L.fbx_adamw_step.argtypes = [ctypes.POINTER(AdamwArgs), ctypes.c_char_p, u32, vp]
        _lib = L
    return _lib


def _why():
    return _library().fbx_train_last_error().decode()


def _slot(arity, n_values, values=4096, offsets=0, ends=0):
    return SLOT.pack(0, arity, n_values, values, offsets, ends)


def _embed(slots, n_slots=1, n=10, tile=0, table=4096, rows=7, dim=4, table_stride=4, dtype=0, out=4096, record_stride=4):
    return _library().fbx_embed_forward(slots, n_slots, n, tile, table, rows, dim, table_stride, dtype, 0, out, record_stride, None)


@pytest.mark.parametrize("change, why", [
    (dict(dtype=3), "dtype"), (dict(rows=0), "rows"), (dict(rows=1 << 31), "rows"), (dict(dim=0), "dim"), (dict(table_stride=3), "table_stride"),
    (dict(record_stride=3), "record_stride"), (dict(n=1 << 32), "n_records"), (dict(slots=None), "slots"), (dict(table=None), "NULL"),
    (dict(out=None), "NULL"), (dict(table=4097), "aligned"), (dict(slots=_slot(1, 9)), "fixed_arity"), (dict(slots=_slot(0, 9)), "offsets"),
    (dict(slots=_slot(1, 10, values=0)), "values"), (dict(slots=_slot(0, 9, offsets=4096, ends=4096)), "arrival"),
    (dict(slots=_slot(0, 9, offsets=4096), tile=32), "tile_ends"),
])
def test_embed_refuses(change, why):
    args = dict(slots=_slot(1, 10))
    args.update(change)
    assert _embed(args.pop("slots"), **args) == B.E_ARG
    assert why in _why()


def test_embed_backward_refuses():
    L, need = _library(), ctypes.c_uint64()
    slot = _slot(1, 10)
    assert L.fbx_embed_backward_scratch(slot, 1, 10, 7, 4, 0, ctypes.byref(need)) == B.OK and need.value > 0
    call = lambda scratch, size, slots=slot, n=10: L.fbx_embed_backward(slots, 1, n, 0, 4096, 4, 7, 4, 4, 0, 0, 4096, scratch, size, None)  # noqa: E731
    assert call(None, need.value) == B.E_ARG
    assert call(4096 + 8, need.value) == B.E_ARG
    assert call(4096, need.value - 1) == B.E_NOMEM and "scratch" in _why()
    assert L.fbx_embed_backward_scratch(_slot(0, 1 << 32, offsets=4096), 1, 10, 7, 4, 0, ctypes.byref(need)) == B.E_ARG
    assert L.fbx_embed_backward_scratch(slot, 1, 10, 7, 4, 0, None) == B.E_ARG
    many = _slot(1, (1 << 31)) * 2    # records x slots does not fit 32 bits
    assert L.fbx_embed_backward_scratch(many, 2, 1 << 31, 7, 4, 0, ctypes.byref(need)) == B.E_ARG


def _gated(**change):
    a = dict(records=8, inputs=16, hidden=32, dtype=0, act=0, d_x=4096, d_w_gate=4096, d_w_up=4096, ld_x=16, ld_w_gate=16, ld_w_up=16)
    a.update(change)
    return GatedArgs(*(a[k] for k, _ in GatedArgs._fields_))


@pytest.mark.parametrize("change", [dict(dtype=3), dict(act=4), dict(records=1 << 31), dict(inputs=0), dict(hidden=0), dict(hidden=(1 << 20) + 1), dict(ld_x=15),
                                    dict(ld_w_up=15), dict(ld_w_gate=1 << 22), dict(d_x=None), dict(d_w_gate=None), dict(d_w_up=None), dict(d_x=4097)])
def test_gated_refuses(change):
    L = _library()
    assert L.fbx_gated_forward(_gated(**change), 4096, 32, 1 << 20, 1 << 30, None) == B.E_ARG, _why()
    assert L.fbx_gated_backward(_gated(**change), 4096, 32, 4096, 16, 4096, 16, 4096, 16, 1 << 20, 1 << 30, None) == B.E_ARG


def test_gated_refuses_outputs():
    L, need = _library(), ctypes.c_uint64()
    assert L.fbx_gated_forward(_gated(), 4096, 31, None, 0, None) == B.E_ARG
    assert L.fbx_gated_forward(_gated(), None, 32, None, 0, None) == B.E_ARG
    assert L.fbx_gated_forward(None, 4096, 32, None, 0, None) == B.E_ARG
    assert L.fbx_gated_forward(_gated(records=0), 4096, 32, None, 0, None) == B.OK   # nothing to do
    assert L.fbx_gated_scratch(_gated(), 1, ctypes.byref(need)) == B.OK and need.value > 0
    back = lambda dh=4096, ld=32, dx=4096, g=4096, u=4096, scratch=4096, size=need.value: L.fbx_gated_backward(  # noqa: E731
        _gated(), dh, ld, dx, 16, g, 16, u, 16, scratch, size, None)
    assert back(dh=None) == B.E_ARG and back(ld=31) == B.E_ARG and back(u=None) == B.E_ARG
    assert back(scratch=None) == B.E_ARG and back(scratch=4100) == B.E_ARG and back(size=need.value - 1) == B.E_NOMEM
    assert L.fbx_gated_scratch(_gated(), 1, None) == B.E_ARG


@pytest.mark.parametrize("change", [dict(param_dtype=3), dict(grad_dtype=-1), dict(state_bits=16), dict(step=0), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=float("nan")),
                                    dict(lr=float("inf")), dict(grad_scale=float("nan")), dict(copy_dtype=0), dict(tensor=(0, 4096, 4096, 4096, 0, 0, 0, 8)),
                                    dict(tensor=(4096, 4096, 4096, 0, 0, 0, 0, 8)), dict(tensor=(4098, 4096, 4096, 4096, 0, 0, 0, 8)),
                                    dict(tensor=(4096, 4096, 4096, 4096, 0, 0, 0, 8), state_bits=8), dict(tensor=(4096, 4096, 4096, 4096, 0, 0, 0, 1 << 40)),
                                    dict(tensors=(None, 1))])
def test_adamw_refuses(change):
    a = dict(param_dtype=0, grad_dtype=0, copy_dtype=2, state_bits=32, step=1, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, grad_scale=1.0, seed=0)
    change = dict(change)
    tensors, n = change.pop("tensors", (TENSOR.pack(*change.pop("tensor", (4096, 4096, 4096, 4096, 4096, 4096, 4096, 8))), 1))
    a.update(change)
    h = AdamwArgs(*(a[k] for k, _ in AdamwArgs._fields_))
    assert _library().fbx_adamw_step(h, tensors, n, None) == B.E_ARG, _why()
    assert _library().fbx_adamw_step(None, tensors, n, None) == B.E_ARG
    assert _library().fbx_adamw_step(AdamwArgs(0, 0, 0, 32, 1, 1e-3, 0.9, 0.999, 1e-8, 0.0, 1.0, 0), None, 0, None) == B.OK   # nothing to do


def test_python_entry_points_refuse():
    x, w = torch.zeros(4, 6), torch.zeros(5, 6)
    for call in (lambda: T.gated(x, w, w), lambda: T.embed([T.Signs(torch.zeros(4, dtype=torch.int64))], x, 4),
                 lambda: T.gated(x, w, w[:, :5]), lambda: T.gated(x, w.double(), w), lambda: T.gated(x.double(), w.double(), w.double()),
                 lambda: T.gated(x.t(), w, w), lambda: T.gated(x, w, w, act="tanh"), lambda: T.gated(x[0], w, w), lambda: T.gated(x[:1].expand(4, 6), w, w),
                 lambda: T.gated(x, w, w, out=torch.zeros(4, 6)), lambda: T.gated_backward(x, x, w, w),
                 lambda: T.embed([T.Signs(torch.zeros(4))], x, 4), lambda: T.embed([T.Signs(torch.zeros(4, dtype=torch.int64))], x),
                 lambda: T.embed([T.Signs(torch.zeros(4, dtype=torch.int64), torch.zeros(4, dtype=torch.int64))], x, 4),
                 lambda: T.embed_backward(torch.zeros(4, 2, 6), [T.Signs(torch.zeros(4, dtype=torch.int64))], 10),
                 lambda: T.adamw([x], [x], [x], [x], step=1), lambda: T.adamw([x], [x[:2]], [x], [x], step=1), lambda: T.adamw([x], [x], [x], [], step=1),
                 lambda: T.adamw([x], [x], [x.half()], [x], step=1), lambda: T.adamw([x], [x], [x], [x], [x], [x], step=1),
                 lambda: T.AdamW([x], bits=4), lambda: T.AdamW([x], copies=[])):
        with pytest.raises(B.FbxError) as e:
            call()
        assert e.value.status == B.E_ARG
    T.adamw([], [], [], [], step=1)
