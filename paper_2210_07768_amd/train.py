"""The trainer's operators of ``libfbx.so`` (see ``include/fbx_train.h``) on torch tensors: rows of a table pooled per
record and slot of signs (``embed``), a gated feed-forward block (``gated``), and an AdamW step over many tensors at
once (``adamw``, and ``AdamW``, which keeps the states).  Beside each forward function stands its gradient; ``embed`` and
``gated`` also take part in autograd where an input asks for it.

Argument checks and marshalling only: all arithmetic runs in the library's kernels, enqueued on torch's current
stream of the tensors' device.  Nothing waits for the GPU.  Scratch and results come from torch's allocator.
"""
from __future__ import annotations

import ctypes
import struct
from typing import List, NamedTuple, Optional, Sequence, Tuple

import torch

from . import binding as _b
from .binding import ExtractResult, FbxError

EXPORTS = [
    "fbx_train_last_error", "fbx_embed_forward", "fbx_embed_backward_scratch", "fbx_embed_backward",
    "fbx_gated_scratch", "fbx_gated_forward", "fbx_gated_backward", "fbx_adamw_step",
]
ACTS = {"silu": 0, "gelu": 1, "relu": 2, "sigmoid": 3}
BLOCK = 32   # elements that share a scale in 8-bit states


class Signs(NamedTuple):
    """One slot of signs; the slots of an ``ExtractResult`` have the same fields and can stand in its place."""
    values: torch.Tensor                       # int64 or uint64
    offsets: Optional[torch.Tensor] = None     # n_records + 1; None: fixed_arity signs a record
    fixed_arity: int = 1                         # ignored where offsets are given
    tile_ends: Optional[torch.Tensor] = None   # results in arrival order only


class _GatedArgs(ctypes.Structure):
    _fields_ = [("records", ctypes.c_uint64), ("inputs", ctypes.c_uint32), ("hidden", ctypes.c_uint32), ("dtype", ctypes.c_int), ("act", ctypes.c_int),
                ("d_x", ctypes.c_void_p), ("d_w_gate", ctypes.c_void_p), ("d_w_up", ctypes.c_void_p),
                ("ld_x", ctypes.c_uint64), ("ld_w_gate", ctypes.c_uint64), ("ld_w_up", ctypes.c_uint64)]


class _AdamwArgs(ctypes.Structure):
    _fields_ = [("param_dtype", ctypes.c_int), ("grad_dtype", ctypes.c_int), ("copy_dtype", ctypes.c_int), ("state_bits", ctypes.c_uint32),
                ("step", ctypes.c_uint64), ("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double),
                ("weight_decay", ctypes.c_double), ("grad_scale", ctypes.c_double), ("seed", ctypes.c_uint64)]


_SLOT = struct.Struct("=IIQQQQ")     # fbx_slot_view
_TENSOR = struct.Struct("=8Q")       # fbx_adamw_tensor
_lib = None
_dtypes = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}


def _library():
    global _lib
    if _lib is None:
        L = _b.lib()
        vp, u64, u32, i32 = ctypes.c_void_p, ctypes.c_uint64, ctypes.c_uint32, ctypes.c_int
        u64p = ctypes.POINTER(u64)
        L.fbx_train_last_error.restype = ctypes.c_char_p
        L.fbx_train_last_error.argtypes = []
        L.fbx_embed_forward.argtypes = [ctypes.c_char_p, u32, u64, u32, vp, u64, u32, u64, i32, i32, vp, u64, vp]
        L.fbx_embed_backward_scratch.argtypes = [ctypes.c_char_p, u32, u64, u64, u32, i32, u64p]
        L.fbx_embed_backward.argtypes = [ctypes.c_char_p, u32, u64, u32, vp, u64, u64, u32, u64, i32, i32, vp, vp, u64, vp]
        L.fbx_gated_scratch.argtypes = [ctypes.POINTER(_GatedArgs), i32, u64p]
        L.fbx_gated_forward.argtypes = [ctypes.POINTER(_GatedArgs), vp, u64, vp, u64, vp]
        L.fbx_gated_backward.argtypes = [ctypes.POINTER(_GatedArgs), vp, u64, vp, u64, vp, u64, vp, u64, vp, u64, vp]
        L.fbx_adamw_step.argtypes = [ctypes.POINTER(_AdamwArgs), ctypes.c_char_p, u32, vp]
        for name in EXPORTS[1:]:
            getattr(L, name).restype = ctypes.c_int
        _lib = L
    return _lib


def _check(status: int):
    if status != _b.OK:
        raise FbxError(status, _lib.fbx_train_last_error().decode())


def _bad(why: str):
    raise FbxError(_b.E_ARG, why)


class _On:
    """Makes the tensors' device the current one, if it is not, and knows its current stream."""
    __slots__ = ("index", "was", "stream")

    def __init__(self, tensor):
        if not tensor.is_cuda:
            _bad("tensors must be on the GPU")
        self.index = tensor.device.index
        self.was = torch._C._cuda_getDevice()
        self.stream = torch._C._cuda_getCurrentRawStream(self.index)

    def __enter__(self):
        if self.was != self.index:
            torch.cuda.set_device(self.index)
        return self.stream

    def __exit__(self, *_):
        if self.was != self.index:
            torch.cuda.set_device(self.was)


def _code(t) -> int:
    code = _dtypes.get(t.dtype)
    if code is None:
        _bad(f"{t.dtype}: float32, float16 and bfloat16 are supported")
    return code


def _matrix(t, name: str, like=None, shape=None) -> int:
    """Checks a matrix whose rows are contiguous and returns its row stride."""
    if t.dim() != 2:
        _bad(f"{name} must have two dimensions")
    if like is not None and (t.dtype != like.dtype or t.device != like.device):
        _bad(f"{name} must have the type and device of the others")
    if shape is not None and tuple(t.shape) != shape:
        _bad(f"{name} must be of shape {shape}, not {tuple(t.shape)}")
    rows, cols = t.shape
    if cols > 1 and t.stride(1) != 1:
        _bad(f"{name}: elements of a row must be adjacent")
    if rows <= 1:
        return cols
    if t.stride(0) < cols:
        _bad(f"{name}: rows may not overlap")
    return t.stride(0)


def _scratch(bytes_needed: int, like):
    return torch.empty(bytes_needed, dtype=torch.uint8, device=like.device) if bytes_needed else None


def _pointer(t) -> int:
    return 0 if t is None else t.data_ptr()


# ------------------------------------------------------------------ rows of a table, pooled
def _table_of(slots, n_records: Optional[int], device) -> Tuple[bytes, int, int, int]:
    """(the library's slot table, slots, records, records of a tile in arrival order)."""
    if isinstance(slots, ExtractResult):
        if n_records is not None and n_records != slots.n_records:
            _bad("n_records is not the result's")
        if slots._table is not None and slots._table[1].device != device:
            _bad("the signs must be on the table's device")
        table = slots._table[0] if slots._table is not None else b""
        return table, len(table) // _SLOT.size, slots.n_records, slots.arrival_tile_records
    if n_records is None:
        _bad("n_records is needed for a list of slots")
    rows, arrival = [], 0
    for s in slots:
        v, o, ends = s.values, s.offsets, s.tile_ends
        if v.device != device or v.itemsize != 8 or v.is_floating_point() or not v.is_contiguous():
            _bad("a slot's values must be contiguous 64-bit integers on the table's device")
        if ends is not None:
            _bad("slots in arrival order are taken as a whole ExtractResult")
        if o is None:
            rows.append(_SLOT.pack(0, s.fixed_arity, v.numel(), v.data_ptr(), 0, 0))
        else:
            if o.device != device or o.itemsize != 8 or o.is_floating_point() or not o.is_contiguous() or o.numel() != n_records + 1:
                _bad("a slot's offsets must be n_records + 1 contiguous 64-bit integers on the table's device")
            rows.append(_SLOT.pack(0, 0, v.numel(), v.data_ptr(), o.data_ptr(), 0))
    return b"".join(rows), len(rows), n_records, arrival


def _embed_forward(slots, table, n_records, mean, out):
    L = _library()
    code, stride = _code(table), _matrix(table, "table")
    views, n_slots, n_records, tile = _table_of(slots, n_records, table.device)
    rows, dim = table.shape
    if out is None:
        out = torch.empty(n_records, n_slots, dim, dtype=table.dtype, device=table.device)
    elif tuple(out.shape) != (n_records, n_slots, dim) or out.dtype != table.dtype or out.device != table.device:
        _bad(f"out must be of shape {(n_records, n_slots, dim)} with the table's type and device")
    elif (dim > 1 and out.stride(2) != 1) or (n_slots > 1 and out.stride(1) != dim):
        _bad("out: a record's rows must be adjacent")
    record_stride = out.stride(0) if n_records > 1 else n_slots * dim
    with _On(table) as stream:
        _check(L.fbx_embed_forward(views, n_slots, n_records, tile, table.data_ptr(), rows, dim, max(stride, dim), code, int(bool(mean)), out.data_ptr(),
                                   record_stride, stream))
    return out


def embed(slots, table, n_records: Optional[int] = None, mean: bool = False, out=None):
    """Rows of ``table`` (rows x dim) for the signs of every slot, summed (or averaged) per record:
    n_records x slots x dim, zeros where a record has no signs.

    slots: an ``ExtractResult``, or a sequence of its slots or of ``Signs`` (with n_records)."""
    if table.requires_grad and torch.is_grad_enabled():
        if out is not None:
            _bad("out cannot take part in autograd")
        return _Embed.apply(table, slots, n_records, mean)
    return _embed_forward(slots, table, n_records, mean, out)


def embed_backward(dout, slots, rows: int, mean: bool = False, out=None):
    """The gradient of ``embed`` with respect to its table: rows x dim, of dout's type; dout: n_records x slots x dim.
    All rows are written.  The same inputs give the same bits."""
    L = _library()
    code = _code(dout)
    if dout.dim() != 3:
        _bad("dout must have three dimensions")
    n_records, n_slots, dim = dout.shape
    views, count, n_records, tile = _table_of(slots, n_records, dout.device)
    if count != n_slots:
        _bad("dout must have as many slots as there are")
    if (dim > 1 and dout.stride(2) != 1) or (n_slots > 1 and dout.stride(1) != dim) or (n_records > 1 and dout.stride(0) < n_slots * dim):
        dout = dout.contiguous()
    if out is None:
        out = torch.empty(rows, dim, dtype=dout.dtype, device=dout.device)
    stride = max(_matrix(out, "out", dout, (rows, dim)), dim)
    need = ctypes.c_uint64()
    _check(L.fbx_embed_backward_scratch(views, n_slots, n_records, rows, dim, int(bool(mean)), ctypes.byref(need)))
    scratch = _scratch(need.value, dout)
    with _On(dout) as stream:
        _check(L.fbx_embed_backward(views, n_slots, n_records, tile, dout.data_ptr(), dout.stride(0) if n_records > 1 else n_slots * dim, rows, dim, stride, code,
                                    int(bool(mean)), out.data_ptr(), _pointer(scratch), need.value, stream))
    return out


# ------------------------------------------------------------------ the gated block
def _gated_args(x, w_gate, w_up, act: str) -> _GatedArgs:
    if act not in ACTS:
        _bad(f"act must be one of {', '.join(ACTS)}")
    code, ld_x = _code(x), _matrix(x, "x")
    shape = (w_gate.shape[0], x.shape[1])
    ld_gate, ld_up = _matrix(w_gate, "w_gate", x, shape), _matrix(w_up, "w_up", x, shape)
    return _GatedArgs(x.shape[0], shape[1], shape[0], code, ACTS[act], x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), ld_x, ld_gate, ld_up)


def _gated_forward(x, w_gate, w_up, act, out):
    L = _library()
    args = _gated_args(x, w_gate, w_up, act)
    if out is None:
        out = torch.empty(args.records, args.hidden, dtype=x.dtype, device=x.device)
    ld = _matrix(out, "out", x, (args.records, args.hidden))
    need = ctypes.c_uint64()
    _check(L.fbx_gated_scratch(args, 0, ctypes.byref(need)))
    scratch = _scratch(need.value, x)
    with _On(x) as stream:
        _check(L.fbx_gated_forward(args, out.data_ptr(), ld, _pointer(scratch), need.value, stream))
    return out


def gated(x, w_gate, w_up, act: str = "silu", out=None):
    """act(x w_gate^T) * (x w_up^T) in one kernel: x records x inputs, weights hidden x inputs, result records x hidden.
    act: silu, gelu, relu or sigmoid."""
    if torch.is_grad_enabled() and (x.requires_grad or w_gate.requires_grad or w_up.requires_grad):
        if out is not None:
            _bad("out cannot take part in autograd")
        return _Gated.apply(x, w_gate, w_up, act)
    return _gated_forward(x, w_gate, w_up, act, out)


def gated_backward(dh, x, w_gate, w_up, act: str = "silu", need_dx: bool = True, need_dw: bool = True):
    """Gradients of ``gated`` with respect to x, w_gate and w_up (None for those not needed), of their type.  The
    projections are computed again, not kept."""
    L = _library()
    args = _gated_args(x, w_gate, w_up, act)
    ld_dh = _matrix(dh, "dh", x, (args.records, args.hidden))
    dx = torch.empty(args.records, args.inputs, dtype=x.dtype, device=x.device) if need_dx else None
    dw_gate, dw_up = (torch.empty(args.hidden, args.inputs, dtype=x.dtype, device=x.device) if need_dw else None for _ in range(2))
    need = ctypes.c_uint64()
    _check(L.fbx_gated_scratch(args, 1, ctypes.byref(need)))
    scratch = _scratch(need.value, x)
    k = args.inputs
    with _On(x) as stream:
        _check(L.fbx_gated_backward(args, dh.data_ptr(), ld_dh, _pointer(dx), k, _pointer(dw_gate), k, _pointer(dw_up), k, _pointer(scratch), need.value,
                                    stream))
    return dx, dw_gate, dw_up


class _Embed(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, slots, n_records, mean):
        ctx.slots, ctx.rows, ctx.mean = slots, table.shape[0], mean
        return _embed_forward(slots, table, n_records, mean, None)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout):
        return embed_backward(dout, ctx.slots, ctx.rows, ctx.mean), None, None, None


class _Gated(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w_gate, w_up, act):
        ctx.save_for_backward(x, w_gate, w_up)
        ctx.act = act
        return _gated_forward(x, w_gate, w_up, act, None)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dh):
        if dh.dim() == 2 and (dh.stride(1) != 1 or dh.stride(0) < dh.shape[1]):
            dh = dh.contiguous()   # (a sum's gradient is one element seen many times)
        need = ctx.needs_input_grad
        dx, dw_gate, dw_up = gated_backward(dh, *ctx.saved_tensors, ctx.act, need_dx=need[0], need_dw=need[1] or need[2])
        return dx, dw_gate if need[1] else None, dw_up if need[2] else None, None


# ------------------------------------------------------------------ AdamW
def adamw(params: Sequence, grads: Sequence, m: Sequence, v: Sequence, m_scale: Optional[Sequence] = None, v_scale: Optional[Sequence] = None,
          copies: Optional[Sequence] = None, *, step: int, lr: float = 1e-3, betas: Tuple[float, float] = (0.9, 0.999), eps: float = 1e-8,
          weight_decay: float = 1e-2, grad_scale: float = 1.0, seed: int = 0):
    """One AdamW step over all tensors, in place (the formulas, the 8-bit states and their random rounding: fbx_adamw_step
    in ``include/fbx_train.h``).  All weights are of one type, and so are all gradients.

    m, v: float32 tensors of the weights' sizes, or, with m_scale and v_scale, their codes (float8_e4m3fn or uint8) with
    ceil(n / 32) scales each (float8_e8m0fnu or uint8).  copies: float16 or bfloat16 tensors that receive the new weights
    too.  step counts from 1; seed: of the random rounding, the same for all steps."""
    L = _library()
    n = len(params)
    eight = m_scale is not None
    lists = [params, grads, m, v] + ([m_scale, v_scale] if eight else []) + ([copies] if copies is not None else [])
    if eight and v_scale is None or any(len(x) != n for x in lists):
        _bad("params, grads, states and copies must be lists of one length")
    if n == 0:
        return
    first = params[0]
    code, grad_code = _code(first), _code(grads[0])
    copy_code = _code(copies[0]) if copies is not None else 0
    rows, where = [], first.device
    none = (None,) * n
    for p, g, a, b, a_s, b_s, c in zip(params, grads, m, v, m_scale or none, v_scale or none, copies if copies is not None else none):
        size = p.numel()
        blocks = -(-size // BLOCK)
        if p.dtype != first.dtype or g.dtype != grads[0].dtype or (c is not None and c.dtype != copies[0].dtype):
            _bad("all weights are of one type, and so are all gradients and all copies")
        if g.shape != p.shape or a.numel() != size or b.numel() != size or (eight and (a_s.numel() != blocks or b_s.numel() != blocks)) or \
                (c is not None and c.numel() != size):
            _bad("a gradient, state or copy is not of its weights' size")
        if eight:
            if a.itemsize != 1 or b.itemsize != 1 or a_s.itemsize != 1 or b_s.itemsize != 1:
                _bad("8-bit states are held in bytes")
        elif a.dtype != torch.float32 or b.dtype != torch.float32:
            _bad("32-bit states are float32")
        for t in (p, g, a, b, a_s, b_s, c):
            if t is not None and (t.device != where or not t.is_contiguous()):
                _bad("all tensors must be contiguous and on one device")
        rows.append(_TENSOR.pack(p.data_ptr(), g.data_ptr(), a.data_ptr(), b.data_ptr(), _pointer(a_s), _pointer(b_s), _pointer(c), size))
    args = _AdamwArgs(code, grad_code, copy_code, 8 if eight else 32, step, lr, betas[0], betas[1], eps, weight_decay, grad_scale, seed & ((1 << 64) - 1))
    with _On(first) as stream:
        _check(L.fbx_adamw_step(args, b"".join(rows), n, stream))
    torch.autograd.graph.increment_version(params)   # (autograd then knows that they changed)


class AdamW:
    """Keeps the states of a list of weights and steps them all at once from their ``.grad``.

    bits: 32 or 8, of a state.  copies: a list of float16 or bfloat16 tensors, one for each weight (float32 then), that
    follow the weights: what the kernels of a model in 16 bits read."""

    def __init__(self, params, lr: float = 1e-3, betas: Tuple[float, float] = (0.9, 0.999), eps: float = 1e-8, weight_decay: float = 1e-2,
                 bits: int = 32, seed: int = 0, copies: Optional[List] = None):
        if bits not in (8, 32):
            _bad("bits must be 8 or 32")
        self.params = list(params)
        self.copies = None if copies is None else list(copies)
        if self.copies is not None and len(self.copies) != len(self.params):
            _bad("one copy for each weight")
        self.lr, self.betas, self.eps, self.weight_decay, self.bits, self.seed = lr, betas, eps, weight_decay, bits, seed
        self.step_count = 0
        kind = torch.uint8 if bits == 8 else torch.float32
        state = lambda p, n, dtype: torch.zeros(n, dtype=dtype, device=p.device)  # noqa: E731
        self.m, self.v = ([state(p, p.numel(), kind) for p in self.params] for _ in range(2))
        if bits == 8:
            self.m_scale, self.v_scale = ([state(p, -(-p.numel() // BLOCK), kind) for p in self.params] for _ in range(2))
        else:
            self.m_scale = self.v_scale = None

    @torch.no_grad()
    def step(self, grads: Optional[Sequence] = None, grad_scale: float = 1.0, lr: Optional[float] = None):
        """grads: one for each weight, instead of their .grad.  Weights without a gradient stay as they are."""
        grads = [p.grad for p in self.params] if grads is None else list(grads)
        if len(grads) != len(self.params):
            _bad("one gradient for each weight")
        kinds = {}
        for i, (p, g) in enumerate(zip(self.params, grads)):
            if g is not None:
                kinds.setdefault((p.dtype, g.dtype, p.device), []).append(i)
        self.step_count += 1
        for k, at in enumerate(kinds.values()):
            pick = lambda x: None if x is None else [x[i] for i in at]  # noqa: E731
            adamw(pick(self.params), pick(grads), pick(self.m), pick(self.v), pick(self.m_scale), pick(self.v_scale), pick(self.copies),
                  step=self.step_count, lr=self.lr if lr is None else lr, betas=self.betas, eps=self.eps, weight_decay=self.weight_decay,
                  grad_scale=grad_scale, seed=self.seed + (k << 32))

    def zero_grad(self):
        for p in self.params:
            p.grad = None

    def state_dict(self) -> dict:
        return {"step": self.step_count, "seed": self.seed, "bits": self.bits,
                **{k: getattr(self, k) for k in ("m", "v", "m_scale", "v_scale")}}

    def load_state_dict(self, state: dict):
        if state["bits"] != self.bits or len(state["m"]) != len(self.m):
            _bad("the states are of another kind")
        self.step_count, self.seed = state["step"], state["seed"]
        for k in ("m", "v", "m_scale", "v_scale"):
            for mine, theirs in zip(getattr(self, k) or (), state[k] or ()):
                mine.copy_(theirs)
