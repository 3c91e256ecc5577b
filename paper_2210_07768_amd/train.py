"""The trainer's operators of ``libfbx.so`` (see ``include/fbx_train.h``) on torch tensors: rows of a table pooled per
record and slot of signs (``embed``), a gated feed-forward block (``gated``), and an AdamW step over many tensors at
once (``adamw``, and ``AdamW``, which keeps the states).  Beside each forward function stands its gradient; ``embed`` and
``gated`` also take part in autograd where an input asks for it (backward mode; a tangent is refused).

Argument checks and marshalling only, natively in ``csrc/train/train_native.cpp``: all arithmetic runs in the library's
kernels, enqueued on torch's current stream of the tensors' device.  Nothing waits for the GPU.  Scratch and results
come from torch's allocator.  What is refused raises ``FbxError``.
"""
from __future__ import annotations

import ctypes
import os
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
    """One slot of signs; the slots of an ``ExtractResult`` have the same fields and can stand in its place.  Values that
    the offsets leave out belong to no record: ``Signs(slot.values, slot.offsets[a:b + 1])`` are the records a to b - 1."""
    values: torch.Tensor                       # int64 or uint64
    offsets: Optional[torch.Tensor] = None     # n_records + 1; None: fixed_arity signs a record
    fixed_arity: int = 1                         # ignored where offsets are given
    tile_ends: Optional[torch.Tensor] = None   # results in arrival order only


_native = None


def _load():
    global _native
    if _native is None:
        L = _b.lib()
        path = os.path.join(os.path.dirname(_b.LIB_PATH), "_train.so")
        if not os.path.exists(path):
            raise ImportError(f"{path} is missing: run `python -m paper_2210_07768_amd.build` first")
        from . import _train as N

        N.bind(FbxError, torch.OutOfMemoryError, torch._C._cuda_getCurrentRawStream,
               *(ctypes.cast(getattr(L, name), ctypes.c_void_p).value for name in EXPORTS))
        _native = N
    return _native


def _bad(why: str):
    raise FbxError(_b.E_ARG, why)


def _tensors(**given):
    for name, t in given.items():
        if not isinstance(t, torch.Tensor):
            _bad(f"{name} must be a tensor")


# ------------------------------------------------------------------ rows of a table, pooled
def _table_of(slots, device, n_records: Optional[int]):
    """(slots as the native part takes them, records, records of a tile in arrival order)."""
    if not isinstance(slots, ExtractResult):
        if n_records is None:
            _bad("n_records is needed for a sequence of slots")
        return slots, n_records, 0
    if n_records is not None and n_records != slots.n_records:
        _bad("n_records is not the result's")
    if slots._table is None:
        return b"", slots.n_records, 0
    if slots._table[1].device != device:
        _bad("the signs must be on the table's device")
    return slots._table[0], slots.n_records, slots.arrival_tile_records


def _embed_forward(slots, table, n_records, mean, out):
    slots, n_records, tile = _table_of(slots, table.device, n_records)
    return _load().embed(slots, table, n_records, tile, mean, out)


def embed(slots, table, n_records: Optional[int] = None, mean: bool = False, out=None):
    """Rows of ``table`` (rows x dim) for the signs of every slot, summed (or averaged) per record:
    n_records x slots x dim, zeros where a record has no signs.

    slots: an ``ExtractResult``, or a sequence of its slots or of ``Signs`` (with n_records).  Under autograd the signs are
    read again by the backward pass: extract the next batch behind it, or into another workspace.  It is refused where torch
    or a ``Plan``'s call has written to them, or to the workspace they lie in, since."""
    _tensors(table=table)
    if table.requires_grad and torch.is_grad_enabled():
        if out is not None:
            _bad("out cannot take part in autograd")
        return _Embed.apply(table, slots, n_records, mean)
    return _embed_forward(slots, table, n_records, mean, out)


def embed_backward(dout, slots, rows: int, mean: bool = False, out=None):
    """The gradient of ``embed`` with respect to its table: rows x dim, of dout's type; dout: n_records x slots x dim.
    All rows are written.  The same inputs give the same bits."""
    _tensors(dout=dout)
    if dout.dim() != 3:
        _bad("dout must have three dimensions")
    slots, _, tile = _table_of(slots, dout.device, dout.shape[0])
    return _load().embed_backward(dout, slots, tile, rows, mean, out)


# ------------------------------------------------------------------ the gated block
def _act(act: str) -> int:
    code = ACTS.get(act)
    if code is None:
        _bad(f"act must be one of {', '.join(ACTS)}")
    return code


def gated(x, w_gate, w_up, act: str = "silu", out=None):
    """act(x w_gate^T) * (x w_up^T) in one kernel: x records x inputs, weights hidden x inputs, result records x hidden.
    act: silu, gelu, relu or sigmoid."""
    _tensors(x=x, w_gate=w_gate, w_up=w_up)
    if (x.requires_grad or w_gate.requires_grad or w_up.requires_grad) and torch.is_grad_enabled():
        if out is not None:
            _bad("out cannot take part in autograd")
        return _Gated.apply(x, w_gate, w_up, act)
    return _load().gated(x, w_gate, w_up, _act(act), out)


def gated_backward(dh, x, w_gate, w_up, act: str = "silu", need_dx: bool = True, need_dw: bool = True):
    """Gradients of ``gated`` with respect to x, w_gate and w_up (None for those not needed), of their type.  The
    projections are computed again, not kept; their gradients are rounded to that type between the products (in float16 one
    beyond its range becomes infinite: scale the loss)."""
    return _load().gated_backward(dh, x, w_gate, w_up, _act(act), need_dx, need_dw)


def _versions(slots) -> int:
    if isinstance(slots, ExtractResult):
        return 0 if slots._table is None else _load().versions(slots._table[1])
    return _load().versions(slots)


class _Embed(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, slots, n_records, mean):
        ctx.slots, ctx.rows, ctx.mean = slots if isinstance(slots, ExtractResult) else tuple(slots), table.shape[0], mean
        pooled = _embed_forward(slots, table, n_records, mean, None)
        ctx.versions = _versions(ctx.slots)
        return pooled

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout):
        if _versions(ctx.slots) != ctx.versions:
            _bad("the signs were written to after embed had read them: their gradient would be another batch's")
        return embed_backward(dout, ctx.slots, ctx.rows, ctx.mean), None, None, None


class _Gated(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w_gate, w_up, act):
        ctx.save_for_backward(x, w_gate, w_up)
        ctx.act = act
        return _load().gated(x, w_gate, w_up, _act(act), None)

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
          weight_decay: float = 1e-2, grad_scale: float = 1.0, seed: int = 0, keep_roots: bool = False):
    """One AdamW step over all tensors, in place (the formulas, the 8-bit states and their random rounding: fbx_adamw_step
    in ``include/fbx_train.h``).  All weights are of one type, and so are all gradients.

    m, v: float32 tensors of the weights' sizes, or, with m_scale and v_scale, their codes (float8_e4m3fn or uint8) with
    ceil(n / 32) scales each (float8_e8m0fnu or uint8).  copies: float16 or bfloat16 tensors that receive the new weights
    too.  step counts from 1; seed: of the random rounding, the same for all steps.  keep_roots, for 8-bit states: a sqrt(v) above
    0 is never rounded to 0.  Without it a weight can be moved by lr * m / eps, thousands of times lr, where gradients of
    very unlike size share a block of 32: a training run sets it, as ``AdamW`` does."""
    if step < 1:
        _bad("step counts from 1")
    _load().adamw(params, grads, m, v, m_scale, v_scale, copies, step, lr, betas[0], betas[1], eps, weight_decay, grad_scale, seed & ((1 << 64) - 1), keep_roots, False)


class AdamW:
    """Keeps the states of a list of weights and steps them all at once from their ``.grad``.

    bits: 32 or 8, of a state (8: with ``keep_roots``, see ``adamw``).  copies: a list of float16 or bfloat16 tensors, one for each weight (float32 then), that
    follow the weights: what the kernels of a model in 16 bits read.  A weight's steps count from its first gradient."""

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
        self.steps = [0] * len(self.params)   # of each weight: its bias corrections are of the gradients it had
        kind = torch.uint8 if bits == 8 else torch.float32
        state = lambda p, n, dtype: torch.zeros(n, dtype=dtype, device=p.device)  # noqa: E731
        self.m, self.v = ([state(p, p.numel(), kind) for p in self.params] for _ in range(2))
        if bits == 8:
            self.m_scale, self.v_scale = ([state(p, -(-p.numel() // BLOCK), kind) for p in self.params] for _ in range(2))
        else:
            self.m_scale = self.v_scale = None

    @torch.no_grad()
    def step(self, grads: Optional[Sequence] = None, grad_scale: float = 1.0, lr: Optional[float] = None):
        """grads: one for each weight, instead of their .grad.  Weights without a gradient stay as they are.  All weights are
        stepped, or, where something is refused, none."""
        grads = [p.grad for p in self.params] if grads is None else list(grads)
        if len(grads) != len(self.params):
            _bad("one gradient for each weight")
        kinds = {}
        for i, (p, g) in enumerate(zip(self.params, grads)):
            if g is not None:
                kinds.setdefault((p.dtype, g.dtype, p.device, self.steps[i]), []).append(i)
        pick = lambda x, at: None if x is None else [x[i] for i in at]  # noqa: E731
        calls = [[*(pick(x, at) for x in (self.params, grads, self.m, self.v, self.m_scale, self.v_scale, self.copies)), self.steps[at[0]] + 1,
                  self.lr if lr is None else lr, *self.betas, self.eps, self.weight_decay, grad_scale, (self.seed + (k << 32)) & ((1 << 64) - 1), True]
                 for k, at in enumerate(kinds.values())]
        step = _load().adamw
        for check_only in (True, False) if len(calls) > 1 else (False,):   # (nothing is stepped if a later list is refused)
            for call in calls:
                step(*call, check_only)
        for at in kinds.values():
            for i in at:
                self.steps[i] += 1
        self.step_count += 1

    def zero_grad(self):
        for p in self.params:
            p.grad = None

    def state_dict(self) -> dict:
        return {"step": self.step_count, "steps": tuple(self.steps), "seed": self.seed, "bits": self.bits,
                **{k: getattr(self, k) for k in ("m", "v", "m_scale", "v_scale")}}

    def load_state_dict(self, state: dict):
        if state["bits"] != self.bits:
            _bad("the states are of another kind")
        names = ("m", "v", "m_scale", "v_scale") if self.bits == 8 else ("m", "v")
        steps = list(state.get("steps", [state["step"]] * len(self.m)))   # (states saved without: all weights took all steps)
        if len(steps) != len(self.m):
            _bad("the states are of another number of weights")
        for k in names:   # (all of them before any is copied)
            if state.get(k) is None or len(state[k]) != len(self.m):
                _bad(f"{k}: the states are of another kind or number of weights")
            for mine, theirs in zip(getattr(self, k), state[k]):
                if mine.shape != theirs.shape or mine.dtype != theirs.dtype:
                    _bad(f"{k}: a state is {tuple(theirs.shape)}, {theirs.dtype}, and its weight's {tuple(mine.shape)}, {mine.dtype}")
        for k in names:
            for mine, theirs in zip(getattr(self, k), state[k]):
                mine.copy_(theirs)
        if self.bits == 8:   # (states of steps without keep_roots)
            for m, v in zip(self.m, self.v):
                v.masked_fill_((v == 0) & ((m & 127) != 0), 1)
        self.step_count, self.seed, self.steps = state["step"], state["seed"], steps
