"""The trainer's operators without a GPU: what lies beyond a launch is refused before any work."""
import ctypes

import pytest
import torch

from paper_2210_07768_amd import binding as B
from paper_2210_07768_amd import train as T
from test_host_train import TENSOR, AdamwArgs, _gated, _library, _slot, _why


def test_embed_backward_refuses_more_records_than_a_launch_holds():
    """A lane a record, in workgroups of 256, lanes counted in 32 bits."""
    L, need = _library(), ctypes.c_uint64()
    scratch = lambda records, slots: L.fbx_embed_backward_scratch(_slot(0, 5, offsets=4096) * slots, slots, records, 7, 4, 0, ctypes.byref(need))  # noqa: E731
    assert scratch((1 << 32) - 256, 1) == B.OK and scratch((1 << 31) - 128, 2) == B.OK
    assert scratch((1 << 32) - 255, 1) == B.E_ARG and "2^32 - 256" in _why()
    assert scratch((1 << 31) - 127, 2) == B.E_ARG


def test_gated_refuses_more_tiles_than_a_launch_holds():
    """2^25 tiles of 512 lanes each, which are counted in 32 bits: of the forward product, or of one of the gradient's alone."""
    L = _library()
    wide = _gated(records=1 << 24, inputs=8, hidden=1 << 16, ld_x=8, ld_w_gate=8, ld_w_up=8)
    assert L.fbx_gated_forward(wide, 4096, 1 << 16, 1 << 20, 1 << 62, None) == B.E_ARG and "too large" in _why()
    for inputs, hidden in ((8, 1 << 16), (1 << 17, 8)):
        g = _gated(records=1 << 24, inputs=inputs, hidden=hidden, ld_x=inputs, ld_w_gate=inputs, ld_w_up=inputs)
        assert L.fbx_gated_backward(g, 4096, hidden, 4096, inputs, 4096, inputs, 4096, inputs, 1 << 20, 1 << 62, None) == B.E_ARG and "too large" in _why()


def test_adamw_refuses_more_elements_than_a_launch_holds():
    """2,048 elements a workgroup of 256 lanes, lanes counted in 32 bits; nothing is enqueued for the tensors before it."""
    h = AdamwArgs(0, 0, 0, 32, 1, 1e-3, 0.9, 0.999, 1e-8, 0.0, 1.0, 0)
    tensors = TENSOR.pack(4096, 4096, 4096, 4096, 0, 0, 0, 8) + TENSOR.pack(4096, 4096, 4096, 4096, 0, 0, 0, (1 << 35) - 2047)
    assert _library().fbx_adamw_step(h, tensors, 2, None) == B.E_ARG and "2^35" in _why()


def _optimizer(sizes, bits):
    opt = T.AdamW([torch.zeros(n) for n in sizes], bits=bits)
    for k, x in enumerate((opt.m, opt.v, opt.m_scale or [], opt.v_scale or [])):
        for t in x:
            t.fill_(k + 1)
    return opt


@pytest.mark.parametrize("bits", [8, 32])
def test_adamw_loads_only_states_of_its_weights(bits):
    """A state that would have to be spread over a weight, cut, or taken for another kind is refused, and nothing is loaded."""
    def change(**to):
        return {**_optimizer([40, 33], bits).state_dict(), "step": 9, "steps": (9, 9), "seed": 4, **to}

    one, short = [torch.zeros(1, dtype=t.dtype) for t in _optimizer([40, 33], bits).m], _optimizer([40], bits)
    refused = [change(m=one), change(v=one), change(m=short.m), change(v=short.v), change(m=[t.double() for t in _optimizer([40, 33], bits).m]), change(v=None),
               change(steps=(9,)), change(bits=40 - bits), _optimizer([33, 40], bits).state_dict()]
    if bits == 8:
        refused += [change(m_scale=None), change(v_scale=None, m_scale=None), change(v_scale=short.v_scale), change(m_scale=[t[:1] for t in _optimizer([40, 33], bits).m_scale])]
    for state in refused:
        opt, same = _optimizer([40, 33], bits), _optimizer([40, 33], bits)
        for t in opt.m + opt.v + (opt.m_scale or []) + (opt.v_scale or []):
            t.add_(10)
        for t in same.m + same.v + (same.m_scale or []) + (same.v_scale or []):
            t.add_(10)
        with pytest.raises(B.FbxError) as e:
            opt.load_state_dict(state)
        assert e.value.status == B.E_ARG
        mine, kept = opt.state_dict(), same.state_dict()
        assert all(torch.equal(x, y) for k in ("m", "v", "m_scale", "v_scale") for x, y in zip(mine[k] or [], kept[k] or []))
        assert (mine["step"], mine["seed"], mine["steps"]) == (0, 0, (0, 0))
    opt = _optimizer([40, 33], bits)
    opt.load_state_dict(change())
    assert opt.step_count == 9 and opt.steps == [9, 9] and opt.seed == 4


def test_forward_mode_is_refused():
    """A tangent that the operators cannot carry on is no reason to return a result without one."""
    from torch.autograd import forward_ad

    x, w, s = torch.zeros(4, 6), torch.zeros(5, 6), [T.Signs(torch.zeros(4, dtype=torch.int64))]
    with forward_ad.dual_level():
        dual = lambda t: forward_ad.make_dual(t, torch.ones_like(t))  # noqa: E731
        for call in (lambda: T.embed(s, dual(x), 4), lambda: T.embed_backward(dual(x.view(4, 1, 6)), s, 10), lambda: T.gated(dual(x), w, w), lambda: T.gated(x, dual(w), w),
                     lambda: T.gated(x, w, dual(w)), lambda: T.gated_backward(dual(torch.zeros(4, 5)), x, w, w), lambda: T.gated_backward(torch.zeros(4, 5), dual(x), w, w)):
            with pytest.raises(B.FbxError) as e:
                call()
            assert e.value.status == B.E_ARG and "forward mode" in str(e.value)
        for call in (lambda: T.embed(s, dual(x.clone().requires_grad_()), 4), lambda: T.gated(x, dual(w.clone().requires_grad_()), w)):
            with pytest.raises(RuntimeError):   # (torch's own error, or the operator's)
                call()
    assert "GPU" in str(pytest.raises(B.FbxError, T.gated, x, w, w).value)


@pytest.mark.parametrize("step", [0, -1, -(1 << 63)])
def test_adamw_steps_count_from_one(step):
    x = torch.zeros(4, 6)
    with pytest.raises(B.FbxError) as e:
        T.adamw([x], [x], [x], [x], step=step)
    assert e.value.status == B.E_ARG and "step" in str(e.value)


def test_what_is_no_tensor_is_refused():
    x, w, s = torch.zeros(4, 6), torch.zeros(5, 6), [T.Signs(torch.zeros(4, dtype=torch.int64))]
    for call in (lambda: T.embed(s, None, 4), lambda: T.embed(s, x.numpy(), 4), lambda: T.embed_backward(None, s, 4), lambda: T.embed_backward(torch.tensor(1.0), s, 4),
                 lambda: T.embed_backward(torch.zeros(4), s, 4), lambda: T.gated(None, w, w), lambda: T.gated(x, [1.0], w), lambda: T.gated(x, w, 3),
                 lambda: T.gated_backward(None, x, w, w), lambda: T.gated_backward(torch.zeros(4, 5), x, w, "w"), lambda: T.adamw([x], [None], [x], [x], step=1)):
        with pytest.raises(B.FbxError) as e:
            call()
        assert e.value.status == B.E_ARG


def test_adamw_loads_states_whose_roots_were_not_kept():
    """A code 0 of sqrt(v) beside a code of m that is not 0, of either sign: 1 from then on; nothing else changes."""
    saved = T.AdamW([torch.zeros(40)], bits=8).state_dict()
    saved["m"][0][:6] = torch.tensor([0, 128, 1, 129, 5, 255], dtype=torch.uint8)
    saved["v"][0][4:6] = torch.tensor([9, 127], dtype=torch.uint8)
    opt = T.AdamW([torch.zeros(40)], bits=8)
    opt.load_state_dict(saved)
    assert torch.equal(opt.m[0], saved["m"][0]) and opt.v[0].tolist() == [0, 0, 1, 1, 9, 127] + [0] * 34
