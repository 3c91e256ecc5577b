"""The trainer's operators without a GPU: what lies beyond a launch is refused before any work."""
import ctypes

from paper_2210_07768_amd import binding as B
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
