"""The trainer's operators without a GPU: what lies beyond a launch is refused before any work."""
import ctypes

from paper_2210_07768_amd import binding as B
from test_host_train import _library, _slot, _why


def test_embed_backward_refuses_more_records_than_a_launch_holds():
    """A lane a record, in workgroups of 256, lanes counted in 32 bits."""
    L, need = _library(), ctypes.c_uint64()
    scratch = lambda records, slots: L.fbx_embed_backward_scratch(_slot(0, 5, offsets=4096) * slots, slots, records, 7, 4, 0, ctypes.byref(need))  # noqa: E731
    assert scratch((1 << 32) - 256, 1) == B.OK and scratch((1 << 31) - 128, 2) == B.OK
    assert scratch((1 << 32) - 255, 1) == B.E_ARG and "2^32 - 256" in _why()
    assert scratch((1 << 31) - 127, 2) == B.E_ARG
