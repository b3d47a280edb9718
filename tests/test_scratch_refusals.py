"""What the queries about scratch buffers refuse (CPU only)."""
import ctypes

from paper_1909_01315_amd import gnnk


def test_whether_a_buffer_was_captured():
    lib = gnnk.load()
    n = ctypes.c_int32(7)
    assert lib.graph_scratch_captured(None, None, ctypes.byref(n)) == gnnk.EINVAL
    assert b"NULL" in lib.gnnk_last_error()
