"""8-bit layer entry points without a GPU: null pointers are refused before anything else is looked at."""
import ctypes as C

import paper_2307_16273_amd as zk
from paper_2307_16273_amd.binding import Mat


def test_null_context_and_matrices_are_refused():
    lib = zk.load_library()
    m = Mat(None, 1, 2, 2, 2, 0, 3, 0)
    p = C.byref(m)
    assert lib.zkdl_quantize_i8(None, p, 1, None, p, None, None) == -1
    assert lib.zkdl_rmsnorm_i8(None, p, None, None, 4, 1e-6, p, None, None, None, None) == -1
    assert lib.zkdl_rmsnorm_i8_backward(None, p, p, None, 4, None, None, p, None) == -1
    assert lib.zkdl_matmul_i8(None, p, p, 0, 0, None, None, p) == -1
    assert lib.zkdl_matmul_i8_backward(None, p, p, p, 0, None, None, p, p) == -1


def test_descriptor_is_the_headers_layout():
    assert C.sizeof(Mat) == 56 and Mat.dtype.offset == 48 and Mat.stack_stride.offset == 40
