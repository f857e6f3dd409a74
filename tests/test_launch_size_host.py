"""A launch of 2^32 threads or more is an error: HIP starts the remainder modulo 2^32 without one."""
import ctypes as C

import pytest
import torch

from paper_2604_04701_amd import binding as B
from test_block_host import AWAY, FAKE


class View(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p), ("n_blocks", C.c_int), ("block_shift", C.c_int),
                ("n_kv_heads", C.c_int), ("head_dim", C.c_int), ("ld_block", C.c_longlong), ("ld_head", C.c_longlong), ("ld_token", C.c_longlong)]


@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are not a GPU's")
def test_a_launch_that_hip_would_cut_is_an_error():
    B.lib()
    launch = C.CDLL(B.LIB_PATH)["_ZN4muxq16launch_kv_gatherEPKiiRKNS_6KvViewEbPDF16_iS5_iP12ihipStream_t"]
    launch.argtypes = [C.c_void_p, C.c_int, C.POINTER(View), C.c_bool, C.c_void_p, C.c_int, C.c_void_p, C.c_int, C.c_void_p]
    launch.restype = C.c_int
    view = View(FAKE, FAKE, None, None, 10, 4, 8, 128, 8 * 16 * 128, 16 * 128, 128)
    invalid = 9                           # hipErrorInvalidConfiguration

    def gather(M):                        # 256 threads for a row of 8 heads of 128
        return launch(FAKE, M, C.byref(view), False, AWAY, 1024, AWAY << 1, 1024, None)
    assert gather(1 << 24) == invalid
    assert gather((1 << 24) - 1) != invalid          # (there is no device for it here)
