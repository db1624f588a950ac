"""What the few-token products' launcher refuses, without a GPU: it answers before any launch
(the pointers are never dereferenced)."""
import ctypes
import os

import pytest

from paper_2602_03839_amd import pulse

A = 1 << 20  # fake, aligned "device" address
FP8, MXFP4, BF16 = 0, 1, 2
INVALID = 1  # hipErrorInvalidValue
NAME = "_ZN5pulse18launch_lowp_matmulENS_10WeightFormEbRKNS_16LowpMatmulParamsEP12ihipStream_t"


class Params(ctypes.Structure):
    """LowpMatmulParams up to its epilogue, which is nulls."""
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("inv_scale", ctypes.c_float),
                ("rows", ctypes.c_uint32), ("cols", ctypes.c_uint32), ("code_bytes", ctypes.c_uint64),
                ("scale_bytes", ctypes.c_uint64), ("x", ctypes.c_void_p), ("x_stride", ctypes.c_uint64),
                ("tokens", ctypes.c_uint32), ("y", ctypes.c_void_p), ("y_stride", ctypes.c_uint64),
                ("y_bf16", ctypes.c_int), ("e", ctypes.c_uint64 * 16)]


@pytest.mark.parametrize("cols", [64, 72, 65, 1 << 16])
def test_bf16_weights_have_no_kernel_for_more_tokens(cols):
    """More than 16 tokens of a BF16 weight are an error, where some sizes launched nothing
    and reported success, and others would have dropped tokens."""
    if not os.path.exists(pulse.LIB_PATH):
        from paper_2602_03839_amd import build
        build.build()
    launch = getattr(pulse.lib(), NAME)
    launch.restype, launch.argtypes = ctypes.c_int, [ctypes.c_int, ctypes.c_bool, ctypes.POINTER(Params), ctypes.c_void_p]
    for tokens in (17, 32, 33, 64, 65, 1 << 20):
        p = Params(codes=A, inv_scale=1.0, rows=32, cols=cols, code_bytes=64 * cols, x=A, x_stride=cols, tokens=tokens,
                   y=A, y_stride=32, y_bf16=1)
        assert launch(BF16, True, ctypes.byref(p), None) == INVALID, tokens
    p = Params(cols=cols)  # no tokens: nothing to do
    assert launch(BF16, True, ctypes.byref(p), None) != INVALID
