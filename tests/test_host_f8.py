"""Refusals of the 8-bit floating-point entry points that happen before any CUDA call, and the sizes the binding computes."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def xq():
    from paper_2503_17513_b200 import build, xq as binding

    build.build_library()
    return binding


def test_null_and_bad_arguments_rejected_before_any_cuda_call(xq):
    L, null, out = xq.lib(), ctypes.c_void_p(0), ctypes.c_void_p()
    some = ctypes.c_void_p(1 << 20)  # never dereferenced: every call below is refused on its sizes or its other pointers
    bad = xq.ERR_INVALID_ARG
    assert L.xq_f8_prepare_weights(null, 4, 8, null, ctypes.byref(out)) == bad
    assert L.xq_f8_prepare_weights(some, 0, 8, null, ctypes.byref(out)) == bad
    assert L.xq_f8_prepare_weights(some, 8, (1 << 24) + 1, null, ctypes.byref(out)) == bad
    assert L.xq_f8_weights_import(null, null, 4, 8, null, ctypes.byref(out)) == bad
    assert L.xq_f8_weights_import(some, some, 4, 0, null, ctypes.byref(out)) == bad
    assert L.xq_f8_weights_export(null, null, null) == bad
    assert L.xq_f8_weights_info(null, None, None) == bad
    assert L.xq_f8_workspace_bytes(4, null) == 0
    assert L.xq_f8_quant(null, 4, 8, 8, null, null, null) == bad
    assert L.xq_f8_quant(null, 0, 8, 8, null, null, null) == xq.OK  # no rows: a no-op
    assert L.xq_f8_quant(some, 4, 0, 8, some, some, null) == bad
    assert L.xq_f8_quant(some, 4, 65537, 65544, some, some, null) == bad  # longer than a row may be
    assert L.xq_f8_quant(some, 4, 16, 8, some, some, null) == bad         # pitch below the row
    assert L.xq_f8_quant(some, 4, 16, 20, some, some, null) == bad        # pitch not a multiple of 8
    assert L.xq_f8_quant(ctypes.c_void_p((1 << 20) + 2), 4, 16, 16, some, some, null) == bad
    assert L.xq_f8_norm_quant(null, 4, 8, 8, null, 0, null, 1e-5, null, null, null, null, 0, null) == bad
    assert L.xq_f8_norm_quant(null, 0, 8, 8, null, 0, null, 1e-5, null, null, null, null, 0, null) == xq.OK
    assert L.xq_f8_norm_quant(some, 4, 8, 8, null, 0, some, -1.0, null, some, some, null, 0, null) == bad
    assert L.xq_f8_norm_quant(some, 4, 8, 8, some, 4, some, 1e-5, null, some, some, null, 0, null) == bad  # residual pitch
    assert L.xq_f8_gemm(null, null, 4, null, null, null, 0, null) == bad
    assert L.xq_f8_linear(null, 4, 8, null, null, null, 0, null) == bad
    assert L.xq_f8_gated(null, null, 4, null, null, null, null, null, null, 0, null) == bad
    L.xq_f8_weights_free(null)


def test_sizes(xq):
    assert [xq.f8_padded(k) for k in (1, 128, 129, 4096)] == [128, 128, 256, 4096]
    assert [xq.f8_scale_pitch(k) for k in (1, 128, 512, 513, 4096)] == [4, 4, 4, 8, 32]


def test_native_calls_check_their_arguments(xq):
    """Wrong names, kinds and places of arguments are Python errors, raised before anything reaches the library."""
    import torch

    X, c = torch.zeros((2, 8), dtype=torch.bfloat16), torch.zeros((2, 128), dtype=torch.uint8)
    with pytest.raises(TypeError):
        xq.xq_f8_quant(X, c)
    with pytest.raises(TypeError):
        xq.xq_f8_quant(X, c, c, nonsense=1)
    with pytest.raises(TypeError):
        xq.xq_f8_quant(X, c, c, codes=c)
    with pytest.raises(TypeError):
        xq.xq_f8_quant(X, c, c, None, None)
    with pytest.raises(AssertionError):
        xq.xq_f8_quant(X, c, c)  # not on a GPU
    with pytest.raises(AssertionError):
        xq.xq_f8_quant(3, c, c)
    with pytest.raises(AttributeError):
        xq.xq_f8_gemm(c, c, 2, X, c, c)  # no weights object
    with pytest.raises(AttributeError):
        xq.no_such_call
