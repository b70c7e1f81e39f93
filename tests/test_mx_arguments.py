"""Sizes and strides of the microscaled calls: what is ignored is not refused, what no argument can hold is (no GPU needed)."""
import pytest


@pytest.fixture(scope="module")
def aiq():
    from paper_2512_14090_b200 import build
    build.build()
    from paper_2512_14090_b200 import binding
    return binding


@pytest.mark.parametrize("stride", [-1, 0, 1 << 62])
def test_the_stride_of_a_single_row(aiq, stride):
    import torch
    if torch.cuda.is_available():
        pytest.skip("would launch with made-up addresses")
    one, L, f16 = 4096, aiq.lib, aiq.DTYPE_F16
    for status in (L.aiq_mx_quantize(one, f16, 1, 32, stride, one, one, None),
                   L.aiq_mx_dequantize(one, one, 1, 32, f16, one, stride, None),
                   L.aiq_mx_linear(one, one, None, 8, 32, one, f16, 1, stride, one, stride, None, 0, None),
                   L.aiq_mx_matmul(one, one, 1, one, one, 8, None, 32, one, f16, stride, None)):
        assert status in (aiq.ERR_CUDA, aiq.ERR_NOT_SM100), aiq.last_error()


@pytest.mark.parametrize("k", [2 ** 31, 2 ** 32 + 5, 2 ** 40 + 512, -2 ** 32 + 64])
def test_sizes_that_no_int_holds(aiq, k):
    """They are refused, not cut to their low 32 bits, by the plain ctypes functions too."""
    one, L, E, f16 = 4096, aiq.lib, aiq.ERR_INVALID_ARG, aiq.DTYPE_F16
    assert aiq.aiq_mx_row_bytes(k) == 0 and aiq.aiq_mx_scale_row_bytes(k) == 0
    for sizes in ((k, 4096, 64), (4096, k, 64), (4096, 4096, k)):
        assert L.aiq_mx_linear_workspace_bytes(*sizes, f16) == 0
    assert L.aiq_mx_quantize(one, f16, 4, k, k, one, one, None) == E
    assert L.aiq_mx_quantize(one, f16, k, 32, 32, one, one, None) == E
    assert L.aiq_mx_dequantize(one, one, 4, k, f16, one, k, None) == E
    assert L.aiq_mx_linear(one, one, None, k, 32, one, f16, 4, 32, one, abs(k), None, 0, None) == E
    assert L.aiq_mx_linear(one, one, None, 8, 32, one, f16, k, 32, one, 8, None, 0, None) == E
    assert L.aiq_mx_matmul(one, one, 4, one, one, 8, None, k, one, f16, 8, None) == E
