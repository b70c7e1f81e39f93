"""Arguments of the microscaled calls that are ignored are not refused (no GPU: the calls get as far as looking for one)."""
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
