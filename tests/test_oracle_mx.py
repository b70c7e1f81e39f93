"""The microscaled oracle against rows worked out by hand, and the layout the C ABI reports."""
import numpy as np
import pytest

from oracle import mx_oracle as X


@pytest.fixture(scope="module")
def aiq():
    from paper_2512_14090_b200 import build
    build.build()
    from paper_2512_14090_b200 import binding
    return binding


def _one_block(values):
    row = np.zeros((1, 32))
    row[0, :len(values)] = values
    codes, scales = X.quantize(row)
    return codes, scales, X.dequantize(codes, scales, 32)[0, :len(values)]


def test_elements_and_ties():
    # the largest is 6, so the unit is 1: exponent byte 127; halfway cases go to the element whose last bit is zero
    codes, scales, v = _one_block([6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -5, -0.25, 0.26, 2.51])
    assert scales[0, 0] == 127
    assert v.tolist() == [6, 0, 1, 1, 2, 2, 4, 4, -4, 0, 0.5, 3]
    assert codes[0, 0] == 0x07 and codes[0, 4] == 0x8E and codes[0, 1] == 0x22


def test_scale_byte():
    for top, byte in ((4.0, 127), (7.99, 127), (8.0, 128), (3.99, 126), (2.0 ** -126, 0), (2.0 ** -124, 1), (0.0, 0),
                      (3.4e38, 252), (1e-40, 0)):
        codes, scales, v = _one_block([top])
        assert scales[0, 0] == byte, top
    assert _one_block([7.99])[2][0] == 6.0                       # saturates
    assert _one_block([2.0 ** -127])[2][0] == 2.0 ** -127


def test_nonfinite_block_is_nan_and_stays_in_its_block():
    row = np.ones((1, 70))
    row[0, 40] = np.inf
    codes, scales = X.quantize(row)
    v = X.dequantize(codes, scales, 70)
    assert np.isnan(v[0, 32:64]).all() and (v[0, :32] == 1).all() and (v[0, 64:] == 1).all()
    assert (codes[0, 16:32] == 0).all()


def test_layout_sizes(aiq):
    for k in (1, 31, 32, 33, 127, 128, 129, 512, 513, 8192, 100001):
        assert aiq.aiq_mx_row_bytes(k) == X.row_bytes(k)
        assert aiq.aiq_mx_scale_row_bytes(k) == X.scale_row_bytes(k)
    assert aiq.aiq_mx_row_bytes(0) == 0 and aiq.aiq_mx_scale_row_bytes(-3) == 0


def test_refusals_of_the_c_abi(aiq):
    one, odd16, odd = 4096, 4096 + 16, 4096 + 1
    L, E = aiq.lib, aiq.ERR_INVALID_ARG
    f32, f16 = aiq.DTYPE_F32, aiq.DTYPE_F16
    quant = lambda x=one, dt=f32, r=4, k=32, st=32, c=one, s=one: L.aiq_mx_quantize(x, dt, r, k, st, c, s, None)
    for bad in (dict(x=None), dict(c=None), dict(s=None), dict(dt=3), dict(dt=-1), dict(r=0), dict(k=0), dict(r=-1), dict(st=-1), dict(k=(1 << 30) + 1), dict(r=2 ** 31 - 1),
                dict(c=odd16), dict(s=odd), dict(x=odd), dict(x=one + 2)):
        assert quant(**bad) == E, bad
        assert "aiq_mx_quantize" in aiq.last_error()
    deq = lambda c=one, s=one, r=4, k=32, dt=f32, y=one, st=32: L.aiq_mx_dequantize(c, s, r, k, dt, y, st, None)
    for bad in (dict(y=None), dict(c=None), dict(s=None), dict(dt=7), dict(r=0), dict(k=0), dict(st=31), dict(c=odd16), dict(y=odd)):
        assert deq(**bad) == E, bad
    lin = lambda c=one, s=one, b=None, n=8, k=32, x=one, dt=f16, m=4, xs=32, y=one, ys=8, ws=None, wb=0: \
        L.aiq_mx_linear(c, s, b, n, k, x, dt, m, xs, y, ys, ws, wb, None)
    for bad in (dict(c=None), dict(s=None), dict(x=None), dict(y=None), dict(n=0), dict(k=0), dict(m=0), dict(dt=9), dict(ys=7),
                dict(xs=-2), dict(c=odd16), dict(s=odd), dict(y=odd), dict(b=odd)):
        assert lin(**bad) == E, bad
    big = dict(n=4096, k=4096, m=64, xs=4096, ys=4096)
    assert lin(**big, ws=odd, wb=1 << 30) == E and "workspace" in aiq.last_error()
    assert lin(**big, ws=one, wb=16) == aiq.ERR_WORKSPACE_TOO_SMALL
    mat = lambda ac=one, as_=one, m=4, bc=one, bs=one, n=8, b=None, k=32, y=one, dt=f16, ys=8: \
        L.aiq_mx_matmul(ac, as_, m, bc, bs, n, b, k, y, dt, ys, None)
    for bad in (dict(ac=None), dict(as_=None), dict(bc=None), dict(bs=None), dict(y=None), dict(m=0), dict(n=0), dict(k=0), dict(dt=4),
                dict(ys=7), dict(n=2 ** 31 - 1, ys=2 ** 31), dict(ac=odd16), dict(bs=odd), dict(b=odd)):
        assert mat(**bad) == E, bad
    assert aiq.lib.aiq_mx_linear_workspace_bytes(0, 32, 1, f16) == 0
    assert aiq.lib.aiq_mx_linear_workspace_bytes(64, 32, 1, 5) == 0
    assert aiq.lib.aiq_mx_linear_workspace_bytes(64, 2 ** 31 - 1, 64, f16) == 0
    assert lin(m=(1 << 30) + 1) == E


def test_refusals_of_the_binding(aiq):
    import torch
    with pytest.raises(ValueError):
        aiq.aiq_mx_quantize(torch.zeros(2, 32), torch.zeros(2, 64, dtype=torch.uint8), torch.zeros(2, 16, dtype=torch.uint8))
    with pytest.raises(ValueError):
        aiq.aiq_mx_linear_workspace_bytes(64, 64, 1, torch.float64)
