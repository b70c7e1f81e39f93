"""Activations far left of zero, where exp(-v) is near the end of float32's range or beyond: small results, not zeros."""
import pytest
import torch

from experts_util import linear_act
from gpu_util import binding
from mx_util import TYPES, held
from oracle import experts_oracle as E

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act,lo,hi", [("silu", -104.0, -75.0), ("gelu_tanh", -11.0, -9.0)])
@pytest.mark.parametrize("n,k,m", [(512, 64, 2), (2000, 640, 1), (4200, 2100, 2), (4200, 2100, 40), (1290, 650, 3500)])
def test_far_left(dtype, act, lo, hi, n, k, m):
    """The values are the biases: the weights are zero."""
    dt = TYPES[dtype]
    codes, scales = held(torch.zeros((n, k), device="cuda"))
    bias = torch.linspace(lo, hi, n)
    x = torch.ones((m, k), dtype=dt, device="cuda")
    v = bias.double()
    for gated in (False, True):
        b = torch.cat((bias[::2], torch.ones(n // 2))) if gated else bias
        y = linear_act(codes, scales, b.cuda(), x, torch.empty((m, n // 2 if gated else n), dtype=dt, device="cuda"), activation=act, gated=gated)
        a = v[::2] if gated else v
        ref = torch.from_numpy(E.activate(a.numpy(), act))
        # SILU: exp (2 units of the last bit), an addition (half), a quotient (2), a product (half); GELU_TANH: its argument u is rounded in four steps, so that
        # exp is off by 4 |u| units more, |u| = 0.8 * 2 (|v| + 0.0447 |v|^3).  A subnormal exponential is off by 2 units of 2^-149.
        units = 5.0 if act == "silu" else 5.0 + 4 * 1.6 * (a.abs() + 0.045 * a.abs() ** 3)
        tol = units * 2.0 ** -23 * ref.abs() + a.abs() * 2.0 ** -148 + 2.0 ** -149
        tol = tol + torch.finfo(dt).eps / 2 * (ref.abs() + tol) + torch.finfo(dt).smallest_normal * torch.finfo(dt).eps
        assert ((y.double().cpu() - ref).abs() <= tol).all()
