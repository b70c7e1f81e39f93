"""Microscaled products at the limits of the format and of their precision, on the GPU against float64."""
import numpy as np
import pytest
import torch

from gpu_util import binding
from mx_util import TYPES, activations, check, held, linear, values, weights

pytestmark = pytest.mark.gpu


# Scale bytes 253 and 254 make 6 * 2^127 of an element, which is no float32.  The stored value is finite all the same, and so is its
# product with a small x.
@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("n,k,m", [(64, 96, 1), (64, 100, 3), (70, 130, 9), (1100, 1000, 1), (700, 2000, 40)])
@pytest.mark.parametrize("workspace", [True, False])
def test_linear_with_scale_bytes_at_both_ends(dtype, n, k, m, workspace):
    dt = TYPES[dtype]
    codes, scales = held(weights(n, k, 1))
    for row, byte in ((1, 254), (2, 253), (3, 252), (4, 0), (5, 1)):
        scales[row, 0] = byte
    x = activations(m, k, torch.float32, 2)
    x[:, :32] = 0 if dtype == "f16" else x[:, :32] * 2.0 ** -115       # a half times 2^126 is out of a half's range
    x[:, 4:9] = 0
    x = x.to(dt)
    y = linear(codes, scales, None, x, torch.full((m, n), float("nan"), dtype=dt, device="cuda"), workspace)
    check(y, x.double().cpu().numpy(), values(codes, scales, k), None, dt, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,k,m", [(64, 96, 1), (64, 100, 3), (70, 130, 9), (700, 2000, 40)])
def test_matmul_with_scale_bytes_at_both_ends(dtype, n, k, m):
    """Blocks near the top of either matrix against blocks near the bottom of the other, and against zeros."""
    b, dt = binding(), TYPES[dtype]
    ac, as_ = held(activations(m, k, torch.float32, 3))
    bc, bs = held(weights(n, k, 4))
    as_[:, 0], as_[:, 1] = 10, 254
    bs[:, 0], bs[:, 1] = 118, 5
    bs[1, 0], bs[2, 0] = 254, 253
    as_[m - 1, 1] = 253
    ac[:, 32:48] = 0                                                   # block 2 of A is zeros, of B at the top
    bs[3, 2] = 254
    y = torch.full((m, n), float("nan"), dtype=dt, device="cuda")
    b.aiq_mx_matmul(ac, as_, bc, bs, None, k, y)
    check(y, values(ac, as_, k), values(bc, bs, k), None, dt, "mx")
