"""Inputs, tolerances and calls that the tests of the microscaled operators share."""
import numpy as np
import torch

from gpu_util import binding
from oracle import mx_oracle as X

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
# tensor-core passes over x: its values enter as that many pieces of 5 bits (see aiq.h)
PIECES = {"f32": 5, "f16": 3, "bf16": 2, "mx": 1}


def held(x):
    """Microscaled form of a CUDA matrix, by the library."""
    b = binding()
    rows, k = x.shape
    codes = torch.full((rows, X.row_bytes(k)), 0xAA, dtype=torch.uint8, device="cuda")
    scales = torch.full((rows, X.scale_row_bytes(k)), 0xAA, dtype=torch.uint8, device="cuda")
    b.aiq_mx_quantize(x, codes, scales)
    return codes, scales


def values(codes, scales, k):
    """float64 values of the stored rows, by the oracle."""
    return X.dequantize(codes.cpu().numpy(), scales.cpu().numpy(), k)


def weights(n, k, seed):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((n, k), generator=g) * 0.02 * torch.exp(0.5 * torch.randn((n, 1), generator=g))).cuda()


def activations(m, k, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((m, k), generator=g) * torch.exp(0.8 * torch.randn((1, k), generator=g))).to(dtype).cuda()


def bound(x, w, ref, dtype, kind):
    """How far y may be from its float64 value.

    Sums: the products are exact.  They are added up in chains of at most ceil(K / 32) additions per piece of x (a tensor-core
    step adds 32 products to the accumulator), plus 64 for the products within a step and the joining of partial sums; an
    addition is off by at most one unit of the last bit, 2^-23 of the sum's magnitude, which never exceeds sum |x w|.
    Pieces: a value far below the largest |x| of its block of 32 is held to 2^-(12 + 5 pieces) of that largest value.
    Rounding to the output type: half a unit.
    """
    s = np.abs(x) @ np.abs(w).T
    pieces = PIECES[kind]
    k = x.shape[1]
    err = (-(-k // 32) * pieces + 64) * 2.0 ** -23 * s
    if kind != "mx":
        pad = -k % X.BLOCK
        xb = np.pad(np.abs(x), ((0, 0), (0, pad))).reshape(x.shape[0], -1, X.BLOCK).max(axis=2)
        wb = np.pad(np.abs(w), ((0, 0), (0, pad))).reshape(w.shape[0], -1, X.BLOCK).sum(axis=2)
        err = err + 2.0 ** -(12 + 5 * pieces) * (xb @ wb.T)
    half = torch.finfo(dtype).eps / 2
    tiny = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    return err + half * (np.abs(ref) + err) + tiny


def check(y, x, w, bias, dtype, kind, what=""):
    ref = X.product(x, w, bias)
    got = y.double().cpu().numpy()
    tol = bound(x, w, ref, dtype, kind)
    assert np.isfinite(got).all(), what
    worst = (np.abs(got - ref) / tol).max()
    assert worst <= 1.0, f"{what}: error is {worst:.3g} of what is allowed"
    return worst


def linear(codes, scales, bias, x, y, workspace=True):
    b = binding()
    ws = None
    if workspace:
        size = b.aiq_mx_linear_workspace_bytes(y.shape[1], x.shape[1], x.shape[0], x.dtype)
        ws = torch.empty(size, dtype=torch.uint8, device="cuda") if size else None
    b.aiq_mx_linear(codes, scales, bias, x, y, workspace=ws)
    return y
