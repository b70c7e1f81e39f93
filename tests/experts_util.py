"""Tolerances and calls that the tests of the layer's way out and of the experts share."""
import numpy as np
import torch

from gpu_util import binding
from mx_util import bound
from oracle import experts_oracle as E
from oracle import mx_oracle as X

ACTS = ["none", "relu", "relu6", "silu", "gelu", "gelu_tanh"]


def act_bound(v, err, name):
    """How far act(v + err) in float32 may be from act(v).

    Slopes are at most 1.13.  SILU: exp (2 units of the last bit), an addition (half), a division (2), a product: below 8 units.  GELU_TANH: its
    argument u is rounded in four steps, so the exponent is off by 4 |u| units, which counts once as a relative error.  GELU: erfc (4 units)
    of an argument a that is off by a unit and a half, of which the relative slope is 2 |a| + 1 at most.  A quotient whose divisor is above 2^126 may be zero.
    """
    a = np.abs(v)
    units = {"none": 0.0, "relu": 0.0, "relu6": 0.0, "silu": 8.0, "gelu": 8.0 + 2 * (a * a + a), "gelu_tanh": 8.0 + 8 * 0.8 * (a + 0.045 * a ** 3)}[name]
    with np.errstate(over="ignore", invalid="ignore"):
        value = np.abs(E.activate(v, name))
    return 1.13 * err + units * 2.0 ** -23 * (value + 1.13 * err) + a * 2.0 ** -125


def tail_check(y, x, w, bias, dtype, kind, name, gated, residual=None, what=""):
    """y against the float64 layer: x [M][K] and w [N][K] float64, bias [N], residual [M][outputs]."""
    v = X.product(x, w, bias)
    err = bound(x, w, v, torch.float32, kind)                    # what the sums may be off, in float32 with their bias
    if gated:
        half = v.shape[1] // 2
        g, u = v[:, :half], v[:, half:]
        eg = act_bound(g, err[:, :half], name)
        h = E.activate(g, name)
        tol = eg * (np.abs(u) + err[:, half:]) + np.abs(h) * err[:, half:]
        ref = h * u
    else:
        tol = act_bound(v, err, name)
        ref = E.activate(v, name)
    tol = tol + 2.0 ** -24 * np.abs(ref)
    if residual is not None:
        ref = ref + residual
        tol = tol + 2.0 ** -24 * np.abs(ref)
    tol = tol + torch.finfo(dtype).eps / 2 * (np.abs(ref) + tol) + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    got = y.double().cpu().numpy()
    assert np.isfinite(got).all(), what
    worst = (np.abs(got - ref) / tol).max()
    assert worst <= 1.0, f"{what}: error is {worst:.3g} of what is allowed"


def linear_act(codes, scales, bias, x, y, workspace=True, **how):
    b = binding()
    ws = None
    if workspace:
        size = b.aiq_mx_linear_workspace_bytes(codes.shape[0], x.shape[1], x.shape[0], x.dtype)
        ws = torch.empty(size, dtype=torch.uint8, device="cuda") if size else None
    b.aiq_mx_linear_act(codes, scales, bias, x, y, workspace=ws, **how)
    return y


def new_plan(t, top_k, e):
    return torch.full((binding().aiq_expert_plan_bytes(t, top_k, e),), 0xCD, dtype=torch.uint8, device="cuda")


def plan_of(ids, e):
    plan = new_plan(*ids.shape, e)
    binding().aiq_plan_experts(ids, e, plan)
    return plan


def parts(plan, t, top_k, e):
    return [p.cpu().numpy() for p in binding().aiq_expert_plan_parts(plan, t, top_k, e)]


def some_ids(t, top_k, e, seed, padded=0):
    """Distinct experts for each token, some experts more popular than others; none in the last rows."""
    g = torch.Generator().manual_seed(seed)
    l = torch.randn((t, e), generator=g) + torch.randn((1, e), generator=g)
    ids = l.topk(top_k, dim=1).indices.int()
    if padded:
        ids[t - padded:] = -1
    return ids.cuda()


def linear_experts(codes, scales, bias, x, plan, top_k, y, **how):
    b = binding()
    e, n = codes.shape[:2]
    size = b.aiq_mx_linear_experts_workspace_bytes(e, n, x.shape[1], y.shape[0], x.dtype)
    ws = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")
    b.aiq_mx_linear_experts(codes, scales, bias, x, plan, top_k, y, workspace=ws, **how)
    return y
