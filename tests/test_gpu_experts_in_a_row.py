"""Calls of the experts' products one behind the other, where one has nothing to do."""
import pytest
import torch

from experts_util import linear_experts, new_plan, some_ids
from gpu_util import binding
from mx_util import TYPES, activations, held, weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("t", [3, 40, 2000])
def test_a_call_without_rows_before_one_with_rows(dtype, t):
    """No token has an expert; the plan, x and the workspace then change hands at once."""
    b, dt, e, n, k, top_k = binding(), TYPES[dtype], 6, 256, 1100, 2
    codes, scales = held(weights(e * n, k, 1))
    codes, scales = codes.view(e, n, -1), scales.view(e, n, -1)
    none = torch.full((t, top_k), -1, dtype=torch.int32, device="cuda")
    ids = [some_ids(t, top_k, e, 5 + i) for i in range(2)]
    xs = [activations(t, k, dt, 3 + i) for i in range(3)]
    plan = new_plan(t, top_k, e)
    want = []
    for i in range(2):
        b.aiq_plan_experts(ids[i], e, plan)
        want.append(linear_experts(codes, scales, None, xs[i], plan, top_k, torch.empty((t * top_k, n), dtype=dt, device="cuda"), activation="silu"))
    ws = torch.empty(b.aiq_mx_linear_experts_workspace_bytes(e, n, k, t * top_k, dt), dtype=torch.uint8, device="cuda")
    ys = [torch.zeros_like(want[0]) for _ in range(20)]
    empty = torch.full_like(want[0], 7.0)
    x = xs[2].clone()
    torch.cuda.synchronize()
    for i, y in enumerate(ys):
        b.aiq_plan_experts(none, e, plan)
        b.aiq_mx_linear_experts(codes, scales, None, x, plan, top_k, empty, "silu", workspace=ws)
        b.aiq_plan_experts(ids[i % 2], e, plan)
        x.copy_(xs[i % 2])
        b.aiq_mx_linear_experts(codes, scales, None, x, plan, top_k, y, "silu", workspace=ws)
    for i, y in enumerate(ys):
        assert torch.equal(y, want[i % 2])
    assert (empty == 7.0).all()
