"""A wait that runs out in the few-row kernel where it takes an expert's rows more than once: NaN in every row."""
import pytest
import torch

from experts_util import linear_experts, plan_of
from gpu_util import binding
from mx_util import TYPES, activations, held, weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("t,top_k", [(1, 5), (2, 2), (2, 7)])
@pytest.mark.parametrize("in_order", [False, True])
@pytest.mark.parametrize("e,n,k", [(2, 258, 1100), (3, 9000, 3000), (9, 40000, 300)])
def test_a_wait_that_runs_out_with_an_expert_more_than_once(dtype, t, top_k, in_order, e, n, k):
    b, dt, top_k = binding(), TYPES[dtype], min(top_k, e)
    codes, scales = held(weights(e * n, k, 1))
    codes, scales = codes.view(e, n, -1), scales.view(e, n, -1)
    ids = torch.full((t, top_k), e - 1, dtype=torch.int32, device="cuda")      # one expert has all rows
    ids[0, 0] = 0
    plan = plan_of(ids, e)
    x = activations(t * top_k if in_order else t, k, dt, 3)
    want = linear_experts(codes, scales, None, x, plan, top_k, torch.empty((t * top_k, n), dtype=dt, device="cuda"), activation="relu", x_sorted=in_order)
    y = torch.zeros_like(want)
    b.aiq_debug_mx_expire_wait(20000)
    linear_experts(codes, scales, None, x, plan, top_k, y, activation="relu", x_sorted=in_order)
    assert torch.isnan(y).all()
    linear_experts(codes, scales, None, x, plan, top_k, y, activation="relu", x_sorted=in_order)
    assert torch.equal(y, want)
