"""The launches of a layer of experts as aiq_profile_start and aiq_profile_stop count them."""
import pytest
import torch

from experts_util import new_plan, some_ids
from gpu_util import binding

pytestmark = pytest.mark.gpu


def _launches(call):
    b = binding()
    call()
    b.aiq_profile_start()
    call()
    return b.aiq_profile_stop()["qlinear"]


@pytest.mark.parametrize("t,plans", [(3, 0), (16, 0), (17, 1), (5000, 1)])
def test_plans_are_counted(t, plans):
    """Up to 16 tokens a plan is made with the choices, or in one launch; beyond that by a launch of its own."""
    b, e, top_k = binding(), 64, 4
    ids, w, plan = some_ids(t, top_k, e, t), torch.empty((t, top_k), device="cuda"), new_plan(t, top_k, e)
    logits = torch.randn((t, e), device="cuda")
    planned = _launches(lambda: b.aiq_plan_experts(ids, e, plan))
    routed = _launches(lambda: b.aiq_route_experts(logits, ids.clone(), w))
    both = _launches(lambda: b.aiq_route_experts(logits, ids.clone(), w, plan=plan))
    assert (planned["launches"], routed["launches"], both["launches"]) == (1 + plans, 1, 1 + plans)
    assert planned["ms"] > 0 and planned["bytes"] >= 4 * 3 * t * top_k
    if plans:
        assert both["bytes"] == routed["bytes"] + 4 * (3 * t * top_k + e + 1)
