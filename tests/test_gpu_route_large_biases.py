"""Routing with biases far larger than the scores: choices are rounded at the biases' size, so float32 alone cannot order them."""
import numpy as np
import pytest
import torch

from experts_util import new_plan
from gpu_util import binding
from oracle import experts_oracle as O

pytestmark = pytest.mark.gpu

LOWEST = torch.finfo(torch.float32).min


def _route(logits, top_k, bias, **how):
    t, e = logits.shape
    ids = torch.full((t, top_k), 77, dtype=torch.int32, device="cuda")
    w = torch.full((t, top_k), 77.0, device="cuda")
    binding().aiq_route_experts(logits.cuda(), ids, w, bias=bias.cuda(), plan=new_plan(t, top_k, e), **how)
    return ids.cpu().numpy()


def _check(logits, top_k, bias, **how):
    ids = _route(logits, top_k, bias, **how)
    want = O.route(logits.double().numpy(), bias.numpy(), top_k=top_k, **how)[0]
    wrong = (ids != want).any(axis=1)
    assert not wrong.any(), f"{wrong.sum()} of {len(ids)} tokens, the first {np.flatnonzero(wrong)[0]}"


def test_two_best_that_cancel():
    """In float64 the groups count 1.276519 and 1.277131; with choices rounded to float32 1.277344 and 1.277131."""
    bias = torch.tensor([3e4, -3e4, -3e4, -3e4, 0, 0, 0, 0])
    logits = torch.tensor([[0.38631517, -0.17255656, 0.75894272, 0.32788253, 0.68614733, -0.64194930, -1.07925999, 0.45581980]])
    _check(logits, 2, bias, scoring="sigmoid", groups=2, top_groups=1, group_best=2)


@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("size", [1.0, 64.0, 1000.0, 2.0 ** 14, 1e5])
@pytest.mark.parametrize("e,groups,top_groups,top_k", [(16, 8, 3, 4), (64, 8, 3, 8), (48, 4, 2, 6), (12, 6, 5, 3)])
def test_groups_with_biases_of_both_signs(scoring, size, e, groups, top_groups, top_k):
    """One expert of every group far up and one as far down (the others at the bottom): the sums of two are as close as scores are."""
    t, n = 2000, e // groups
    g = torch.Generator().manual_seed(int(size) + e)
    bias = torch.full((groups, n), -4 * size)
    bias[:, 0] = size
    bias[:, n - 1] = -size
    logits = 0.5 * torch.randn((t, e), generator=g)
    for best in (1, 2):
        _check(logits, top_k, bias.flatten(), scoring=scoring, groups=groups, top_groups=top_groups, group_best=best)
    # sums of two that float32 cannot tell apart at all
    logits = 0.5 + torch.randint(-2, 3, (t, e), generator=g) * 2.0 ** -22
    _check(logits, top_k, bias.flatten(), scoring=scoring, groups=groups, top_groups=top_groups, group_best=2)


@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("size", [16.0, 64.0, 256.0])
@pytest.mark.parametrize("e,top_k,above", [(24, 3, 2), (64, 6, 2), (64, 8, 6), (200, 31, 20)])
def test_order_of_choices_with_a_large_bias(scoring, size, e, top_k, above):
    """Some experts are lifted far above the last one that is chosen, by biases that undo the differences of their scores: their choices are as
    close as logits can be, and may lie on either side of a float32 number."""
    t = 3000
    g = torch.Generator().manual_seed(e)
    most = 0.8 if scoring == "sigmoid" else 0.8 / above
    lifted = torch.randperm(e, generator=g)[:above]
    bias = torch.zeros(e)
    bias[lifted] = size + 0.5 * most * torch.rand(above, generator=g)
    p = most * (0.75 + 0.25 * torch.rand((t, 1), generator=g, dtype=torch.float64)) - (bias[lifted].double() - size)
    if scoring == "sigmoid":
        logits = torch.full((t, e), -3.0) + torch.randn((t, e), generator=g)
        logits[:, lifted] = torch.log(p / (1 - p)).float()
    else:
        rest = (1 - p.sum(dim=1, keepdim=True)) / (e - above)
        logits = torch.log(rest).float().repeat(1, e)
        logits[:, lifted] = torch.log(p).float()
    _check(logits, top_k, bias, scoring=scoring)


@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("size", [1e9, -LOWEST])
def test_groups_masked_by_a_large_finite_bias(scoring, size):
    """Groups of which one or all experts are masked are groups all the same; a sum of two below the lowest float32 is no infinity."""
    t, e, groups, n = 500, 32, 4, 8
    g = torch.Generator().manual_seed(3)
    logits = torch.randn((t, e), generator=g)
    bias = 0.1 * torch.randn((groups, n), generator=g)
    bias[3] = -size
    bias[2, 1:] = -size
    barred = bias.clone()
    barred[0] = -np.inf
    high = bias.clone()
    high[0, 2:4] = high[1, 5:] = size
    for b in (bias, barred, high, barred.flip(0), high.flip(0)):
        for top_groups in (1, 2, 3, 4):
            for best in (1, 2):
                _check(logits, 8 * top_groups - 3, b.flatten(), scoring=scoring, groups=groups, top_groups=top_groups, group_best=best)
