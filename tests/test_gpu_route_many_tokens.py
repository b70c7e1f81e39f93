"""Routing of more tokens than one pass of a warp for each takes, where eight lanes share a token whatever the number of experts: sampled rows against
the float64 oracle, all rows against the same rows in fewer tokens a call, where a warp has one token (more than 64 experts)."""
import numpy as np
import pytest
import torch

from experts_util import new_plan
from gpu_util import binding
from mx_util import TYPES
from oracle import experts_oracle as O

pytestmark = pytest.mark.gpu

SLICE = 2500


def _route(logits, top_k, bias=None, plan=None, **how):
    t = logits.shape[0]
    ids = torch.full((t, top_k), 77, dtype=torch.int32, device="cuda")
    w = torch.full((t, top_k), 77.0, device="cuda")
    binding().aiq_route_experts(logits, ids, w, bias=bias, plan=plan, **how)
    return ids, w


def _check(logits, top_k, bias=None, rows=60, **how):
    t, e = logits.shape
    plan = new_plan(t, top_k, e)
    ids, w = _route(logits, top_k, bias, plan, **how)
    parts = [_route(logits[a:a + SLICE], top_k, bias, **how) for a in range(0, t, SLICE)]
    assert torch.equal(ids, torch.cat([p[0] for p in parts]))
    # two orders of the same additions: sums of up to 1024 exponentials, 40 additions deep
    other = torch.cat([p[1] for p in parts])
    assert torch.equal(torch.isnan(w), torch.isnan(other))
    assert ((w - other).nan_to_num().abs() <= 80 * 2.0 ** -24 * other.nan_to_num().abs()).all()
    # sampled rows, the first and the last among them
    some = np.unique(np.concatenate(([0, t - 1, t - 2, t - 5], np.random.default_rng(t).integers(0, t, rows))))
    how.setdefault("scoring", "softmax")
    want_ids, want = O.route(logits[torch.from_numpy(some).cuda()].double().cpu().numpy(), None if bias is None else bias.cpu().numpy(), top_k=top_k, **how)
    assert np.array_equal(ids.cpu().numpy()[some], want_ids)
    got = w.double().cpu().numpy()[some]
    assert np.array_equal(np.isnan(got), np.isnan(want))
    # exponentials of arguments up to 200 that are rounded once, sums of up to 1024 terms by 137 additions at most, a quotient and a product
    assert (np.abs(np.nan_to_num(got) - np.nan_to_num(want)) <= (200 + 137 + 8) * 2.0 ** -23 * np.nan_to_num(np.abs(want)) + 2.0 ** -126).all()
    # the plan against a stable sort
    offsets, slots, positions = binding().aiq_expert_plan_parts(plan, t, top_k, e)
    flat = ids.reshape(-1).long()
    order = torch.sort(torch.where(flat < 0, e, flat), stable=True).indices
    n = int((flat >= 0).sum())
    assert torch.equal(offsets[1:].long(), torch.bincount(flat[flat >= 0], minlength=e).cumsum(0)) and int(offsets[0]) == 0
    assert torch.equal(slots[:n].long(), order[:n]) and (slots[n:] == -1).all()
    back = torch.full_like(flat, -1)
    back[order[:n]] = torch.arange(n, device="cuda")
    assert torch.equal(positions.reshape(-1).long(), back)


def _logits(t, e, dtype, seed, padded=0):
    g = torch.Generator().manual_seed(seed)
    l = torch.randn((t, e), generator=g) + 0.5 * torch.randn((1, e), generator=g)
    if padded:
        l[t - padded:] = -np.inf
    return l.to(TYPES[dtype]).cuda()


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("t,e,top_k,groups,top_groups", [(4737, 65, 6, 1, 1), (5003, 256, 8, 8, 4), (4737, 256, 8, 8, 3), (5003, 513, 9, 1, 1), (4737, 1024, 31, 1, 1),
                                                         (5003, 1024, 16, 32, 7), (5003, 96, 7, 32, 5), (4999, 300, 5, 5, 2), (4739, 64, 8, 2, 1), (9001, 128, 4, 4, 2)])
def test_many_tokens(dtype, t, e, top_k, groups, top_groups):
    logits = _logits(t, e, dtype, t + e, t // 16)
    bias = 0.1 * torch.randn(e, generator=torch.Generator().manual_seed(e)).cuda()
    bias[[0, e // 2]] = -np.inf
    for scoring in ("softmax", "sigmoid"):
        for b in (None, bias):
            for best in ((1, 2) if groups > 1 else (1,)):
                _check(logits, top_k, b, scoring=scoring, groups=groups, top_groups=top_groups, group_best=best, renormalise=scoring == "softmax")


@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("e,groups,top_groups,top_k", [(65, 1, 1, 6), (256, 8, 4, 8), (1024, 4, 2, 20)])
def test_ties_of_more_than_32_candidates(scoring, e, groups, top_groups, top_k):
    """A few values for all logits, and scores closer than float32."""
    t = 4751
    g = torch.Generator().manual_seed(e)
    logits = torch.randint(-1, 2, (t, e), generator=g).float()
    near = 0.5 + logits * 2.0 ** -22
    tiny = (torch.randint(0, 4, (e,), generator=g).float() * 2.0 ** -28).cuda()
    for best in ((1, 2) if groups > 1 else (1,)):
        how = dict(scoring=scoring, groups=groups, top_groups=top_groups, group_best=best, rows=40)
        for l, b in ((logits, None), (logits, torch.zeros(e).cuda()), (near, None), (near, tiny), (near, tiny + 100.0)):
            _check(l.cuda(), top_k, b, **how)


def test_what_is_not_a_number_among_many_tokens():
    t, e = 4801, 200
    logits = _logits(t, e, "f32", 1)
    logits[::7, 3] = float("nan")
    logits[1::7, 5] = float("inf")
    logits[2::7] = -np.inf
    logits[3::7, 4:] = -np.inf
    bias = 0.1 * torch.randn(e, generator=torch.Generator().manual_seed(e)).cuda()
    for scoring in ("softmax", "sigmoid"):
        for b in (None, bias):
            for groups, top_groups, best in ((1, 1, 1), (8, 3, 2)):
                _check(logits, 6, b, scoring=scoring, groups=groups, top_groups=top_groups, group_best=best)
