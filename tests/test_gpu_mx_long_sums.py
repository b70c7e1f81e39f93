"""16-bit results of sums so long that they leave the accumulator every 512 k, in the layer with a way out and in the experts' products."""
import numpy as np
import pytest
import torch

from experts_util import linear_act, linear_experts, plan_of, some_ids, tail_check
from mx_util import TYPES, held, values, weights
from oracle import experts_oracle as O

pytestmark = pytest.mark.gpu

LONG = {"f16": 33000, "bf16": 262700}                    # beyond 32,768 and 262,144


def _x(m, k, dt, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn((m, k), generator=g, device="cuda") * torch.exp(0.8 * torch.randn((1, k), generator=g, device="cuda"))).to(dt)


@pytest.mark.parametrize("dtype", sorted(LONG))
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("m", [7, 20, 130, 3200])
def test_linear_act(dtype, gated, m):
    """Tiles with a split of K, and as many as write what they have directly."""
    dt, n, k = TYPES[dtype], 258, LONG[dtype]
    codes, scales = held(weights(n, k, 1))
    outputs = n // 2 if gated else n
    x = _x(m, k, dt, 2)
    g = torch.Generator().manual_seed(3)
    bias, residual = torch.randn(n, generator=g).cuda(), torch.randn((m, outputs), generator=g).to(dt).cuda()
    y = linear_act(codes, scales, bias, x, torch.full((m, outputs), float("nan"), dtype=dt, device="cuda"), activation="silu", gated=gated, residual=residual)
    assert torch.isfinite(y).all()
    rows = torch.unique(torch.cat((torch.tensor([0, m - 1]), torch.randint(0, m, (20,), generator=g)))).cuda()
    tail_check(y[rows], x[rows].double().cpu().numpy(), values(codes, scales, k), bias.double().cpu().numpy(), dt, dtype, "silu", gated,
               residual[rows].double().cpu().numpy())


@pytest.mark.parametrize("dtype", sorted(LONG))
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("t,top_k,e,in_order", [(6, 1, 2, False), (30, 2, 3, True), (100, 1, 2, False), (90, 2, 2, True), (700, 2, 3, False)])
def test_experts(dtype, gated, t, top_k, e, in_order):
    """Narrow blocks of rows, and wide ones, whose pieces come in one copy."""
    dt, n, k = TYPES[dtype], 130, LONG[dtype]
    codes, scales = held(weights(e * n, k, 1))
    codes, scales = codes.view(e, n, -1), scales.view(e, n, -1)
    outputs = n // 2 if gated else n
    ids = some_ids(t, top_k, e, t, padded=t // 8)
    offsets, slots, _ = O.plan(ids.cpu().numpy(), e)
    x = _x(t * top_k if in_order else t, k, dt, 2)
    bias = torch.randn((e, n), generator=torch.Generator().manual_seed(3)).cuda()
    y = torch.full((t * top_k, outputs), 7.0, dtype=dt, device="cuda")
    linear_experts(codes, scales, bias, x, plan_of(ids, e), top_k, y, activation="gelu_tanh", gated=gated, x_sorted=in_order)
    assert torch.isfinite(y).all() and (y[offsets[-1]:] == 7.0).all()
    rng = np.random.default_rng(t)
    for i in range(e):
        rows = np.arange(offsets[i], offsets[i + 1])
        if len(rows):
            rows = np.unique(np.concatenate((rows[[0, -1]], rng.choice(rows, 12))))
            of = torch.from_numpy(rows if in_order else slots[rows] // top_k).long().cuda()
            tail_check(y[torch.from_numpy(rows).cuda()], x[of].double().cpu().numpy(), values(codes[i], scales[i], k), bias[i].double().cpu().numpy(), dt, dtype,
                       "gelu_tanh", gated, what=f"expert {i}")
