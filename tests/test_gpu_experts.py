"""A layer of experts on the GPU against the float64 oracle: routing, plans, the experts' products, the weighted sum."""
import numpy as np
import pytest
import torch

from experts_util import ACTS, linear_experts, new_plan, parts, plan_of, some_ids, tail_check
from gpu_util import binding
from mx_util import TYPES, activations, held, values, weights
from oracle import experts_oracle as O

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------- plans
def _plan_check(plan, ids, e):
    for got, want in zip(parts(plan, *ids.shape, e), O.plan(ids.cpu().numpy(), e)):
        assert np.array_equal(got, want)


@pytest.mark.parametrize("t,top_k,e", [(1, 1, 1), (1, 4, 32), (3, 31, 1024), (16, 2, 2), (33, 6, 60), (64, 8, 256), (65, 8, 256), (100, 1, 5), (997, 6, 60),
                                       (2048, 3, 1000), (2500, 4, 8), (5000, 8, 130)])
def test_plan(t, top_k, e):
    for padded in (0, t // 3, t):
        ids = some_ids(t, top_k, e, t + e, padded)
        _plan_check(plan_of(ids, e), ids, e)


@pytest.mark.parametrize("t", [5, 700])
def test_plan_of_any_ids(t):
    """The same expert twice, ids that are none, all the same one."""
    g = torch.Generator().manual_seed(t)
    e = 7
    ids = torch.randint(-3, e + 3, (t, 5), generator=g, dtype=torch.int32)
    ids[0] = torch.tensor([2 ** 31 - 1, -2 ** 31, 3, 3, 3], dtype=torch.int32)
    clean = torch.where((ids < 0) | (ids >= e), -1, ids)
    plan = plan_of(ids.cuda(), e)
    _plan_check(plan, clean, e)
    one = torch.full((t, 5), 6, dtype=torch.int32)
    _plan_check(plan_of(one.cuda(), e), one, e)


# ----------------------------------------------------------------------------- routing
def _route(logits, top_k, bias=None, plan=True, **how):
    b = binding()
    t, e = logits.shape
    ids = torch.full((t, top_k), 77, dtype=torch.int32, device="cuda")
    w = torch.full((t, top_k), 77.0, device="cuda")
    p = new_plan(t, top_k, e) if plan else None
    b.aiq_route_experts(logits, ids, w, bias=bias, plan=p, **how)
    if plan:
        _plan_check(p, ids, e)
    return ids.cpu().numpy(), w.double().cpu().numpy()


def _route_check(logits, top_k, bias=None, **how):
    ids, w = _route(logits, top_k, bias, **how)
    how.setdefault("scoring", "softmax")
    want_ids, want = O.route(logits.double().cpu().numpy(), None if bias is None else bias.cpu().numpy(), top_k=top_k, **how)
    assert np.array_equal(ids, want_ids)
    assert np.array_equal(np.isnan(w), np.isnan(want))
    # exponentials of arguments up to 200 that are rounded once (their relative error: 200 units of 2^-24), sums of up to 1024 terms by 37 additions,
    # a quotient and a product
    tol = (200 + 37 + 8) * 2.0 ** -23 * np.nan_to_num(np.abs(want)) + 2.0 ** -126 * abs(how.get("scale", 1.0))
    assert (np.abs(np.nan_to_num(w) - np.nan_to_num(want)) <= tol).all()


def _logits(t, e, dtype, seed, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    return (spread * torch.randn((t, e), generator=g) + 0.5 * torch.randn((1, e), generator=g)).to(TYPES[dtype]).cuda()


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("t,e,top_k", [(1, 1, 1), (1, 32, 4), (3, 5, 5), (17, 31, 3), (64, 64, 6), (65, 33, 2), (130, 256, 8), (500, 60, 6), (40, 1024, 31),
                                       (70, 513, 9)])
def test_route(dtype, t, e, top_k):
    logits = _logits(t, e, dtype, t + e)
    bias = 0.1 * torch.randn(e, generator=torch.Generator().manual_seed(e)).cuda()
    for scoring in ("softmax", "sigmoid"):
        for b in (None, bias):
            for renormalise in (False, True):
                _route_check(logits, top_k, b, scoring=scoring, renormalise=renormalise, scale=2.5 if renormalise else 1.0)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("t,e,top_k,groups,top_groups", [(1, 8, 2, 4, 1), (33, 256, 8, 8, 4), (200, 256, 8, 8, 3), (20, 96, 7, 32, 5), (50, 60, 6, 5, 2), (70, 1024, 16, 2, 1),
                                                         (9, 24, 3, 3, 3), (30, 32, 3, 32, 9)])
def test_route_in_groups(dtype, t, e, top_k, groups, top_groups):
    logits = _logits(t, e, dtype, t + e)
    bias = 0.1 * torch.randn(e, generator=torch.Generator().manual_seed(e)).cuda()
    for scoring in ("softmax", "sigmoid"):
        for b in (None, bias):
            for best in (1, 2):
                _route_check(logits, top_k, b, scoring=scoring, groups=groups, top_groups=top_groups, group_best=best)


@pytest.mark.parametrize("groups,top_groups,best", [(1, 1, 1), (4, 2, 1), (4, 2, 2)])
@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
def test_ties_and_scores_closer_than_float32(groups, top_groups, best, scoring):
    """Equal logits with equal biases: the lower index.  Scores a few 2^-30 apart: the larger, which float32 cannot tell."""
    t, e = 300, 64
    g = torch.Generator().manual_seed(5)
    logits = torch.randint(-2, 3, (t, e), generator=g).float()
    how = dict(scoring=scoring, groups=groups, top_groups=top_groups, group_best=best)
    _route_check(logits.cuda(), 6, None, **how)
    _route_check(logits.cuda(), 6, torch.zeros(e).cuda(), **how)
    _route_check(logits.cuda(), 6, 0.25 * torch.randint(0, 2, (e,), generator=g).float().cuda(), **how)
    near = 0.5 + logits * 2.0 ** -22
    _route_check(near.cuda(), 6, None, **how)
    _route_check(near.cuda(), 6, (torch.randint(0, 4, (e,), generator=g).float() * 2.0 ** -28).cuda(), **how)


def test_masks_and_what_is_not_a_number():
    e, top_k = 40, 4
    g = torch.Generator().manual_seed(6)
    inf, nan, low = float("inf"), float("nan"), torch.finfo(torch.float32).min
    logits = torch.randn((12, e), generator=g)
    logits[1] = -inf                                   # nothing left
    logits[2, 3:] = -inf                               # fewer than top_k
    logits[3, ::2] = -inf
    logits[4] = low
    logits[5, 7:] = low
    logits[6, 9] = nan
    logits[7, 9] = inf
    logits[8, :] = -inf
    logits[8, 11] = nan
    logits[9] = -150.0 - 20 * torch.rand(e, generator=g)      # logistic functions that vanish
    logits[10] = 150.0
    logits[11, 5] = 3e38
    bias = 0.1 * torch.randn(e, generator=g)
    masked = bias.clone()
    masked[[1, 5, 9, 30]] = -inf
    broken = bias.clone()
    broken[2] = nan
    for scoring in ("softmax", "sigmoid"):
        for b in (None, bias, masked, torch.full((e,), -inf), broken):
            for renormalise in (True, False):
                for groups, top_groups, best in ((1, 1, 1), (4, 2, 1), (4, 2, 2)):
                    _route_check(logits.cuda(), top_k, None if b is None else b.cuda(), scoring=scoring, renormalise=renormalise, groups=groups,
                                 top_groups=top_groups, group_best=best)


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_route_strides_and_without_a_plan(dtype):
    wide = _logits(90, 77, dtype, 8)
    for a, b in ((0, 60), (1, 61), (7, 77)):
        _route_check(wide[:, a:b], 5)
        ids, w = _route(wide[:, a:b], 5, plan=False)
        same, sw = _route(wide[:, a:b].contiguous(), 5)
        assert np.array_equal(ids, same) and np.array_equal(w, sw)
    _route_check(wide[:1].expand(80, 77), 5)


# ------------------------------------------------------------------------------ products
def _experts(e, n, k, seed):
    codes, scales = held(weights(e * n, k, seed))
    return codes.view(e, n, -1), scales.view(e, n, -1)


def _experts_check(t, top_k, e, n, k, dtype, act, gated, in_order, bias, padded=0, ids=None):
    dt = TYPES[dtype]
    outputs = n // 2 if gated else n
    codes, scales = _experts(e, n, k, n + k)
    ids = some_ids(t, top_k, e, t + e, padded) if ids is None else ids
    plan = plan_of(ids, e)
    offsets, slots, _ = O.plan(ids.cpu().numpy(), e)
    x = activations(t * top_k if in_order else t, k, dt, t)
    b = torch.randn((e, n), generator=torch.Generator().manual_seed(3)).cuda() if bias else None
    y = torch.full((t * top_k, outputs), 7.0, dtype=dt, device="cuda")
    linear_experts(codes, scales, b, x, plan, top_k, y, activation=act, gated=gated, x_sorted=in_order)
    assert (y[offsets[-1]:] == 7.0).all()
    x64 = x.double().cpu().numpy()
    for i in range(e):
        rows = np.arange(offsets[i], offsets[i + 1])
        if len(rows):
            tail_check(y[offsets[i]:offsets[i + 1]], x64[rows if in_order else slots[rows] // top_k], values(codes[i], scales[i], k),
                       None if b is None else b[i].double().cpu().numpy(), dt, dtype, act, gated, what=f"expert {i}")


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("i,t,top_k,e,n,k", [(0, 1, 1, 1, 2, 1), (1, 1, 4, 32, 384, 320), (2, 1, 2, 4, 130, 2100), (3, 3, 2, 5, 66, 33), (4, 16, 4, 8, 258, 700),
                                             (5, 50, 6, 60, 140, 500), (6, 40, 2, 3, 520, 1030), (7, 200, 2, 4, 300, 640), (8, 700, 4, 6, 514, 1100),
                                             (9, 300, 8, 8, 128, 512), (10, 900, 3, 3, 1290, 129)])
def test_experts(dtype, gated, i, t, top_k, e, n, k):
    _experts_check(t, top_k, e, n, k, dtype, ACTS[i % 6], gated, bool(i & 1), i % 3 != 0, padded=t // 4 if i % 4 else 0)
    _experts_check(t, top_k, e, n, k, dtype, ACTS[(i + 3) % 6], gated, not i & 1, i % 3 == 0)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("t", [5, 90, 600])
def test_uneven_experts(dtype, t):
    """Every token at one expert; one at each; none anywhere; the same expert twice."""
    e, n, k = 40, 256, 640
    one = torch.full((t, 2), -1, dtype=torch.int32, device="cuda")
    one[:, 1] = 17
    _experts_check(t, 2, e, n, k, dtype, "silu", True, False, True, ids=one)
    _experts_check(t, 2, e, n, k, dtype, "none", False, True, False, ids=torch.full_like(one, -1))
    twice = torch.full((t, 2), 3, dtype=torch.int32, device="cuda")
    _experts_check(t, 2, e, n, k, dtype, "relu", False, False, True, ids=twice)
    spread = (torch.arange(2 * t, device="cuda", dtype=torch.int32) % e).view(t, 2).contiguous()
    _experts_check(t, 2, e, n, k, dtype, "gelu", True, True, True, ids=spread)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("t", [2, 100])
def test_experts_strides(dtype, t):
    dt, e, n, k, top_k = TYPES[dtype], 6, 300, 700, 3
    codes, scales = _experts(e, n, k, 1)
    plan = plan_of(some_ids(t, top_k, e, 2), e)
    x = activations(t, k, dt, 3)
    ref = linear_experts(codes, scales, None, x, plan, top_k, torch.empty((t * top_k, n), dtype=dt, device="cuda"), activation="silu")
    for skip in (1, 8):
        wide_x = torch.full((t, k + 9), 3.0, dtype=dt, device="cuda")
        wide_x[:, skip:skip + k] = x
        wide = torch.full((t * top_k, n + 9), 7.0, dtype=dt, device="cuda")
        linear_experts(codes, scales, None, wide_x[:, skip:skip + k], plan, top_k, wide[:, skip:skip + n], activation="silu")
        assert torch.equal(wide[:, skip:skip + n], ref)
        wide[:, skip:skip + n] = 7.0
        assert (wide == 7.0).all()


@pytest.mark.parametrize("t", [3, 200])
def test_a_plan_of_other_sizes_is_not_used(t):
    """A plan for fewer tokens in a buffer that is large enough, and memory that holds none: y stays; NaN where rows are combined."""
    b, e, n, k, top_k = binding(), 6, 128, 256, 2
    codes, scales = _experts(e, n, k, 1)
    x = activations(t, k, torch.float32, 3)
    plan = new_plan(t, top_k, e)
    for _ in range(2):
        y = torch.full((t * top_k, n), 7.0, device="cuda")
        linear_experts(codes, scales, None, x, plan, top_k, y)
        assert (y == 7.0).all()
        out = torch.zeros((t, n), device="cuda")
        b.aiq_combine_experts(y, torch.ones((t, top_k), device="cuda"), plan, e, out)
        assert torch.isnan(out).all()
        plan = new_plan(t, top_k, e)
        b.aiq_plan_experts(some_ids(t - 1, top_k, e, 2), e, plan)


@pytest.mark.parametrize("t", [4, 300])
def test_experts_wait_that_runs_out(t):
    b, e, n, k, top_k = binding(), 4, 256, 2100, 2
    codes, scales = _experts(e, n, k, 1)
    plan = plan_of(some_ids(t, top_k, e, 2), e)
    x = activations(t, k, torch.bfloat16, 3)
    y = torch.zeros((t * top_k, n // 2), dtype=torch.bfloat16, device="cuda")
    b.aiq_debug_mx_expire_wait(20000)
    linear_experts(codes, scales, None, x, plan, top_k, y, activation="relu", gated=True)
    assert torch.isnan(y).all()
    linear_experts(codes, scales, None, x, plan, top_k, y, activation="relu", gated=True)
    assert torch.isfinite(y).all()


# ------------------------------------------------------------------------- weighted sums
@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("t,top_k,e,h", [(1, 1, 1, 1), (1, 4, 32, 2048), (5, 3, 7, 33), (64, 8, 16, 264), (300, 2, 5, 4100), (130, 31, 64, 96)])
def test_combine(dtype, t, top_k, e, h):
    b, dt = binding(), TYPES[dtype]
    for i, padded in enumerate((0, t // 2)):
        ids = some_ids(t, top_k, e, t, padded)
        ids[:, 0] = torch.where(torch.arange(t, device="cuda") % 3 == 1, -1, ids[:, 0])
        plan = plan_of(ids, e)
        positions = O.plan(ids.cpu().numpy(), e)[2]
        g = torch.Generator().manual_seed(h)
        z = torch.randn((t * top_k, h + 8), generator=g).to(dt).cuda()[:, 8 * i:h + 8 * i]
        w = torch.rand((t, top_k), generator=g).cuda()
        residual = torch.randn((t, h), generator=g).to(dt).cuda() if i or t > 5 else None
        wide = torch.full((t, h + 8), 7.0, dtype=dt, device="cuda")
        y = wide[:, i:h + i]
        b.aiq_combine_experts(z, w, plan, e, y, residual=residual)
        z64, w64 = z.double().cpu().numpy(), w.double().cpu().numpy()
        ref, size = np.zeros((t, h)), np.zeros((t, h))
        if residual is not None:
            ref += residual.double().cpu().numpy()
            size += np.abs(ref)
        for j in range(top_k):
            live = positions[:, j] >= 0
            part = w64[live, j, None] * z64[positions[live, j]]
            ref[live] += part
            size[live] += np.abs(part)
        # a fused multiply-add per expert, each off by half a unit of a sum that is at most `size`; rounded once
        tol = (top_k + 1) * 2.0 ** -24 * size * (1 + 2.0 ** -10) + torch.finfo(dt).eps / 2 * (np.abs(ref) + size * 2.0 ** -18) + 2.0 ** -24 * torch.finfo(dt).smallest_normal
        assert (np.abs(y.double().cpu().numpy() - ref) <= tol + torch.finfo(dt).smallest_normal * torch.finfo(dt).eps).all()
        kept = wide.clone()
        kept[:, i:h + i] = 7.0
        assert (kept == 7.0).all()
        if residual is not None:
            same = residual.clone()
            b.aiq_combine_experts(z, w, plan, e, same, residual=same)
            assert torch.equal(same, y)


def test_combine_shows_weights_that_are_no_numbers():
    b = binding()
    ids = torch.tensor([[0, 1], [-1, -1], [1, -1]], dtype=torch.int32, device="cuda")
    w = torch.tensor([[1.0, 2.0], [float("nan"), float("nan")], [0.5, 0.0]], device="cuda")
    y = torch.empty((3, 40), device="cuda")
    z = torch.ones((6, 40), device="cuda")
    z[3:] = float("nan")                               # rows that no pair has
    b.aiq_combine_experts(z, w, plan_of(ids, 2), 2, y)
    assert (y[0] == 3.0).all() and torch.isnan(y[1]).all() and (y[2] == 0.5).all()


# ------------------------------------------------------------------------ all of a layer
def _layer(logits, x, up, down, plan, ids, w, hidden, z, y, ws):
    b = binding()
    e, top_k = logits.shape[1], ids.shape[1]
    b.aiq_route_experts(logits, ids, w, scoring="sigmoid", plan=plan)
    b.aiq_mx_linear_experts(*up, None, x, plan, top_k, hidden, "silu", gated=True, workspace=ws)
    b.aiq_mx_linear_experts(*down, None, hidden, plan, top_k, z, x_sorted=True, workspace=ws)
    b.aiq_combine_experts(z, w, plan, e, y, residual=x)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("t,top_k,e,d,f", [(1, 4, 32, 512, 384), (20, 3, 8, 320, 200), (300, 4, 16, 640, 320)])
def test_a_layer_and_its_graph(dtype, t, top_k, e, d, f):
    """Router, experts up and down, weighted sum: against the oracle on the stored values between the steps, then captured and replayed with
    other inputs."""
    b, dt = binding(), TYPES[dtype]
    up, down = _experts(e, 2 * f, d, 1), _experts(e, d, f, 2)
    ids, w = torch.empty((t, top_k), dtype=torch.int32, device="cuda"), torch.empty((t, top_k), device="cuda")
    plan = new_plan(t, top_k, e)
    hidden, z, y = (torch.empty(s, dtype=dt, device="cuda") for s in ((t * top_k, f), (t * top_k, d), (t, d)))
    ws = torch.empty(max(b.aiq_mx_linear_experts_workspace_bytes(e, n, k, t * top_k, dt) for n, k in ((2 * f, d), (d, f))), dtype=torch.uint8, device="cuda")
    logits, x = _logits(t, e, dtype, 4), activations(t, d, dt, 5)
    args = (logits, x, up, down, plan, ids, w, hidden, z, y, ws)
    _layer(*args)
    want_ids, want_w = O.route(logits.double().cpu().numpy(), None, "sigmoid", top_k)
    assert np.array_equal(ids.cpu().numpy(), want_ids)
    offsets, slots, positions = O.plan(want_ids, e)
    x64, h64, z64 = (v.double().cpu().numpy() for v in (x, hidden, z))
    ref = x64.copy()
    for i in range(e):
        a, c = offsets[i], offsets[i + 1]
        if a < c:
            tail_check(hidden[a:c], x64[slots[a:c] // top_k], values(up[0][i], up[1][i], d), None, dt, dtype, "silu", True)
            tail_check(z[a:c], h64[a:c], values(down[0][i], down[1][i], f), None, dt, dtype, "none", False)
    for j in range(top_k):
        ref += want_w[:, j, None] * z64[positions[:, j]]
    assert np.abs(y.double().cpu().numpy() - ref).max() <= (torch.finfo(dt).eps + 2.0 ** -20) * np.abs(ref).max()

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _layer(*args)
    for seed in (11, 12):
        logits.copy_(_logits(t, e, dtype, seed))
        x.copy_(activations(t, d, dt, seed))
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        _layer(*args)
        assert torch.equal(y, got)


def test_a_plan_of_many_token_blocks():
    """More pairs than the usual number of token blocks may have: against a stable sort."""
    t, top_k, e = 330_001, 31, 33
    g = torch.Generator(device="cuda").manual_seed(1)
    ids = (torch.rand((t, top_k), generator=g, device="cuda") ** 2 * (e + 1)).int() - 1
    offsets, slots, positions = binding().aiq_expert_plan_parts(plan_of(ids, e), t, top_k, e)
    flat = ids.reshape(-1).long()
    order = torch.sort(torch.where(flat < 0, e, flat), stable=True).indices
    rows = int((flat >= 0).sum())
    assert int(offsets[-1]) == rows
    assert torch.equal(offsets.long(), torch.cat((torch.zeros(1, dtype=torch.int64, device="cuda"), torch.bincount(flat[flat >= 0], minlength=e).cumsum(0))))
    assert torch.equal(slots[:rows].long(), order[:rows]) and (slots[rows:] == -1).all()
    back = torch.full_like(flat, -1)
    back[order[:rows]] = torch.arange(rows, device="cuda")
    assert torch.equal(positions.reshape(-1).long(), back)


@pytest.mark.parametrize("t", [3, 40, 300])
def test_two_streams_at_once(t):
    """Two layers on two streams, with plans and workspaces of their own, many times over."""
    b, dt, e, n, k, top_k = binding(), torch.bfloat16, 6, 1024, 2100, 2
    codes, scales = _experts(e, n, k, 1)
    sides = [torch.cuda.Stream() for _ in range(2)]
    xs = [activations(t, k, dt, 3 + i) for i in range(2)]
    ids = [some_ids(t, top_k, e, 5 + i) for i in range(2)]
    plans = [plan_of(i, e) for i in ids]
    size = b.aiq_mx_linear_experts_workspace_bytes(e, n, k, t * top_k, dt)
    ws = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(2)]
    want = [linear_experts(codes, scales, None, xs[i], plans[i], top_k, torch.empty((t * top_k, n), dtype=dt, device="cuda"), activation="silu") for i in range(2)]
    ys = [[torch.zeros((t * top_k, n), dtype=dt, device="cuda") for _ in range(10)] for _ in range(2)]
    torch.cuda.synchronize()
    for j in range(10):
        for i in range(2):
            b.aiq_mx_linear_experts(codes, scales, None, xs[i], plans[i], top_k, ys[i][j], "silu", workspace=ws[i], stream=sides[i])
    torch.cuda.synchronize()
    for i in range(2):
        for y in ys[i]:
            assert torch.equal(y, want[i])
