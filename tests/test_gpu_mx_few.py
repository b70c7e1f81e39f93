"""Up to four rows through the layer and the experts in one launch (x as three-bit digits), and calls that follow one another without a pause."""
import numpy as np
import pytest
import torch

from experts_util import ACTS, linear_act, linear_experts, new_plan, plan_of, tail_check
from gpu_util import binding
from mx_util import TYPES, activations, held, values, weights
from oracle import experts_oracle as O

pytestmark = pytest.mark.gpu

# clusters of 1, 2, 4 and 8, ends of K inside a chunk, a block and a digit row of all kinds, channels that do not fill a tile
SHAPES = [(8400, 1030, 2), (33000, 520, 1), (4200, 2100, 2), (4202, 8200, 1), (2600, 2200, 3), (2100, 2100, 4), (1100, 8192, 2), (514, 33000, 1), (130, 65000, 3),
          (66, 70001, 4), (17000, 1985, 1), (20000, 1700, 1)]


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_few_rows(dtype, i):
    (n, k, m), dt = SHAPES[i], TYPES[dtype]
    codes, scales = held(weights(n, k, n))
    x = activations(m, k, dt, k)
    w, x64 = values(codes, scales, k), x.double().cpu().numpy()
    bias = torch.randn(n, generator=torch.Generator().manual_seed(3)).cuda()
    for gated in (False, True):
        outputs = n // 2 if gated else n
        residual = torch.randn((m, outputs), generator=torch.Generator().manual_seed(4)).to(dt).cuda() if i % 2 == gated else None
        y = torch.full((m, outputs + 3), 7.0, dtype=dt, device="cuda")
        act = ACTS[(i + 3 * gated) % 6]
        linear_act(codes, scales, bias, x, y[:, 1:1 + outputs], activation=act, gated=gated, residual=residual)
        tail_check(y[:, 1:1 + outputs], x64, w, bias.double().cpu().numpy(), dt, dtype, act, gated,
                   None if residual is None else residual.double().cpu().numpy())
        assert (y[:, 0] == 7.0).all() and (y[:, 1 + outputs:] == 7.0).all()


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_digits_of_every_size(dtype):
    """A row times the unit matrix shows what the digits hold: blocks with one value far above the rest, powers of two and what lies next to them, both signs,
    subnormal numbers, zeros."""
    dt, k = TYPES[dtype], 4224
    g = torch.Generator().manual_seed(1)
    x = torch.randn((2, k), generator=g)
    x[:, 512:1024] *= torch.exp2(-torch.randint(0, 20, (2, 512), generator=g).float())
    x[:, 1024:1536] = torch.exp2(torch.randint(-14, 15, (2, 512), generator=g).float()) * torch.tensor([1.0, -1.0]).repeat(256)
    x[:, 1536:2048] = torch.exp2(torch.randint(-14, 15, (2, 512), generator=g).float()) * (2 - torch.finfo(dt).eps)
    x[:, 2048:2560:32] = 60000.0
    x[:, 2560:3000] = 0
    x[:, 3000:3200] = torch.finfo(dt).smallest_normal * torch.rand((2, 200), generator=g)
    x[:, 3200:3232] = -torch.finfo(dt).max
    x = x.to(dt).cuda()
    eye = torch.zeros((k, k), device="cuda")
    eye[torch.arange(k), torch.arange(k)] = 1.0
    codes, scales = held(eye)
    y = linear_act(codes, scales, None, x, torch.empty((2, k), dtype=torch.float32 if dtype == "f32" else dt, device="cuda"))
    d = x.double().cpu()
    top = d.abs().view(2, -1, 32).amax(dim=2).repeat_interleave(32, dim=1)
    digits = {"bf16": 8, "f16": 10, "f32": 13}[dtype]
    # half a unit of the last digit, which is 2^-(3 (digits - 1)) of the power of two below the largest value, but not below 4 * 2^-127: the scale byte of the last digit
    # is 0 there, and sums are multiplied by 4, so half of it is 2^-126; the sum of the digits' sums in float32 (one rounding each); the result's rounding
    tol = top * 2.0 ** (1 - 3 * (digits - 1) - 1) + 2.0 ** -126 + digits * 2.0 ** -24 * d.abs() + torch.finfo(dt).eps / 2 * d.abs() + torch.finfo(dt).smallest_normal * torch.finfo(dt).eps
    assert ((y.double().cpu() - d).abs() <= tol).all()


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("m", [1, 2])
def test_blocks_that_are_no_numbers(dtype, m):
    dt, n, k = TYPES[dtype], 4200, 8200
    codes, scales = held(weights(n, k, 5))
    x = activations(m, k, dt, 6)
    x[m - 1, 4000] = float("inf")
    y = linear_act(codes, scales, None, x, torch.zeros((m, n), dtype=dt, device="cuda"), activation="silu")
    assert torch.isnan(y[m - 1]).all() and torch.isfinite(y[:m - 1]).all()
    scales = scales.clone()
    scales[77, 3] = 255
    y = linear_act(codes, scales, None, activations(m, k, dt, 6), torch.zeros((m, n), dtype=dt, device="cuda"), activation="relu")
    bad = torch.zeros((m, n), dtype=torch.bool)
    bad[:, 77] = True
    assert torch.equal(torch.isnan(y).cpu(), bad)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("t,top_k,e", [(1, 4, 4), (1, 31, 64), (2, 2, 3), (3, 5, 6), (4, 8, 9), (4, 31, 40)])
@pytest.mark.parametrize("in_order", [False, True])
def test_tokens_with_the_same_expert_more_than_once(dtype, t, top_k, e, in_order):
    """More rows than tokens at an expert; more than a block of rows."""
    dt, n, k = TYPES[dtype], 258, 1100
    codes, scales = held(weights(e * n, k, 1))
    codes, scales = codes.view(e, n, -1), scales.view(e, n, -1)
    for ids in (torch.full((t, top_k), e - 1), torch.arange(t * top_k).view(t, top_k) % 2, torch.arange(t * top_k).view(t, top_k) % (e + 1) - 1):
        ids = ids.int().cuda().contiguous()
        plan = plan_of(ids, e)
        offsets, slots, _ = O.plan(ids.cpu().numpy(), e)
        x = activations(t * top_k if in_order else t, k, dt, 2)
        y = torch.full((t * top_k, n // 2), 7.0, dtype=dt, device="cuda")
        linear_experts(codes, scales, None, x, plan, top_k, y, activation="silu", gated=True, x_sorted=in_order)
        assert (y[offsets[-1]:] == 7.0).all()
        x64 = x.double().cpu().numpy()
        for i in range(e):
            rows = np.arange(offsets[i], offsets[i + 1])
            if len(rows):
                tail_check(y[offsets[i]:offsets[i + 1]], x64[rows if in_order else slots[rows] // top_k], values(codes[i], scales[i], k), None, dt, dtype,
                           "silu", True)


@pytest.mark.parametrize("m", [1, 3, 40])
def test_a_wait_that_runs_out(m):
    b, n, k = binding(), 4200, 8200
    codes, scales = held(weights(n, k, 5))
    x = activations(m, k, torch.bfloat16, 6)
    y = torch.zeros((m, n // 2), dtype=torch.bfloat16, device="cuda")
    b.aiq_debug_mx_expire_wait(20000)
    linear_act(codes, scales, None, x, y, activation="relu", gated=True)
    assert torch.isnan(y).all()
    linear_act(codes, scales, None, x, y, activation="relu", gated=True)
    assert torch.isfinite(y).all()


@pytest.mark.parametrize("m", [1, 2, 40])
def test_weights_written_just_before(m):
    """Weights, rows and residual that the kernel before the call writes, over and over, and the result read by the one behind it."""
    b, dt, n, k = binding(), torch.bfloat16, 4200, 8200
    versions = [(held(weights(n, k, i)), activations(m, k, dt, i)) for i in range(3)]
    codes, scales = torch.empty_like(versions[0][0][0]), torch.empty_like(versions[0][0][1])
    x = torch.empty_like(versions[0][1])
    ws = torch.empty(max(16, b.aiq_mx_linear_workspace_bytes(n, k, m, dt)), dtype=torch.uint8, device="cuda")
    want = [linear_act(c, s, None, v, torch.empty((m, n), dtype=dt, device="cuda"), activation="silu") for (c, s), v in versions]
    got = [torch.empty((m, n), dtype=dt, device="cuda") for _ in range(30)]
    y = torch.empty((m, n), dtype=dt, device="cuda")
    torch.cuda.synchronize()
    for i, out in enumerate(got):
        (c, s), v = versions[i % 3]
        x.copy_(v)
        scales.copy_(s)
        codes.copy_(c)
        b.aiq_mx_linear_act(codes, scales, None, x, y, "silu", workspace=ws)
        out.copy_(y)
        y.zero_()
    for i, out in enumerate(got):
        assert torch.equal(out, want[i % 3])


@pytest.mark.parametrize("t", [1, 3, 20, 200])
def test_layers_one_after_the_other(t):
    """A layer's output is the next one's input: 24 layers without a pause give what they give one at a time."""
    b, dt, e, top_k, d, f = binding(), torch.bfloat16, 8, 3, 512, 320
    up, down = held(weights(e * 2 * f, d, 1) * 2), held(weights(e * d, f, 2) * 2)
    up, down = [v.view(e, 2 * f, -1) for v in up], [v.view(e, d, -1) for v in down]
    gate = (torch.randn((d, e), generator=torch.Generator().manual_seed(3)) * 0.05).cuda().to(dt)
    ids, w = torch.empty((t, top_k), dtype=torch.int32, device="cuda"), torch.empty((t, top_k), device="cuda")
    plan = new_plan(t, top_k, e)
    hidden, z = torch.empty((t * top_k, f), dtype=dt, device="cuda"), torch.empty((t * top_k, d), dtype=dt, device="cuda")
    ws = torch.empty(max(b.aiq_mx_linear_experts_workspace_bytes(e, n, k, t * top_k, dt) for n, k in ((2 * f, d), (d, f))), dtype=torch.uint8, device="cuda")

    def go(pause):
        x = activations(t, d, dt, 7)
        for _ in range(24):
            steps = [lambda: b.aiq_route_experts(x @ gate, ids, w, plan=plan),
                     lambda: b.aiq_mx_linear_experts(*up, None, x, plan, top_k, hidden, "silu", gated=True, workspace=ws),
                     lambda: b.aiq_mx_linear_experts(*down, None, hidden, plan, top_k, z, x_sorted=True, workspace=ws),
                     lambda: b.aiq_combine_experts(z, w, plan, e, x, residual=x)]
            for step in steps:
                step()
                if pause:
                    torch.cuda.synchronize()
            x = x / x.float().pow(2).mean(dim=1, keepdim=True).sqrt().to(dt)
        torch.cuda.synchronize()
        return x

    want = go(True)
    assert torch.isfinite(want).all()
    for _ in range(3):
        assert torch.equal(go(False), want)
