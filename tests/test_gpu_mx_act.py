"""The microscaled linear layer with activation, gate and residual on the GPU against the float64 oracle."""
import numpy as np
import pytest
import torch

from experts_util import ACTS, linear_act, tail_check
from gpu_util import binding
from mx_util import TYPES, activations, held, linear, values, weights

pytestmark = pytest.mark.gpu

# every kernel: few rows, one row in integers, tensor cores with split K, pieces beside and above each other, more tiles than SMs, half tiles
SHAPES = [(2, 1, 1), (6, 33, 2), (8, 32, 1), (130, 100, 5), (64, 320, 9), (1280, 320, 1), (1000, 1281, 4), (2048, 1024, 1), (2050, 520, 1), (258, 2500, 130),
          (384, 4097, 64), (130, 8192, 3), (5672, 609, 37), (1002, 1300, 20), (64, 20000, 9), (9500, 2176, 5), (9500, 520, 16), (1290, 650, 3500),
          (2500, 520, 2200), (260, 3100, 129)]


def _inputs(n, k, m, dt, outputs):
    codes, scales = held(weights(n, k, n + k))
    x = activations(m, k, dt, m + k)
    bias = torch.randn(n, generator=torch.Generator().manual_seed(3)).cuda()
    residual = torch.randn((m, outputs), generator=torch.Generator().manual_seed(4)).to(dt).cuda()
    return codes, scales, x, bias, residual


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_linear_act(dtype, gated, i):
    (n, k, m), dt = SHAPES[i], TYPES[dtype]
    outputs = n // 2 if gated else n
    codes, scales, x, bias, residual = _inputs(n, k, m, dt, outputs)
    act = ACTS[(i + gated) % len(ACTS)]
    bias = bias if i % 3 else None
    residual = residual if i % 2 else None
    for workspace in (True, False):
        y = torch.full((m, outputs), float("nan"), dtype=dt, device="cuda")
        linear_act(codes, scales, bias, x, y, workspace, activation=act, gated=gated, residual=residual)
        tail_check(y, x.double().cpu().numpy(), values(codes, scales, k), bias.double().cpu().numpy() if bias is not None else None, dt, dtype, act, gated,
                   residual.double().cpu().numpy() if residual is not None else None, f"workspace {workspace}")


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("n,k,m", [(300, 96, 3), (1536, 800, 1), (640, 1100, 40), (640, 1100, 400)])
def test_every_activation(dtype, act, n, k, m):
    dt = TYPES[dtype]
    for gated in (False, True):
        outputs = n // 2 if gated else n
        codes, scales, x, bias, residual = _inputs(n, k, m, dt, outputs)
        bias = bias * 4
        y = linear_act(codes, scales, bias, x, torch.full((m, outputs), float("nan"), dtype=dt, device="cuda"), activation=act, gated=gated)
        tail_check(y, x.double().cpu().numpy(), values(codes, scales, k), bias.double().cpu().numpy(), dt, dtype, act, gated)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("n,k,m", [(300, 700, 3), (1600, 800, 1), (513, 2100, 20), (1290, 650, 300)])
def test_nothing_on_the_way_out_is_the_plain_layer(dtype, n, k, m):
    dt = TYPES[dtype]
    codes, scales, x, bias, _ = _inputs(n, k, m, dt, n)
    for workspace in (True, False):
        a = linear(codes, scales, bias, x, torch.empty((m, n), dtype=dt, device="cuda"), workspace)
        b = linear_act(codes, scales, bias, x, torch.empty((m, n), dtype=dt, device="cuda"), workspace)
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("m", [1, 3, 20, 150])
@pytest.mark.parametrize("skip", [0, 1, 4])
def test_strides_and_what_lies_around(dtype, gated, m, skip):
    """x, y and residual slices of wider rows; a residual row for all; the residual in y itself."""
    dt, n, k = TYPES[dtype], 330, 1100
    outputs = n // 2 if gated else n
    codes, scales, x, bias, residual = _inputs(n, k, m, dt, outputs)
    ref = linear_act(codes, scales, bias, x, torch.empty((m, outputs), dtype=dt, device="cuda"), activation="silu", gated=gated, residual=residual)
    wide_x = torch.full((m, k + 9), 3.0, dtype=dt, device="cuda")
    wide_x[:, skip:skip + k] = x
    wide_r = torch.full((m, outputs + 6), 5.0, dtype=dt, device="cuda")
    wide_r[:, 1:1 + outputs] = residual
    wide = torch.full((m, outputs + 11), 7.0, dtype=dt, device="cuda")
    linear_act(codes, scales, bias, wide_x[:, skip:skip + k], wide[:, skip:skip + outputs], activation="silu", gated=gated, residual=wide_r[:, 1:1 + outputs])
    assert torch.equal(wide[:, skip:skip + outputs], ref)
    wide[:, skip:skip + outputs] = 7.0
    assert (wide == 7.0).all()
    y = residual.clone()
    linear_act(codes, scales, bias, x, y, activation="silu", gated=gated, residual=y)
    assert torch.equal(y, ref)
    one = residual[:1].expand(m, outputs)
    a = linear_act(codes, scales, bias, x, torch.empty((m, outputs), dtype=dt, device="cuda"), activation="relu", gated=gated, residual=one)
    b = linear_act(codes, scales, bias, x, torch.empty((m, outputs), dtype=dt, device="cuda"), activation="relu", gated=gated, residual=one.contiguous())
    assert torch.equal(a, b)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("m", [1, 2, 40])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_nan_stays_one(act, m, dtype):
    """In x: its row; in the residual: its value; in a scale byte: its channel.  Not rounded away by an activation."""
    dt, n, k = TYPES[dtype], 640, 2100
    for gated in (False, True):
        outputs = n // 2 if gated else n
        codes, scales, x, bias, residual = _inputs(n, k, m, dt, outputs)
        x, residual, scales = x.clone(), residual.clone(), scales.clone()
        residual[-1, 7] = float("nan")
        scales[n - 3, 1] = 255
        if m > 1:
            x[0, 5] = float("nan")
        y = linear_act(codes, scales, bias, x, torch.zeros((m, outputs), dtype=dt, device="cuda"), activation=act, gated=gated, residual=residual)
        bad = torch.zeros((m, outputs), dtype=torch.bool)
        bad[-1, 7] = True
        bad[:, (n - 3) % outputs] = True
        if m > 1:
            bad[0] = True
        assert torch.equal(torch.isnan(y).cpu(), bad)


@pytest.mark.parametrize("act", ACTS)
def test_large_values(act):
    """Sums of every size through the activations, infinities of a bias among them."""
    n = 512
    codes, scales = held(torch.zeros((n, 64), device="cuda"))
    v = torch.cat((torch.logspace(-30, 38, n // 4), -torch.logspace(-30, 38, n // 4), torch.linspace(-20, 20, n // 2 - 1), torch.tensor([float("inf")])))
    x = torch.ones((2, 64), device="cuda")
    y = linear_act(codes, scales, v.cuda(), x, torch.empty((2, n), device="cuda"), activation=act)
    from experts_util import act_bound
    from oracle import experts_oracle as E
    d = v.double().numpy()
    ref = E.activate(d, act)
    got = y[1].double().cpu().numpy()
    assert got[-1] == ref[-1] == (6.0 if act == "relu6" else np.inf)
    tol = act_bound(d[:-1], 0.0, act) + 2.0 ** -24 * np.abs(ref[:-1]) + 2.0 ** -149
    assert (np.abs(got[:-1] - ref[:-1]) <= tol).all()


@pytest.mark.parametrize("m", [2, 40, 300])
def test_streams_and_graphs(m):
    """On a stream of its own and captured, with inputs that change between replays."""
    b, dt, n, k = binding(), torch.bfloat16, 1280, 2100
    codes, scales, x, bias, residual = _inputs(n, k, m, dt, n // 2)
    how = dict(activation="silu", gated=True, residual=residual)
    ref = linear_act(codes, scales, bias, x, torch.empty((m, n // 2), dtype=dt, device="cuda"), **how)
    x2 = (x * 0.5).clone()
    ref2 = linear_act(codes, scales, bias, x2, torch.empty((m, n // 2), dtype=dt, device="cuda"), **how)
    ws = torch.empty(max(16, b.aiq_mx_linear_workspace_bytes(n, k, m, dt)), dtype=torch.uint8, device="cuda")
    xs, y = x.clone(), torch.empty((m, n // 2), dtype=dt, device="cuda")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    b.aiq_mx_linear_act(codes, scales, bias, xs, y, workspace=ws, stream=side, **how)
    side.synchronize()
    assert torch.equal(y, ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.aiq_mx_linear_act(codes, scales, bias, xs, y, workspace=ws, **how)
    for source, want in ((x2, ref2), (x, ref), (x2, ref2)):
        xs.copy_(source)
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)


def test_a_wait_that_runs_out():
    b, dt, n, k, m = binding(), torch.bfloat16, 640, 2100, 40
    codes, scales, x, bias, residual = _inputs(n, k, m, dt, n // 2)
    for rows in (40, 300):
        x = activations(rows, k, dt, 1)
        y = torch.zeros((rows, n // 2), dtype=dt, device="cuda")
        b.aiq_debug_mx_expire_wait(20000)
        linear_act(codes, scales, bias, x, y, activation="relu", gated=True)
        assert torch.isnan(y).all()
        linear_act(codes, scales, bias, x, y, activation="relu", gated=True)
        assert torch.isfinite(y).all()
