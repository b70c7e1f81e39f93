"""What the calls of the layer's way out and of the experts refuse, and the layout of a plan (no GPU needed: nothing is launched)."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def aiq():
    from paper_2512_14090_b200 import build
    build.build()
    from paper_2512_14090_b200 import binding
    return binding


ONE = 4096                                             # an address that is aligned to everything and never used


def _call(aiq, name, **change):
    """The call with arguments that are in order, save for `change`."""
    args = {
        "aiq_mx_linear_act": dict(codes=ONE, scales=ONE, bias=None, N=8, K=32, x=ONE, dtype=1, M=4, x_stride=32, activation=3, gated=1, residual=None,
                                  r_stride=0, y=ONE, y_stride=8, workspace=None, workspace_bytes=0, stream=None),
        "aiq_plan_experts": dict(ids=ONE, T=4, top_k=2, E=8, plan=ONE, plan_bytes=1 << 20, stream=None),
        "aiq_route_experts": dict(logits=ONE, dtype=0, T=4, E=8, stride=8, bias=None, scoring=0, top_k=2, groups=2, top_groups=1, group_best=2,
                                  renormalise=1, scale=1.0, ids=ONE, weights=ONE, plan=None, plan_bytes=0, stream=None),
        "aiq_mx_linear_experts": dict(codes=ONE, scales=ONE, bias=None, E=8, N=8, K=32, x=ONE, dtype=1, x_stride=32, x_sorted=0, plan=ONE,
                                      plan_bytes=1 << 20, T=4, top_k=2, activation=3, gated=1, y=ONE, y_stride=8, workspace=ONE,
                                      workspace_bytes=1 << 20, stream=None),
        "aiq_combine_experts": dict(z=ONE, dtype=1, T=4, top_k=2, E=8, H=32, z_stride=32, weights=ONE, plan=ONE, plan_bytes=1 << 20, residual=None,
                                    r_stride=0, y=ONE, y_stride=32, stream=None),
    }[name]
    assert set(change) <= set(args)
    return getattr(aiq._mxcall, name)(*{**args, **change}.values()), getattr(aiq.lib, name)(*{**args, **change}.values())


def _skip_on_gpu():
    import torch
    if torch.cuda.is_available():
        pytest.skip("would launch with made-up addresses")


@pytest.mark.parametrize("name", ["aiq_mx_linear_act", "aiq_plan_experts", "aiq_route_experts", "aiq_mx_linear_experts", "aiq_combine_experts"])
def test_the_calls_that_the_others_differ_from_are_in_order(aiq, name):
    _skip_on_gpu()
    assert set(_call(aiq, name)) <= {aiq.ERR_CUDA, aiq.ERR_NOT_SM100}, aiq.last_error()


@pytest.mark.parametrize("name,change", [
    ("aiq_mx_linear_act", dict(activation=6)), ("aiq_mx_linear_act", dict(activation=-1)), ("aiq_mx_linear_act", dict(gated=2)),
    ("aiq_mx_linear_act", dict(N=9)), ("aiq_mx_linear_act", dict(y_stride=3)), ("aiq_mx_linear_act", dict(gated=0, y_stride=7)),
    ("aiq_mx_linear_act", dict(residual=ONE, r_stride=-1)), ("aiq_mx_linear_act", dict(residual=ONE + 1)), ("aiq_mx_linear_act", dict(codes=ONE + 16)),
    ("aiq_mx_linear_act", dict(scales=ONE + 8)), ("aiq_mx_linear_act", dict(bias=ONE + 2)), ("aiq_mx_linear_act", dict(x=None)),
    ("aiq_mx_linear_act", dict(M=0)), ("aiq_mx_linear_act", dict(dtype=3)), ("aiq_mx_linear_act", dict(workspace=ONE + 8, workspace_bytes=1 << 20)),
    ("aiq_mx_linear_act", dict(K=2 ** 32 + 32)),
    ("aiq_plan_experts", dict(ids=None)), ("aiq_plan_experts", dict(plan=None)), ("aiq_plan_experts", dict(plan=ONE + 4)), ("aiq_plan_experts", dict(T=0)),
    ("aiq_plan_experts", dict(top_k=0)), ("aiq_plan_experts", dict(top_k=9)), ("aiq_plan_experts", dict(top_k=32, E=64)), ("aiq_plan_experts", dict(E=1025)),
    ("aiq_plan_experts", dict(T=2 ** 30, top_k=2)), ("aiq_plan_experts", dict(ids=ONE + 2)),
    ("aiq_route_experts", dict(logits=None)), ("aiq_route_experts", dict(ids=None)), ("aiq_route_experts", dict(weights=None)),
    ("aiq_route_experts", dict(scoring=2)), ("aiq_route_experts", dict(groups=0)), ("aiq_route_experts", dict(groups=3)),
    ("aiq_route_experts", dict(top_groups=0)), ("aiq_route_experts", dict(top_groups=3)), ("aiq_route_experts", dict(group_best=3)),
    ("aiq_route_experts", dict(E=64, stride=64, groups=64)), ("aiq_route_experts", dict(top_k=5)), ("aiq_route_experts", dict(renormalise=2)),
    ("aiq_route_experts", dict(scale=float("nan"))), ("aiq_route_experts", dict(scale=float("inf"))), ("aiq_route_experts", dict(stride=-8)),
    ("aiq_route_experts", dict(bias=ONE + 1)), ("aiq_route_experts", dict(plan=ONE + 8, plan_bytes=1 << 20)), ("aiq_route_experts", dict(dtype=-1)),
    ("aiq_mx_linear_experts", dict(codes=None)), ("aiq_mx_linear_experts", dict(plan=None)), ("aiq_mx_linear_experts", dict(workspace=None)),
    ("aiq_mx_linear_experts", dict(x_sorted=2)), ("aiq_mx_linear_experts", dict(N=7)), ("aiq_mx_linear_experts", dict(activation=9)),
    ("aiq_mx_linear_experts", dict(y_stride=3)), ("aiq_mx_linear_experts", dict(x_stride=-1)), ("aiq_mx_linear_experts", dict(codes=ONE + 16)),
    ("aiq_mx_linear_experts", dict(scales=ONE + 8)), ("aiq_mx_linear_experts", dict(workspace=ONE + 8)), ("aiq_mx_linear_experts", dict(K=0)),
    ("aiq_mx_linear_experts", dict(y=ONE + 1)), ("aiq_mx_linear_experts", dict(T=-1)),
    ("aiq_combine_experts", dict(z=None)), ("aiq_combine_experts", dict(weights=None)), ("aiq_combine_experts", dict(plan=None)),
    ("aiq_combine_experts", dict(H=0)), ("aiq_combine_experts", dict(y_stride=31)), ("aiq_combine_experts", dict(weights=ONE + 2)),
    ("aiq_combine_experts", dict(residual=ONE + 1)), ("aiq_combine_experts", dict(E=0)), ("aiq_combine_experts", dict(dtype=7))])
def test_refusals(aiq, name, change):
    assert _call(aiq, name, **change) == (aiq.ERR_INVALID_ARG, aiq.ERR_INVALID_ARG), aiq.last_error()
    assert name in aiq.last_error()


@pytest.mark.parametrize("name", ["aiq_plan_experts", "aiq_mx_linear_experts", "aiq_combine_experts"])
def test_a_plan_or_workspace_that_is_too_small(aiq, name):
    small = aiq.aiq_expert_plan_bytes(4, 2, 8) - 4
    assert _call(aiq, name, plan_bytes=small) == (aiq.ERR_WORKSPACE_TOO_SMALL,) * 2
    assert _call(aiq, "aiq_route_experts", plan=ONE, plan_bytes=small) == (aiq.ERR_WORKSPACE_TOO_SMALL,) * 2
    size = aiq.aiq_mx_linear_experts_workspace_bytes(8, 8, 32, 8, aiq.DTYPE_F16)
    assert _call(aiq, "aiq_mx_linear_experts", workspace_bytes=size - 1) == (aiq.ERR_WORKSPACE_TOO_SMALL,) * 2


@pytest.mark.parametrize("t,top_k,e", [(1, 1, 1), (5, 3, 7), (64, 8, 256), (65, 8, 256), (1000, 31, 1024), (100000, 2, 64)])
def test_the_parts_of_a_plan(aiq, t, top_k, e):
    """In order, on 16 bytes, apart, inside the plan."""
    at = [C.c_size_t() for _ in range(3)]
    assert aiq.lib.aiq_expert_plan_parts(t, top_k, e, *[C.byref(a) for a in at]) == aiq.OK
    at = [a.value for a in at]
    assert all(a % 16 == 0 for a in at)
    ends = [at[0] + 4 * (e + 1), at[1] + 4 * t * top_k, at[2] + 4 * t * top_k]
    assert 16 <= at[0] and ends[0] <= at[1] and ends[1] <= at[2] and ends[2] <= aiq.aiq_expert_plan_bytes(t, top_k, e)


def test_sizes_of_nothing(aiq):
    assert aiq.aiq_expert_plan_bytes(0, 1, 1) == 0 and aiq.aiq_expert_plan_bytes(4, 9, 8) == 0 and aiq.aiq_expert_plan_bytes(4, 1, 1025) == 0
    assert aiq.aiq_mx_linear_experts_workspace_bytes(8, 8, 0, 8, aiq.DTYPE_F16) == 0
    assert aiq.aiq_mx_linear_experts_workspace_bytes(8, 8, 32, 2 ** 40, aiq.DTYPE_F16) == 0


def test_the_number_of_arguments(aiq):
    if aiq._mxcall is aiq.lib:
        pytest.skip("no call module")
    for name in ("aiq_mx_linear_act", "aiq_plan_experts", "aiq_route_experts", "aiq_mx_linear_experts", "aiq_combine_experts"):
        with pytest.raises(TypeError, match=name):
            getattr(aiq._mxcall, name)(1, 2, 3)
    with pytest.raises(TypeError):
        _call(aiq, "aiq_route_experts", scale="1")
