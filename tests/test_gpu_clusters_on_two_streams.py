"""Kernels whose clusters hold tensor memory, on two streams at once: the linear layer of many rows and the few-row kernel, both of little shared
memory.  Results are those of the calls by themselves."""
import pytest
import torch

from gpu_util import binding
from mx_util import activations, held, weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [4, 8, 16])
def test_linear_layer_beside_few_rows(bits):
    b = binding()
    n, k, m = 7600, 520, 100                              # pairs of CTAs that cut K in two
    w, x = weights(n, k, 1), activations(m, k, torch.float32, 2)
    packed = torch.empty((n, b.aiq_packed_row_bytes(k, bits)), dtype=torch.uint8, device="cuda")
    scales = torch.empty(n, device="cuda")
    b.aiq_quantize_layer(w, bits, packed, scales)
    ws = torch.empty(b.aiq_qlinear_workspace_bytes(n, k, bits, m), dtype=torch.uint8, device="cuda")
    few_n, few_k, few_m = 8400, 1100, 2                   # pairs, too
    codes, few_scales = held(weights(few_n, few_k, 3))
    few_x = activations(few_m, few_k, torch.bfloat16, 4)
    few_ws = torch.empty(b.aiq_mx_linear_workspace_bytes(few_n, few_k, few_m, torch.bfloat16), dtype=torch.uint8, device="cuda")
    assert few_ws.numel() > 0

    def linear(y, stream=None):
        b.aiq_qlinear(packed, scales, None, n, k, bits, x, y, workspace=ws, stream=stream)

    def few(y, stream=None):
        b.aiq_mx_linear_act(codes, few_scales, None, few_x, y, "silu", workspace=few_ws, stream=stream)

    want, few_want = torch.empty((m, n), device="cuda"), torch.empty((few_m, few_n), dtype=torch.bfloat16, device="cuda")
    linear(want)
    few(few_want)
    ys = [torch.zeros_like(want) for _ in range(20)]
    few_ys = [torch.zeros_like(few_want) for _ in range(40)]
    sides = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for i, y in enumerate(ys):
        linear(y, sides[0])
        few(few_ys[2 * i], sides[1])
        few(few_ys[2 * i + 1], sides[1])
    torch.cuda.synchronize()
    assert all(torch.equal(y, want) for y in ys) and all(torch.equal(y, few_want) for y in few_ys)
