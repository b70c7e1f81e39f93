"""Microscaled 4-bit operators on the GPU against the float64 oracle."""
import numpy as np
import pytest
import torch

from gpu_util import binding
from mx_util import PIECES, TYPES, activations, check, held, linear, values, weights
from oracle import mx_oracle as X

pytestmark = pytest.mark.gpu


def _special(rows, k, dtype):
    """Rows that meet every rule of the quantizer: halfway cases, zeros, subnormal numbers, the largest, NaN, infinities."""
    g = torch.Generator().manual_seed(rows * 1000 + k)
    x = torch.randn((rows, k), generator=g) * torch.exp(3 * torch.randn((rows, 1), generator=g))
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, -0.25, -0.75, -2.5, -5.0, 7.0, 7.5, 0.0, -0.0])
    x = x.to(dtype)
    big = torch.finfo(dtype).max
    for r in range(rows):
        if r % 4 == 1:
            x[r] = ties.repeat(k // 16 + 1)[:k].to(dtype)
        if r % 4 == 2:
            x[r, ::3] = 0
            x[r, : min(k, 40)] = torch.finfo(dtype).smallest_normal / 4
        if r % 8 == 3:
            x[r, -1] = big
        if r % 8 == 7:
            x[r, k // 2] = [float("nan"), float("inf"), -float("inf")][r % 3]
    return x


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("rows,k,pad,skip", [(1, 1, 0, 0), (9, 31, 0, 0), (8, 32, 0, 0), (17, 33, 3, 1), (16, 127, 0, 0), (24, 128, 8, 0),
                                             (24, 129, 7, 5), (9, 511, 1, 1), (16, 512, 0, 0), (11, 513, 0, 0), (40, 1280, 0, 0),
                                             (7, 1283, 5, 5), (8, 2056, 8, 8)])
def test_quantize(dtype, rows, k, pad, skip):
    dt = TYPES[dtype]
    wide = torch.zeros((rows, k + pad), dtype=dt)
    wide[:, skip:skip + k] = _special(rows, k, dt)
    x = wide.cuda()[:, skip:skip + k]
    codes, scales = held(x)
    ref_codes, ref_scales = X.quantize(x.cpu().double().numpy())
    assert np.array_equal(scales.cpu().numpy(), ref_scales)
    assert np.array_equal(codes.cpu().numpy(), ref_codes)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("rows,k,pad", [(1, 1, 0), (9, 31, 0), (8, 32, 8), (17, 33, 3), (24, 129, 7), (16, 512, 0), (11, 513, 0), (40, 1281, 0),
                                        (8, 2056, 8)])
def test_dequantize(dtype, rows, k, pad):
    b, dt = binding(), TYPES[dtype]
    codes, scales = held(_special(rows, k, torch.float32).cuda())
    if rows > 1:
        scales[0, 0] = 254
        scales[1, 0] = 0
    wide = torch.full((rows, k + pad), 7.0, dtype=dt, device="cuda")
    b.aiq_mx_dequantize(codes, scales, wide[:, :k])
    with np.errstate(over="ignore"):
        ref = torch.from_numpy(values(codes, scales, k).astype(np.float32)).to(dt)
    got = wide.cpu()
    assert torch.equal(torch.isnan(got[:, :k]), torch.isnan(ref))
    assert torch.equal(torch.nan_to_num(got[:, :k]), torch.nan_to_num(ref))
    assert (got[:, k:] == 7.0).all()


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("rows,k,step", [(3, 700, 1), (5, 1031, 0), (2, 8, 1), (9, 25, 2), (300, 4000, 3)])
def test_rows_that_start_anywhere(dtype, rows, k, step):
    """Every offset of a row's start from a 16- or 32-byte boundary, reading and writing; nothing beside the rows is touched."""
    b, dt = binding(), TYPES[dtype]
    g = torch.Generator().manual_seed(k)
    for skip in range(9):
        wide = (torch.randn((rows, k + skip + step), generator=g) * 3).to(dt).cuda()
        x = wide[:, skip:skip + k]
        codes, scales = held(x)
        ref_codes, ref_scales = X.quantize(x[:3].cpu().double().numpy())
        assert np.array_equal(codes[:3].cpu().numpy(), ref_codes) and np.array_equal(scales[:3].cpu().numpy(), ref_scales)
        plain_codes, plain_scales = held(x.contiguous())
        assert torch.equal(codes, plain_codes) and torch.equal(scales, plain_scales)
        out = torch.full_like(wide, 7.0)
        b.aiq_mx_dequantize(codes, scales, out[:, skip:skip + k])
        ref = torch.from_numpy(values(codes, scales, k).astype(np.float32)).to(dt)
        assert torch.equal(out[:, skip:skip + k].cpu(), ref)
        out[:, skip:skip + k] = 7.0
        assert (out == 7.0).all()


def test_every_code_and_scale():
    """All 256 bytes of codes under all 256 scale bytes."""
    b = binding()
    codes = torch.arange(256, dtype=torch.uint8).repeat(256, 1).cuda()            # 512 values a row
    scales = torch.arange(256, dtype=torch.uint8).repeat(16, 1).t().contiguous().cuda()
    y = torch.empty((256, 512), device="cuda")
    b.aiq_mx_dequantize(codes, scales, y)
    with np.errstate(over="ignore"):
        ref = torch.from_numpy(values(codes, scales, 512).astype(np.float32))
    assert torch.equal(torch.nan_to_num(y.cpu()), torch.nan_to_num(ref)) and torch.equal(torch.isnan(y.cpu()), torch.isnan(ref))


SHAPES = [(1, 1, 1), (3, 33, 2), (8, 32, 1), (10, 64, 1), (129, 100, 5), (64, 320, 9), (200, 609, 17), (128, 512, 33), (1280, 320, 1),
          (1000, 1281, 4), (257, 2500, 130), (512, 1024, 300), (384, 4097, 64), (130, 8192, 3),
          # beyond the kernel for few rows: split K ranges, rows of x beside and above each other, odd ends everywhere
          (129, 4100, 17), (200, 6000, 33), (1001, 1300, 20), (5671, 609, 37), (130, 9000, 70), (1000, 3001, 48), (64, 20000, 9), (3, 70000, 40),
          (260, 3100, 129), (700, 640, 257), (128, 512, 600),
          # long K ranges per block, more tiles than SMs
          (9500, 2176, 5), (9500, 2176, 16), (19000, 1100, 7), (1290, 650, 3500), (2500, 520, 2200), (1152, 1030, 4700)]


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("n,k,m", SHAPES)
@pytest.mark.parametrize("workspace", [True, False])
def test_linear(dtype, n, k, m, workspace):
    dt = TYPES[dtype]
    codes, scales = held(weights(n, k, n + k))
    x = activations(m, k, dt, m + k)
    bias = torch.randn(n, generator=torch.Generator().manual_seed(3)).cuda() if (n + m) % 2 else None
    y = linear(codes, scales, bias, x, torch.full((m, n), float("nan"), dtype=dt, device="cuda"), workspace)
    check(y, x.double().cpu().numpy(), values(codes, scales, k), bias.cpu().numpy() if bias is not None else None, dt, dtype)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("n,k,m", SHAPES)
def test_matmul(dtype, n, k, m):
    b, dt = binding(), TYPES[dtype]
    bc, bs = held(weights(n, k, n + k))
    ac, as_ = held(activations(m, k, torch.float32, m + k))
    bias = torch.randn(n, generator=torch.Generator().manual_seed(3)).cuda() if (n + m) % 2 else None
    y = torch.full((m, n), float("nan"), dtype=dt, device="cuda")
    b.aiq_mx_matmul(ac, as_, bc, bs, bias, k, y)
    check(y, values(ac, as_, k), values(bc, bs, k), bias.cpu().numpy() if bias is not None else None, dt, "mx")


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("m", [1, 3, 20, 150])
def test_strides_and_what_lies_around(dtype, m):
    """x a slice of wider rows, or one row repeated; y a slice whose surroundings stay as they were."""
    dt, n, k = TYPES[dtype], 300, 700
    codes, scales = held(weights(n, k, 5))
    w = values(codes, scales, k)
    for skip, pad in ((0, 0), (1, 4), (8, 8), (3, 13)):
        x = activations(m, skip + k + pad, dt, 7)[:, skip:skip + k]
        wide = torch.full((m + 2, n + 9), 7.0, dtype=dt, device="cuda")
        linear(codes, scales, None, x, wide[1:m + 1, 4:4 + n])
        check(wide[1:m + 1, 4:4 + n], x.double().cpu().numpy(), w, None, dt, dtype, f"skip {skip}")
        wide[1:m + 1, 4:4 + n] = 7.0
        assert (wide == 7.0).all()
    x = activations(1, k, dt, 8).expand(m, k)
    y = linear(codes, scales, None, x, torch.empty((m, n), dtype=dt, device="cuda"))
    check(y, x.double().cpu().numpy(), w, None, dt, dtype, "repeated row")


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("m", [1, 40, 120])
def test_values_of_every_size(dtype, m):
    """Blocks of x and of W whose sizes lie far apart, all-zero blocks and rows, weights near both ends of the scales."""
    dt, n, k = TYPES[dtype], 160, 640
    w = weights(n, k, 11).cpu()
    w[0] = 0
    w[1] *= 2.0 ** -110
    w[2] *= 2.0 ** 100
    w[3, 32:64] *= 2.0 ** 30
    w[4, ::2] = 0
    x = activations(m, k, torch.float32, 12).cpu()
    x[:, 64:96] *= 2.0 ** -12
    x[:, 96:128] *= 2.0 ** 8
    x[:, 128:160] = 0
    x[0, 200:300] = 0
    x = x.to(dt).cuda()
    codes, scales = held(w.cuda())
    y = linear(codes, scales, None, x, torch.empty((m, n), dtype=dt, device="cuda"))
    wv = values(codes, scales, k)
    rows = [i for i in range(n) if dtype != "f16" or i not in (2, 3)]        # these two leave the range of halves
    check(y[:, rows], x.double().cpu().numpy(), wv[rows], None, dt, dtype)
    if dtype == "f16":
        assert torch.isinf(y[:, 2]).all()
    assert (y[:, 0] == 0).all()


@pytest.mark.parametrize("m", [1, 24, 250])
def test_nan_scales_and_nonfinite_activations_stay_in_their_rows(m):
    dt, n, k = torch.float32, 140, 300
    w = weights(n, k, 21)
    w[5, 40] = float("nan")
    codes, scales = held(w)
    x = activations(m, k, dt, 22)
    if m > 3:
        x[2, 17] = float("nan")
        x[3, 299] = float("inf")
    y = linear(codes, scales, None, x, torch.empty((m, n), dtype=dt, device="cuda"))
    assert torch.isnan(y[:, 5]).all()
    keep = [i for i in range(m) if m <= 3 or i not in (2, 3)]
    cols = [i for i in range(n) if i != 5]
    if m > 3:
        assert torch.isnan(y[2]).all() and not torch.isfinite(y[3]).any()
    check(y[keep][:, cols], x[keep].double().cpu().numpy(), values(codes, scales, k)[cols], None, dt, "f32")


def test_quantize_activations_then_multiply():
    """The operators in a run: weights quantized once, each batch quantized, multiplied, compared with the product of what the
    codes stand for and with the layer that quantizes its weights alone."""
    b = binding()
    n, k, m = 512, 1000, 50
    w, x = weights(n, k, 31), activations(m, k, torch.bfloat16, 32)
    wc, ws = held(w)
    xc, xs = held(x)
    wv = torch.empty((n, k), device="cuda")
    xv = torch.empty((m, k), dtype=torch.bfloat16, device="cuda")
    b.aiq_mx_dequantize(wc, ws, wv)
    b.aiq_mx_dequantize(xc, xs, xv)
    y = torch.empty((m, n), device="cuda")
    b.aiq_mx_matmul(xc, xs, wc, ws, None, k, y)
    check(y, xv.double().cpu().numpy(), wv.double().cpu().numpy(), None, torch.float32, "mx")
    z = linear(wc, ws, None, xv.float(), torch.empty((m, n), device="cuda"))
    check(z, xv.double().cpu().numpy(), wv.double().cpu().numpy(), None, torch.float32, "f32")


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_captured_calls_on_two_streams(dtype):
    """Two graphs on two streams, each with its own workspace, replayed with new inputs in place; bit-equal to eager calls."""
    b, dt, n, k, m = binding(), TYPES[dtype], 1100, 1500, 70
    codes, scales = held(weights(n, k, 41))
    size = b.aiq_mx_linear_workspace_bytes(n, k, m, dt)
    assert size > 0
    runs = []
    for i in range(2):
        x = activations(m, k, dt, 42 + i)
        s = torch.cuda.Stream()
        ws = torch.empty(size, dtype=torch.uint8, device="cuda")
        xc, xs = held(x)
        y, z = torch.empty((m, n), dtype=dt, device="cuda"), torch.empty((m, n), dtype=dt, device="cuda")
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            b.aiq_mx_quantize(x, xc, xs)
            b.aiq_mx_matmul(xc, xs, codes, scales, None, k, z)
            b.aiq_mx_linear(codes, scales, None, x, y, workspace=ws)
        runs.append((g, s, x, ws, xc, xs, y, z))
    for rep in range(3):
        new = [activations(m, k, dt, 50 + 2 * rep + i) for i in range(2)]
        for (g, s, x, *_), v in zip(runs, new):
            x.copy_(v)
        torch.cuda.synchronize()
        for g, s, *_ in runs:
            with torch.cuda.stream(s):
                g.replay()
                g.replay()
        torch.cuda.synchronize()
        for (g, s, x, ws, xc, xs, y, z), v in zip(runs, new):
            ey = linear(codes, scales, None, v, torch.empty_like(y))
            vc, vs = held(v)
            ez = torch.empty_like(z)
            b.aiq_mx_matmul(vc, vs, codes, scales, None, k, ez)
            assert torch.equal(y, ey) and torch.equal(z, ez)


@pytest.mark.parametrize("m", [1, 24, 250])
def test_nan_blocks_of_either_matrix(m):
    """aiq_mx_matmul: a NaN block makes its row or column NaN and nothing else."""
    b, n, k = binding(), 140, 1300
    w, x = weights(n, k, 61), activations(m, k, torch.float32, 62)
    w[7, 1299] = float("inf")
    if m > 1:
        x[m - 1, 33] = float("nan")
    bc, bs = held(w)
    ac, as_ = held(x)
    y = torch.empty((m, n), device="cuda")
    b.aiq_mx_matmul(ac, as_, bc, bs, None, k, y)
    assert torch.isnan(y[:, 7]).all() and (m == 1 or torch.isnan(y[m - 1]).all())
    rows, cols = [i for i in range(m) if m == 1 or i != m - 1], [i for i in range(n) if i != 7]
    check(y[rows][:, cols], values(ac, as_, k)[rows], values(bc, bs, k)[cols], None, torch.float32, "mx")


def test_two_calls_are_bit_equal():
    """The same call twice, and among others on the same workspace."""
    for n, k, m, dt in ((1000, 5000, 40, torch.float32), (4096, 2048, 20, torch.bfloat16), (300, 700, 3, torch.float16)):
        codes, scales = held(weights(n, k, 71))
        x = activations(m, k, dt, 72)
        first = linear(codes, scales, None, x, torch.empty((m, n), dtype=dt, device="cuda"))
        linear(codes, scales, None, activations(m, k, dt, 73), torch.empty((m, n), dtype=dt, device="cuda"))
        assert torch.equal(first, linear(codes, scales, None, x, torch.empty((m, n), dtype=dt, device="cuda")))


def test_scale_bytes_at_both_ends():
    """Stored weights whose scales the quantizer seldom or never writes: 2^-127, 2^126 and 2^127."""
    b, n, k, m = binding(), 256, 2048, 40
    codes, scales = held(weights(n, k, 81))
    scales[0] = 0
    scales[1] = 254
    scales[2] = 253
    scales[3, ::2] = 0
    scales[:, 64:] = 0                                       # behind the last block
    x = activations(m, k, torch.float32, 82)
    x[0] *= 2.0 ** -100
    y = linear(codes, scales, None, x, torch.empty((m, n), device="cuda"))
    w = values(codes, scales, k)
    keep = [i for i in range(n) if i not in (1, 2)]
    check(y[:, keep], x.double().cpu().numpy(), w[keep], None, torch.float32, "f32")
    check(y[:1], x[:1].double().cpu().numpy(), w, None, torch.float32, "f32")


def test_refusals_on_the_device():
    b = binding()
    codes, scales = held(weights(256, 2000, 1))
    x, y = activations(64, 2000, torch.bfloat16, 2), torch.empty((64, 256), dtype=torch.bfloat16, device="cuda")
    bad = [dict(x=x.float()), dict(x=x[:, :1800]), dict(x=x.t()), dict(x=x[:32]), dict(y=y[:, :255]), dict(y=y.t()), dict(y=y.expand(1, 64, 256)),
           dict(x=x.cpu()), dict(codes=codes[:255]), dict(codes=codes[:, :512]), dict(scales=scales.cpu()), dict(x=x.double()),
           dict(bias=torch.zeros(255, device="cuda")), dict(bias=torch.zeros(256, dtype=torch.float16, device="cuda"))]
    for change in bad:
        a = dict(codes=codes, scales=scales, bias=None, x=x, y=y) | change
        with pytest.raises(ValueError):
            b.aiq_mx_linear(a["codes"], a["scales"], a["bias"], a["x"], a["y"])
    with pytest.raises(b.AiqError) as e:
        b.aiq_mx_linear(codes, scales, None, x, y, workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    assert e.value.status == b.ERR_WORKSPACE_TOO_SMALL
    with pytest.raises(b.AiqError):                          # rows of y on top of each other
        b.aiq_mx_linear(codes, scales, None, x, y[:1].expand(64, 256))


# One row of x against more than 2^20 weights: a kernel of its own, which multiplies integers.  Its x is held closer than the pieces that
# the bound counts (2^-23 of a block's largest for bfloat16, 2^-31 for half, against 2^-22 and 2^-27).  Additions: one within a block, 5
# in a warp, at most 15 over warps and K / 16384 over rounds, fewer than the bound's K / 32 + 64.  A block's planes are joined from
# sums of up to 2^25 units of at most 2^-22 of its largest |x|, rounded to 24 bits: one unit of 2^-22 2^-6 at bfloat16, far less at half.
ONE_ROW = [(1100, 1000), (4099, 257), (9000, 120), (70, 16500), (33, 33000), (1031, 2049), (40000, 32), (131073, 8), (1025, 1024), (4097, 4096),
           (8200, 4100)]


def _one_row(kind, codes, scales, bias, x, k, workspace=True):
    n = codes.shape[0]
    if kind == "mx":
        y = torch.full((1, n), float("nan"), device="cuda")
        binding().aiq_mx_matmul(*x, codes, scales, bias, k, y)
        return y
    return linear(codes, scales, bias, x, torch.full((1, n), float("nan"), dtype=TYPES[kind], device="cuda"), workspace)


@pytest.mark.parametrize("kind", ["bf16", "f16", "mx"])
@pytest.mark.parametrize("n,k", ONE_ROW)
def test_one_row(kind, n, k):
    dt = TYPES.get(kind, torch.float32)
    codes, scales = held(weights(n, k, n + k))
    w = values(codes, scales, k)
    bias = torch.randn(n, generator=torch.Generator().manual_seed(3)).cuda() if n % 2 else None
    for skip in (0, 1) if kind != "mx" else (0,):
        x = activations(1, k + skip, dt, k)[:, skip:]
        given = held(x) if kind == "mx" else x
        xv = values(*given, k) if kind == "mx" else x.double().cpu().numpy()
        for workspace in (True, False) if n * k > 2 ** 25 else (True,):
            y = _one_row(kind, codes, scales, bias, given, k, workspace)
            check(y, xv, w, bias.cpu().numpy() if bias is not None else None, dt, kind, f"skip {skip} workspace {workspace}")
            assert torch.equal(y, _one_row(kind, codes, scales, bias, given, k, workspace))


@pytest.mark.parametrize("kind", ["bf16", "f16", "mx"])
def test_one_row_of_every_size(kind):
    """Blocks of x from the type's subnormal values to 2^100, weights' scales that bring them back, zeros, negative and mixed signs."""
    dt, n, k = TYPES.get(kind, torch.float32), 2050, 640
    w = weights(n, k, 91).cpu()
    w[3, 40:80] = 0
    codes, scales = held(w.cuda())
    x = activations(1, k, torch.float32, 92).cpu()
    x[0, 64:96] = 0
    x[0, 96:128] = -x[0, 96:128].abs()
    x[0, 128:160] *= torch.logspace(-8, 0, 32)                     # far below the block's largest
    if kind == "f16":
        x[0, :32] *= 2.0 ** -16
        x[0, 32:64] = 60000.0
        scales[:, 0] = 140
        scales[:, 1] = 100
    else:
        x[0, :32] *= 2.0 ** -122
        x[0, 32:64] *= 2.0 ** 100
        x[0, 160:192] = torch.arange(1, 33) * 2.0 ** -133
        scales[:, 0] = 245
        scales[:, 1] = 10
        scales[:, 5] = 254
    x = x.to(dt).cuda()
    given = held(x) if kind == "mx" else x
    xv = values(*given, k) if kind == "mx" else x.double().cpu().numpy()
    check(_one_row(kind, codes, scales, None, given, k), xv, values(codes, scales, k), None, dt, kind)


@pytest.mark.parametrize("kind", ["bf16", "f16", "mx"])
def test_one_row_with_nan_and_infinity(kind):
    dt, n, k = TYPES.get(kind, torch.float32), 1030, 1100
    w = weights(n, k, 93)
    w[5, 1099] = float("nan")
    w[1029, 0] = float("inf")
    codes, scales = held(w)
    for what in (None, float("nan"), float("inf"), -float("inf")):
        x = activations(1, k, dt, 94)
        if what is not None:
            x[0, 1070] = what
        given = held(x) if kind == "mx" else x
        y = _one_row(kind, codes, scales, None, given, k)
        if what is not None:
            assert torch.isnan(y).all()
            continue
        assert torch.isnan(y[0, [5, 1029]]).all()
        keep = [i for i in range(n) if i not in (5, 1029)]
        xv = values(*given, k) if kind == "mx" else x.double().cpu().numpy()
        check(y[:, keep], xv, values(codes, scales, k)[keep], None, dt, kind)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_one_row_captured_and_what_lies_around(kind):
    """A captured call reads the x of its replay; elements of y's buffer beside the row stay as they were."""
    dt, n, k = TYPES[kind], 2051, 520
    codes, scales = held(weights(n, k, 95))
    w = values(codes, scales, k)
    x, wide = activations(1, k, dt, 96), torch.full((1, n + 7), 7.0, dtype=dt, device="cuda")
    y = wide[:, 3:3 + n]
    linear(codes, scales, None, x, y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        linear(codes, scales, None, x, y)
    for seed in (97, 98):
        x.copy_(activations(1, k, dt, seed))
        graph.replay()
        torch.cuda.synchronize()
        check(y, x.double().cpu().numpy(), w, None, dt, kind)
        assert (wide[:, :3] == 7.0).all() and (wide[:, 3 + n:] == 7.0).all()
