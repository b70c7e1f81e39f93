"""Microscaled products at the limits of the format and of their precision, on the GPU against float64."""
import numpy as np
import pytest
import torch

from gpu_util import binding
from mx_util import TYPES, activations, check, held, linear, values, weights

pytestmark = pytest.mark.gpu


# Scale bytes 253 and 254 make 6 * 2^127 of an element, which is no float32.  The stored value is finite all the same, and so is its
# product with a small x.
@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("n,k,m", [(64, 96, 1), (64, 100, 3), (70, 130, 9), (1100, 1000, 1), (4400, 1000, 1), (700, 2000, 40)])
@pytest.mark.parametrize("workspace", [True, False])
def test_linear_with_scale_bytes_at_both_ends(dtype, n, k, m, workspace):
    dt = TYPES[dtype]
    codes, scales = held(weights(n, k, 1))
    for row, byte in ((1, 254), (2, 253), (3, 252), (4, 0), (5, 1)):
        scales[row, 0] = byte
    x = activations(m, k, torch.float32, 2)
    x[:, :32] = 0 if dtype == "f16" else x[:, :32] * 2.0 ** -115       # a half times 2^126 is out of a half's range
    x[:, 4:9] = 0
    x = x.to(dt)
    y = linear(codes, scales, None, x, torch.full((m, n), float("nan"), dtype=dt, device="cuda"), workspace)
    check(y, x.double().cpu().numpy(), values(codes, scales, k), None, dt, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,k,m", [(64, 96, 1), (64, 100, 3), (70, 130, 9), (700, 2000, 40)])
def test_matmul_with_scale_bytes_at_both_ends(dtype, n, k, m):
    """Blocks near the top of either matrix against blocks near the bottom of the other, and against zeros."""
    b, dt = binding(), TYPES[dtype]
    ac, as_ = held(activations(m, k, torch.float32, 3))
    bc, bs = held(weights(n, k, 4))
    as_[:, 0], as_[:, 1] = 10, 254
    bs[:, 0], bs[:, 1] = 118, 5
    bs[1, 0], bs[2, 0] = 254, 253
    as_[m - 1, 1] = 253
    ac[:, 32:48] = 0                                                   # block 2 of A is zeros, of B at the top
    bs[3, 2] = 254
    y = torch.full((m, n), float("nan"), dtype=dt, device="cuda")
    b.aiq_mx_matmul(ac, as_, bc, bs, None, k, y)
    check(y, values(ac, as_, k), values(bc, bs, k), None, dt, "mx")


def _rows_of(codes, scales, k):
    """float64 values of stored rows, on the GPU."""
    return torch.from_numpy(values(codes, scales, k)).cuda()


# One row: every product is exact, whatever else is in its block.  Additions: a block's 32 products become one float32 (one rounding, 2^-24 of
# the block's sum), what the block's integers cannot hold is added value by value (32 at most, 32 roundings of a sum of small values, and one for
# adding it), then 5 in a warp, at most 15 over warps, K / 16384 over rounds and one for the bias.  The kernel for few rows: K / 512 / 2 in a lane's
# chain of pairs, 1 + 5 + 8 behind it.  64 + K / 512 roundings of 2^-24 of sum |x w| cover both, and half a step of the output type.
def _check_exact_products(y, x, w, what):
    x, w = x.double(), w.double()
    ref, s = x @ w.t(), x.abs() @ w.abs().t()
    err = (64 + x.shape[1] / 512) * 2.0 ** -24 * s
    f = torch.finfo(y.dtype)
    tol = err + f.eps / 2 * (ref.abs() + err) + f.smallest_normal * f.eps
    worst = ((y.double() - ref).abs() / tol).max().item()
    assert worst <= 1.0, f"{what}: error is {worst:.3g} of what is allowed"


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n,k", [(1100, 1000), (4200, 1000), (8192, 1024), (35000, 130), (300, 16500), (110, 40000)])
@pytest.mark.parametrize("log2", [0, 10, 14, 20, 40])
def test_one_row_with_values_far_apart_in_a_block(dtype, n, k, log2):
    """One value of every block far above the others, and channels whose codes there are zero: what is left are products with the others."""
    if dtype == "f16" and log2 > 20:
        log2 = 28                                                      # half: from 2^-18 to 2^10
    dt = TYPES[dtype]
    codes, scales = held(weights(n, k, 5))
    c = codes.clone()
    g = torch.Generator().manual_seed(log2)
    down = log2 // 2 + 4 if dtype == "f16" else 0                      # halves: around the middle of their range
    x = torch.randn((1, k), generator=g)
    at = torch.arange(7, k, 32)
    c[: n // 2, (at // 2).cuda()] &= 0x0F                              # element 7 of a block is in a high nibble
    x *= 2.0 ** -down
    x[0, at] = torch.randn(len(at), generator=g).sign() * 2.0 ** (log2 - down) * 1.5
    x[0, 3::32] *= 2.0 ** -6
    x = x.to(dt).cuda()
    assert torch.isfinite(x).all()
    w = _rows_of(c, scales, k)
    y = linear(c, scales, None, x, torch.full((1, n), float("nan"), dtype=dt, device="cuda"), workspace=False)
    _check_exact_products(y, x, w, f"2^{log2}")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_one_row_with_one_weight_per_channel(dtype):
    """Each channel has one element other than zero, a power of two: y is that value of x times it, to the last bit."""
    dt, n, k = TYPES[dtype], 8192, 1024
    g = torch.Generator().manual_seed(3)
    at = torch.randperm(k, generator=g).repeat(8)[:n]
    e = torch.randint(0, 3, (n,), generator=g)                         # elements 1, 2, 4: codes 2, 4, 6
    sign = torch.randint(0, 2, (n,), generator=g)
    codes = torch.zeros((n, k), dtype=torch.uint8)
    codes[torch.arange(n), at] = (2 * (e + 1) + 8 * sign).to(torch.uint8)
    codes = (codes[:, 0::2] | (codes[:, 1::2] << 4)).contiguous().cuda()
    scales = torch.full((n, 32), 125, dtype=torch.uint8, device="cuda")
    x = torch.randn((1, k), generator=g) * torch.exp2(torch.randint(-12, 13, (1, k), generator=g).float())
    if dtype == "bf16":
        x *= torch.exp2(torch.randint(-30, 31, (1, k), generator=g).float())
    x = x.to(dt)
    want = (x[0, at].double() * 2.0 ** (e.double() - 2) * (1 - 2 * sign)).to(dt)
    y = linear(codes, scales, None, x.cuda(), torch.full((1, n), float("nan"), dtype=dt, device="cuda"))
    assert torch.equal(y[0].cpu(), want)


TABLE = [0, .5, 1, 1.5, 2, 3, 4, 6]


def _positive(n, k, seed):
    """Random codes without a sign, rows of k, and scale bytes around 2^-15, made on the GPU."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    codes = torch.randint(0, 256, (n, -(-k // 128) * 64), dtype=torch.uint8, device="cuda", generator=g) & 0x77
    at = 2 * torch.arange(codes.shape[1], device="cuda")
    codes &= ((at < k).to(torch.uint8) * 0x0F) | ((at + 1 < k).to(torch.uint8) * 0xF0)
    scales = torch.randint(111, 114, (n, -(-k // 512) * 16), dtype=torch.uint8, device="cuda", generator=g)
    scales[:, -(-k // 32):] = 0
    return codes, scales


def _positive_sums(x, codes, scales, k):
    """float64 x w^T for x [M][k] or (codes, scales), w as codes and scales without signs."""
    table = torch.tensor(TABLE, dtype=torch.float64, device="cuda")

    def part(c, s, a, b):
        v = table[torch.stack((c[:, a // 2:b // 2] & 15, c[:, a // 2:b // 2] >> 4), 2).view(c.shape[0], -1).int()]
        return v * torch.exp2(s[:, a // 32:-(-b // 32)].double() - 127).repeat_interleave(32, 1)[:, :v.shape[1]]
    total = 0
    for a in range(0, k, 32768):
        b = min(a + 32768, -(-k // 32) * 32)
        xs = part(*x, a, b) if isinstance(x, tuple) else torch.nn.functional.pad(x[:, a:b].double(), (0, b - min(b, k)))
        total = total + xs @ part(codes, scales, a, b).t()
    return total


# Nothing cancels in sums of positive products, so what the additions drop adds up.  Up to 512 k at a time stay in the accumulator: 16 MMAs per
# piece of x (8 with both microscaled), each of which drops less than 2^-23 of the sum so far; what leaves it is added in float32, K / 512
# roundings of 2^-24 and 8 for splits and bias.  The mean error of R rounded results is below that plus 6 standard deviations of their own
# rounding, which is at most eps / 2 either way: eps / 2 / sqrt(3 R).  (Halves below 2^-14 lie 2^-24 apart, the smallest normal number times eps:
# half of that is what their rounding may take, whatever their size.  "matmul" with halves sums up to about 2^-19, "matmul up" to 2^-12.)
@pytest.mark.parametrize("dtype,kind,n,k,m", [("f16", "linear", 2048, 131072, 520), ("f16", "linear", 256, 100001, 33), ("f16", "linear", 300, 40000, 130),
                                              ("f16", "matmul", 2048, 200000, 520), ("f16", "matmul up", 2048, 200000, 520),
                                              ("bf16", "linear", 1024, 300000, 300),
                                              ("bf16", "linear", 130, 270000, 70), ("bf16", "matmul", 130, 1050000, 40),
                                              ("f32", "linear", 10240, 20000, 40), ("f32", "matmul", 10240, 20000, 40)])
def test_long_sums_of_positive_products(dtype, kind, n, k, m):
    b, dt = binding(), TYPES[dtype]
    codes, scales = _positive(n, k, 1)
    few = torch.cat((torch.arange(min(n, 64)), torch.arange(max(n - 64, 64), n))).cuda()
    y = torch.full((m, n), float("nan"), dtype=dt, device="cuda")
    if kind == "linear":
        g = torch.Generator(device="cuda").manual_seed(2)
        x = (torch.rand((m, k), device="cuda", generator=g) * 2.0 ** -6).to(dt)
        linear(codes, scales, None, x, y)
    else:
        x = _positive(m, k, 3)
        x[1][:, : k // 32].sub_(8 if kind == "matmul" else 0)
        b.aiq_mx_matmul(*x, codes, scales, None, k, y)
    ref = _positive_sums(x, codes[few], scales[few], k)
    e = (y[:, few].double() - ref) / ref
    pieces = {"f32": 5, "f16": 3, "bf16": 2}[dtype]
    chain = 16 * pieces if kind == "linear" else 8
    sums = chain * 2.0 ** -23 + (k / 512 + 8) * 2.0 ** -24
    if kind == "linear":
        sums += 2.0 ** -(12 + 5 * pieces) * 32                        # x itself: 2^-(12 + 5 pieces) of the largest, which is below 32 of a block's sum
    f = torch.finfo(dt)
    half = torch.clamp(f.smallest_normal / ref, min=1) * f.eps / 2
    assert (e.abs() <= sums + half * (1 + sums)).all(), e.abs().max()
    assert abs(e.mean().item()) <= sums + 6 * half.max().item() / (3 * e.numel()) ** 0.5


GUARD = 4096


@pytest.mark.parametrize("start", [0x00, 0xFF])
def test_one_workspace_for_every_shape_and_type(start):
    """Calls of several shapes and types in turn on one workspace, filled with 0xFF (as a scale byte: NaN) or zeros before the first and never
    again: each gives what it gives on a fresh one, and nothing behind the bytes it asks for changes."""
    b = binding()
    calls = [("f32", 700, 640, 257), ("bf16", 129, 4100, 17), ("f16", 5671, 609, 37), ("bf16", 512, 1025, 300), ("f32", 200, 6000, 33), ("f16", 260, 3100, 129),
             ("f32", 1001, 1300, 20), ("bf16", 9500, 2176, 5), ("f16", 300, 40000, 60), ("f32", 8192, 4096, 1), ("bf16", 700, 1500, 2048)]
    made = []
    for kind, n, k, m in calls:
        codes, scales = held(weights(n, k, n + k))
        x = activations(m, k, TYPES[kind], m + k)
        size = b.aiq_mx_linear_workspace_bytes(n, k, m, TYPES[kind])
        y = torch.full((m, n), float("nan"), dtype=TYPES[kind], device="cuda")
        if size:
            ws = torch.full((size,), 0xFF - start, dtype=torch.uint8, device="cuda")
            b.aiq_mx_linear(codes, scales, None, x, y, workspace=ws)
            check(y[:, :130], x.double().cpu().numpy(), values(codes[:130], scales[:130], k), None, TYPES[kind], kind)
            made.append((kind, codes, scales, x, y, size))
    assert len(made) >= 10
    ws = torch.full((max(c[-1] for c in made) + GUARD,), start, dtype=torch.uint8, device="cuda")
    for order in (made, made[::-1]):
        for kind, codes, scales, x, y, size in order:
            behind = ws[size:].clone()
            out = torch.full_like(y, float("nan"))
            b.aiq_mx_linear(codes, scales, None, x, out, workspace=ws[:size])
            assert torch.equal(out, y), (kind, y.shape)
            assert torch.equal(ws[size:], behind)


def _one_weight_per_channel(n, k, seed):
    """Channels with one element other than zero, +-1, 2 or 4 times 2^-2: (codes, scales, its k, its value)."""
    g = torch.Generator().manual_seed(seed)
    # every k in turn, the last ones first: the ends of blocks, of 128, 512 and of K are all met
    at = (k - 1 - torch.arange(n) * max(1, k // n)) % k
    e, sign = torch.randint(0, 3, (n,), generator=g), torch.randint(0, 2, (n,), generator=g)
    codes = torch.zeros((n, -(-k // 128) * 128), dtype=torch.uint8)
    codes[torch.arange(n), at] = (2 * (e + 1) + 8 * sign).to(torch.uint8)
    scales = torch.zeros((n, -(-k // 512) * 16), dtype=torch.uint8)
    scales[:, : -(-k // 32)] = 125
    return (codes[:, 0::2] | (codes[:, 1::2] << 4)).cuda(), scales.cuda(), at, 2.0 ** (e.double() - 2) * (1 - 2 * sign)


# With one weight other than zero there is nothing to add up: y is x times a power of two, and float32, half and bfloat16 hold that.  x has every
# bit of its type's mantissa and lies within 2^-8 of its block's largest, so its pieces hold it: 2^-22 of that one at bfloat16 (8 bits below 2^-8),
# 2^-27 at half (11), 2^-37 at float32 (24).  A piece left out, or scaled or placed wrongly, shows in the last bits of some channel.
# In turn: rows of x beside each other (pieces stacked), above each other, split K ranges, whole tiles and halves of them, the few-row kernel.
@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("n,k,m", [(1100, 1000, 20), (609, 4100, 37), (200, 6000, 33), (700, 640, 257), (2500, 520, 2200), (1290, 650, 3500), (257, 9000, 70),
                                   (1001, 3001, 48), (9500, 520, 16), (128, 8192, 600), (300, 33000, 40), (64, 320, 9), (100, 3001, 3), (2050, 640, 1), (4300, 1000, 1), (700, 6001, 1)])
def test_one_weight_per_channel_is_exact(dtype, n, k, m):
    dt = TYPES[dtype]
    codes, scales, at, w = _one_weight_per_channel(n, k, n)
    g = torch.Generator().manual_seed(k + m)
    x = (1 + torch.rand((m, k), generator=g)) * torch.exp2(torch.randint(-4, 4, (m, k), generator=g).float())
    x = (x * (1 - 2 * torch.randint(0, 2, (m, k), generator=g))).to(dt)
    y = linear(codes, scales, None, x.cuda(), torch.full((m, n), float("nan"), dtype=dt, device="cuda"))
    assert torch.equal(y.cpu(), (x[:, at].double() * w).to(dt))


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("n,k,m", [(1100, 1000, 20), (200, 6000, 33), (700, 640, 257), (2500, 520, 2200), (1290, 650, 3500), (128, 8192, 600), (300, 200000, 40),
                                   (64, 320, 9), (2050, 640, 1)])
def test_one_weight_per_channel_is_exact_with_both_microscaled(dtype, n, k, m):
    b, dt = binding(), TYPES[dtype]
    codes, scales, at, w = _one_weight_per_channel(n, k, n)
    ac, as_ = held(activations(m, k, torch.float32, k + m))
    x = torch.from_numpy(values(ac, as_, k))
    y = torch.full((m, n), float("nan"), dtype=dt, device="cuda")
    b.aiq_mx_matmul(ac, as_, codes, scales, None, k, y)
    assert torch.equal(y.cpu(), (x[:, at] * w).float().to(dt))


# How far float32 sums are off in the mean.  An MMA drops what is below the last place of the sum so far, up to a unit of 2^-23 of it, 0.58 of one in
# root mean square.  Of the 16 MMAs of a piece and 512 k only the largest piece's meet sums of full size (the smaller pieces come first, each
# 2^-5 of the next), the j-th of them sqrt(j / 16) of it: 0.58 (1 + 2^-5 + ...) sum_j sqrt(j / 16) < 7 units, if all add up.  From set to set the sums'
# signs are as good as independent, as are the K / 512 roundings of half a unit behind them.  With s = sqrt(sum (x w)^2), the standard
# deviation of y: below (7 + sqrt(K / 512) / 2) 2^-23 s.  (What one accumulator for all of K costs shows in the long sums above, the pieces in
# the single weights.)
@pytest.mark.parametrize("n,k,m", [(4096, 4096, 256), (10240, 20000, 40), (2048, 8192, 2048)])
def test_float32_sums_in_the_mean(n, k, m):
    codes, scales = held(weights(n, k, n + k))
    x = activations(m, k, torch.float32, m + k)
    y = linear(codes, scales, None, x, torch.full((m, n), float("nan"), device="cuda"))
    few = torch.cat((torch.arange(64), torch.arange(n - 64, n))).cuda()
    w, xd = _rows_of(codes[few], scales[few], k), x.double()
    e = y[:, few].double() - xd @ w.t()
    s = ((xd * xd) @ (w * w).t()).sqrt()
    rms = (e / s).square().mean().sqrt().item()
    print(f"{n} x {k}, {m} rows: {rms:.3g}, allowed {(7 + (k / 512) ** 0.5 / 2) * 2.0 ** -23:.3g}")
    assert rms <= (7 + (k / 512) ** 0.5 / 2) * 2.0 ** -23


# In turn: whole tiles written by their block, a cluster that writes its sums into each other's shared memory, one that reads them from there.
@pytest.mark.parametrize("kind", ["f32", "f16", "bf16", "mx"])
@pytest.mark.parametrize("n,k,m", [(1290, 650, 3500), (200, 6000, 33), (128, 8192, 600)])
def test_a_wait_that_runs_out_ends_in_nan(kind, n, k, m):
    """An arrival held back, a limit of about a millisecond: the kernel ends by itself with NaN in y; the next call is as ever."""
    b, dt = binding(), TYPES.get(kind, torch.float32)
    codes, scales = held(weights(n, k, 1))
    x = activations(m, k, dt, 2)
    xc, xs = held(x)
    size = b.aiq_mx_linear_workspace_bytes(n, k, m, dt)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")

    def call():
        y = torch.zeros((m, n), dtype=dt, device="cuda")
        if kind == "mx":
            b.aiq_mx_matmul(xc, xs, codes, scales, None, k, y)
        else:
            b.aiq_mx_linear(codes, scales, None, x, y, workspace=ws)
        return y
    want = call()
    assert torch.isfinite(want).all()
    b.aiq_debug_mx_expire_wait(2_000_000)
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    y = call()
    end.record()
    torch.cuda.synchronize()
    assert torch.isnan(y).all()
    assert start.elapsed_time(end) < 1000.0
    assert torch.equal(call(), want)
    b.aiq_debug_mx_expire_wait(2_000_000)
    b.aiq_debug_mx_expire_wait(0)                                      # taken back
    assert torch.equal(call(), want)


def test_limits_that_are_refused():
    b = binding()
    for limit in (-1, 2_000_000_001):
        with pytest.raises(b.AiqError) as e:
            b.aiq_debug_mx_expire_wait(limit)
        assert e.value.status == b.ERR_INVALID_ARG


@pytest.mark.parametrize("stride", [-1, 0, 1 << 62])
def test_the_stride_of_a_single_row_is_ignored(stride):
    b, n, k = binding(), 300, 700
    codes, scales = held(weights(n, k, 1))
    for kind, dt in TYPES.items():
        code = b._dtype(dt)
        x = activations(1, k, dt, 2)
        xc, xs = held(x)
        c, s = torch.zeros_like(xc), torch.zeros_like(xs)
        assert b.lib.aiq_mx_quantize(x.data_ptr(), code, 1, k, stride, c.data_ptr(), s.data_ptr(), None) == b.OK
        wide = torch.full((1, k), float("nan"), dtype=dt, device="cuda")
        assert b.lib.aiq_mx_dequantize(c.data_ptr(), s.data_ptr(), 1, k, code, wide.data_ptr(), stride, None) == b.OK
        y, z = (torch.full((1, n), float("nan"), dtype=dt, device="cuda") for _ in range(2))
        assert b.lib.aiq_mx_linear(codes.data_ptr(), scales.data_ptr(), None, n, k, x.data_ptr(), code, 1, stride, y.data_ptr(), stride, None, 0, None) == b.OK
        assert b.lib.aiq_mx_matmul(xc.data_ptr(), xs.data_ptr(), 1, codes.data_ptr(), scales.data_ptr(), n, None, k, z.data_ptr(), code, stride, None) == b.OK
        torch.cuda.synchronize()
        assert torch.equal(c, xc) and torch.equal(s, xs)
        assert torch.equal(wide.cpu(), torch.from_numpy(values(c, s, k)).to(dt))
        check(y, x.double().cpu().numpy(), values(codes, scales, k), None, dt, kind)
        check(z, values(xc, xs, k), values(codes, scales, k), None, dt, "mx")


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("n,k,m", [(300, 700, 1), (1100, 1500, 70), (4400, 1000, 1)])
def test_calls_through_ctypes(monkeypatch, dtype, n, k, m):
    """The four calls on the way that the binding takes where its CPython module is not built: the same bits."""
    b, dt = binding(), TYPES[dtype]
    assert b._mxcall is not b.lib, "the module is built where the tests run"
    w, x = weights(n, k, 1), activations(m, k, dt, 2)
    bias = torch.randn(n, generator=torch.Generator().manual_seed(3)).cuda()

    def run():
        codes, scales = held(w)
        xc, xs = held(x)
        back = torch.empty((n, k), dtype=dt, device="cuda")
        b.aiq_mx_dequantize(codes, scales, back)
        y = linear(codes, scales, bias, x, torch.empty((m, n), dtype=dt, device="cuda"))
        z = torch.empty((m, n), dtype=dt, device="cuda")
        b.aiq_mx_matmul(xc, xs, codes, scales, bias, k, z)
        return codes, scales, xc, xs, back, y, z
    want = run()
    monkeypatch.setattr(b, "_mxcall", b.lib)
    for got, w_ in zip(run(), want):
        assert torch.equal(got, w_)
    with pytest.raises(b.AiqError):
        b.aiq_mx_dequantize(want[0], want[1], torch.empty((1, k), dtype=dt, device="cuda").expand(n, k))


def test_codes_that_are_no_matrix():
    b = binding()
    codes, scales = held(weights(8, 64, 1))
    x, y = activations(2, 64, torch.float32, 2), torch.empty((2, 8), device="cuda")
    for bad in (codes[0, 0], codes[0], codes[None]):
        with pytest.raises(ValueError):
            b.aiq_mx_linear(bad, scales, None, x, y)
        with pytest.raises(ValueError):
            b.aiq_mx_quantize(x, bad, scales)
        with pytest.raises(ValueError):
            b.aiq_mx_matmul(codes, scales, bad, scales, None, 64, y)


# The integer kernel (one row of 16 bits, N K > 2^20), well above its border: every end of a row, few channels and many, x on odd addresses, NaN and infinities, a captured
# call, blocks from subnormal numbers to the largest.
MANY = [(4200, 1000), (16500, 257), (36000, 120), (300, 16500), (70, 60500), (127, 33100), (2100, 2049), (131100, 32), (530000, 8), (4200000, 1)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n,k", MANY)
def test_one_row_against_many_weights(dtype, n, k):
    dt = TYPES[dtype]
    codes, scales = held(weights(n, k, n + k))
    w = _rows_of(codes, scales, k)
    bias = torch.randn(n, generator=torch.Generator().manual_seed(3)).cuda() if n % 2 == 0 else None
    for skip in (0, 1):
        x = activations(1, k + skip, dt, k)[:, skip:]
        y = linear(codes, scales, bias, x, torch.full((1, n), float("nan"), dtype=dt, device="cuda"))
        z = x.double() if bias is None else torch.cat((x.double(), torch.ones((1, 1), dtype=torch.float64, device="cuda")), 1)
        _check_exact_products(y, z, w if bias is None else torch.cat((w, bias.double()[:, None]), 1), f"skip {skip}")
        assert torch.equal(y, linear(codes, scales, bias, x, torch.empty_like(y)))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_one_row_of_every_size_against_many_weights(dtype):
    dt, n, k = TYPES[dtype], 6600, 640
    w = weights(n, k, 91).cpu()
    w[3, 40:80] = 0
    codes, scales = held(w.cuda())
    x = activations(1, k, torch.float32, 92).cpu()
    x[0, 64:96] = 0
    x[0, 96:128] = -x[0, 96:128].abs()
    x[0, 128:160] *= torch.logspace(-8, 0, 32)
    if dtype == "f16":
        x[0, :32] *= 2.0 ** -16
        x[0, 32:64] = 60000.0
        scales[:, 0], scales[:, 1] = 140, 100
    else:
        x[0, :32] *= 2.0 ** -122
        x[0, 32:64] *= 2.0 ** 100
        x[0, 160:192] = torch.arange(1, 33) * 2.0 ** -133
        x[0, 192:224] = torch.logspace(-39, 35, 32, dtype=torch.float64).float()
        scales[:, 0], scales[:, 1], scales[:, 5], scales[:, 6] = 245, 10, 254, 2
    x = x.to(dt).cuda()
    y = linear(codes, scales, None, x, torch.full((1, n), float("nan"), dtype=dt, device="cuda"))
    _check_exact_products(y, x, _rows_of(codes, scales, k), "")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_one_row_with_nan_and_infinity_against_many_weights(dtype):
    dt, n, k = TYPES[dtype], 4100, 1100
    w = weights(n, k, 93)
    w[5, 1099], w[4099, 0] = float("nan"), float("inf")
    codes, scales = held(w)
    for what in (float("nan"), float("inf"), -float("inf")):
        x = activations(1, k, dt, 94)
        x[0, 1070] = what
        assert torch.isnan(linear(codes, scales, None, x, torch.zeros((1, n), dtype=dt, device="cuda"))).all()
    x = activations(1, k, dt, 94)
    y = linear(codes, scales, None, x, torch.zeros((1, n), dtype=dt, device="cuda"))
    assert torch.isnan(y[0, [5, 4099]]).all()
    keep = [i for i in range(n) if i not in (5, 4099)]
    _check_exact_products(y[:, keep], x, _rows_of(codes[keep], scales[keep], k), "")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_one_row_against_many_weights_captured(dtype):
    """A replay reads the x of its time, what its blocks leave out too; elements of y's buffer beside the row stay as they were."""
    dt, n, k = TYPES[dtype], 8205, 520
    codes, scales = held(weights(n, k, 95))
    w = _rows_of(codes, scales, k)
    x, wide = activations(1, k, dt, 96), torch.full((1, n + 7), 7.0, dtype=dt, device="cuda")
    y = wide[:, 3:3 + n]
    linear(codes, scales, None, x, y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        linear(codes, scales, None, x, y)
    for seed in (97, 98):
        new = activations(1, k, dt, seed)
        new[0, 5::32] *= 2.0 ** -(14 if dtype == "f16" else 40)
        x.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        _check_exact_products(y, x, w, f"{seed}")
        assert (wide[:, :3] == 7.0).all() and (wide[:, 3 + n:] == 7.0).all()
