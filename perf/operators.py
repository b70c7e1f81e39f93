"""Microscaled 4-bit operators as measurable cases: quantising, expanding, and the two products.

A row of K values is cut into blocks of 32.  A block is held as 32 four-bit floating-point codes (sign, two exponent
bits, one mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) and one byte s that scales them by 2^(s - 127):

  quantize    aiq_mx_quantize: values to codes and scale bytes (what it stored is read back with aiq_mx_dequantize)
  dequantize  aiq_mx_dequantize: codes and scale bytes to values
  linear      aiq_mx_linear: y = x * W^T + bias, W microscaled, x in 16 or 32 bits
  matmul      aiq_mx_matmul: y = A * B^T + bias, both microscaled

`run` computes them from elementary torch operations where `own` is false, and through the package's entry points
where it is true.  Everything is drawn on the GPU from the case's seed.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def listed():
    return [
        # packing the weights of MobileNetV2's head: the smallest call
        dict(name="quantize_head_f32", op="quantize", rows=1280, k=320, dtype="f32", pad=0),
        # packing a large layer of a 16-bit checkpoint
        dict(name="quantize_8192_bf16", op="quantize", rows=8192, k=8192, dtype="bf16", pad=0),
        # activations of a ragged batch, rows of odd length that are a slice of wider ones
        dict(name="quantize_ragged_f16", op="quantize", rows=4099, k=1283, dtype="f16", pad=5),
        # expanding a classifier with rows of odd length, for a layer that wants float32
        dict(name="dequantize_1000_f32", op="dequantize", rows=1000, k=1281, dtype="f32"),
        # expanding a large layer back to 16 bits
        dict(name="dequantize_8192_bf16", op="dequantize", rows=8192, k=8192, dtype="bf16"),
        # one row through MobileNetV2's head: nothing but latency
        dict(name="linear_head_f32_m1", op="linear", n=1280, k=320, m=1, dtype="f32", bias=True),
        # a single token through a large layer: the weight stream
        dict(name="linear_8192_bf16_m1", op="linear", n=8192, k=8192, m=1, dtype="bf16", bias=False),
        # a small ragged batch through a layer of odd sizes
        dict(name="linear_ragged_f16_m37", op="linear", n=5671, k=609, m=37, dtype="f16", bias=True),
        # a batch of the linear sweep in the package's own activation type
        dict(name="linear_4096_f32_m256", op="linear", n=4096, k=4096, m=256, dtype="f32", bias=False),
        # a prompt through a large layer: the tensor cores
        dict(name="linear_8192_bf16_m2048", op="linear", n=8192, k=8192, m=2048, dtype="bf16", bias=True),
        # a small batch, activations microscaled too
        dict(name="matmul_4096_bf16_m16", op="matmul", n=4096, k=4096, m=16, dtype="bf16", bias=True),
        # a prompt, activations microscaled too
        dict(name="matmul_8192_bf16_m2048", op="matmul", n=8192, k=8192, m=2048, dtype="bf16", bias=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["quantize", "dequantize", "linear", "linear", "linear", "matmul", "matmul"])
    dtype = rng.choice(sorted(TYPES))
    n, k = _log_int(rng, 64, 8192), _log_int(rng, 64, 8192)
    # half of them rows a multiple of 32 long, as layers usually are; the rest of any length
    if rng.random() < 0.5:
        k = max(64, k // 32 * 32)
    if op == "quantize":
        return dict(op=op, rows=n, k=k, dtype=dtype, pad=rng.choice([0, 0, rng.randint(1, 64)]))
    if op == "dequantize":
        return dict(op=op, rows=n, k=k, dtype=dtype)
    return dict(op=op, n=n, k=k, m=_log_int(rng, 1, 2048), dtype=dtype, bias=rng.random() < 0.5)


# ------------------------------------------------------------------------- layout
# Codes: rows of ceil(K / 128) * 64 bytes, element 2j in the low and 2j + 1 in the high nibble of byte j.  Scales: rows
# of ceil(K / 512) * 16 bytes, one for each block.  What lies behind K is zero.
def _row_bytes(k):
    return (k + 127) // 128 * 64


def _scale_row_bytes(k):
    return (k + 511) // 512 * 16


def _power(e):
    """2^e as float32 for whole numbers -126 <= e <= 127, from its bits: pow() and ldexp() are a bit off on a GPU."""
    return ((e + 127) << 23).int().view(torch.float32)


def _scaled(v, s):
    """v * 2^(s - 127), exactly; s may be 0, whose power is subnormal."""
    return v * 0.5 * _power(s - 126)[:, :, None]


def _values(codes, scales, k):
    """The float32 values that codes and scales stand for, [rows][k]."""
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0],
                         dtype=torch.float32, device=codes.device)
    rows = codes.shape[0]
    nibbles = torch.stack((codes & 15, codes >> 4), dim=2).view(rows, -1)
    v = table[nibbles.int()].view(rows, -1, 32)
    s = scales[:, :v.shape[1]].int()
    return _scaled(v, s).view(rows, -1)[:, :k]


def _quantize(x):
    """(magnitude index 0..7, negative, scale byte) of float32 rows, blocks of 32; [rows][blocks][32] and [rows][blocks]."""
    rows, k = x.shape
    x = torch.nn.functional.pad(x, (0, -k % 32)).view(rows, -1, 32)
    top = x.abs().amax(dim=2)
    exponent = (top.view(torch.int32) >> 23) & 255            # floor(log2) + 127; 0 for zero and subnormal numbers
    s = (exponent - 2).clamp_min(0)
    a = x.abs() * _power(127 - s)[:, :, None]
    # round to nearest, ties to the code with a zero mantissa bit
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    return code, torch.signbit(x), s


def _pack(x):
    """Codes and scales of float32 rows in the stored layout."""
    rows, k = x.shape
    code, negative, s = _quantize(x)
    nibbles = (code | (negative.to(torch.uint8) << 3)).view(rows, -1)
    nibbles = torch.nn.functional.pad(nibbles, (0, 2 * _row_bytes(k) - nibbles.shape[1]))
    codes = nibbles[:, 0::2] | (nibbles[:, 1::2] << 4)
    scales = torch.nn.functional.pad(s.to(torch.uint8), (0, _scale_row_bytes(k) - s.shape[1]))
    return codes.contiguous(), scales.contiguous()


# ------------------------------------------------------------------------- inputs
def _randn(shape, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda")


def _weights(n, k, seed):
    """Weights of a trained layer: normal, with output channels of different size."""
    return _randn((n, k), seed) * (0.02 * torch.exp(0.5 * _randn((n, 1), seed + 1)))


def _activations(m, k, seed):
    """Activations: normal, with some columns an order of magnitude larger than the rest."""
    return _randn((m, k), seed) * torch.exp(0.8 * _randn((1, k), seed + 1))


def prepare(case, seed):
    op, k, dtype = case["op"], case["k"], TYPES[case["dtype"]]
    base = 8 * seed
    aiq = None
    if own:
        from paper_2512_14090_b200 import binding as aiq
    if op in ("quantize", "dequantize"):
        rows = case["rows"]
        s = dict(case=case, aiq=aiq, y=torch.empty((rows, k), dtype=dtype, device="cuda"))
        if op == "quantize":
            wide = _weights(rows, k + case["pad"], base).to(dtype)
            s["x"] = wide[:, case["pad"]:]
            s["codes"] = torch.empty((rows, _row_bytes(k)), dtype=torch.uint8, device="cuda")
            s["scales"] = torch.empty((rows, _scale_row_bytes(k)), dtype=torch.uint8, device="cuda")
        else:
            s["codes"], s["scales"] = _pack(_weights(rows, k, base))
        return s
    n, m = case["n"], case["m"]
    s = dict(case=case, aiq=aiq, y=torch.empty((m, n), dtype=dtype, device="cuda"),
             bias=_randn((n,), base + 4) * 0.1 if case["bias"] else None)
    s["codes"], s["scales"] = _pack(_weights(n, k, base))
    x = _activations(m, k, base + 2)
    if op == "linear":
        s["x"] = x.to(dtype)
        if own:
            s["ws"] = torch.empty(aiq.aiq_mx_linear_workspace_bytes(n, k, m, dtype), dtype=torch.uint8, device="cuda")
    else:
        s["x_codes"], s["x_scales"] = _pack(x)
    return s


# ------------------------------------------------------------------------- one pass
def run(s):
    case = s["case"]
    op, k, y = case["op"], case["k"], s["y"]
    if own:
        aiq = s["aiq"]
        if op == "quantize":
            aiq.aiq_mx_quantize(s["x"], s["codes"], s["scales"])
            aiq.aiq_mx_dequantize(s["codes"], s["scales"], y)
        elif op == "dequantize":
            aiq.aiq_mx_dequantize(s["codes"], s["scales"], y)
        elif op == "linear":
            aiq.aiq_mx_linear(s["codes"], s["scales"], s["bias"], s["x"], y, workspace=s["ws"])
        else:
            aiq.aiq_mx_matmul(s["x_codes"], s["x_scales"], s["codes"], s["scales"], s["bias"], k, y)
        return y
    if op == "quantize":
        code, negative, e = _quantize(s["x"].float())
        table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float32, device=code.device)
        v = _scaled(table[code.int()], e)
        v = torch.where(negative, -v, v).view(code.shape[0], -1)[:, :k]
    elif op == "dequantize":
        v = _values(s["codes"], s["scales"], k)
    else:
        x = s["x"].float() if op == "linear" else _values(s["x_codes"], s["x_scales"], k)
        v = x @ _values(s["codes"], s["scales"], k).t()
        if s["bias"] is not None:
            v = v + s["bias"]
    return v.to(y.dtype).contiguous()


def work(case):
    k, size = case["k"], {"f32": 4, "f16": 2, "bf16": 2}[case["dtype"]]
    held = k / 2 + k / 32                                      # bytes of a microscaled row
    if case["op"] == "quantize":                               # values in, codes and scales out, and the values they stand for
        return dict(bytes=case["rows"] * (2 * size * k + held), flops=2 * case["rows"] * k)
    if case["op"] == "dequantize":
        return dict(bytes=case["rows"] * (held + size * k), flops=case["rows"] * k)
    n, m = case["n"], case["m"]
    x = m * (size * k if case["op"] == "linear" else held)
    return dict(bytes=n * held + x + m * n * size + (4 * n if case["bias"] else 0), flops=2 * m * n * k)


# ------------------------------------------------------------------------- in 64 bits
def _power64(e):
    return ((e + 1023) << 52).view(torch.float64)


def _exact_values(codes, scales, k):
    """Sign, exponent and mantissa of every code, put together in float64."""
    c = torch.empty((codes.shape[0], 2 * codes.shape[1]), dtype=torch.int64, device=codes.device)
    c[:, 0::2] = codes.long() % 16
    c[:, 1::2] = codes.long() // 16
    c = c[:, :k]
    e, mantissa = c // 2 % 4, c % 2
    v = torch.where(e == 0, mantissa.double() / 2, (1 + mantissa.double() / 2) * _power64(e - 1))
    block = torch.arange(k, device=codes.device) // 32
    v = v * _power64(scales.long() - 127)[:, block]
    return torch.where(c >= 8, -v, v)


def _exact_quantized(x):
    """The nearest of the eight magnitudes times the block's scale, in float64; between two, the one of even index."""
    rows, k = x.shape
    out = torch.empty((rows, k), dtype=torch.float64, device=x.device)
    step = max(1, (1 << 24) // k)
    for r in range(0, rows, step):
        a = x[r:r + step].double()
        blocks = torch.nn.functional.pad(a.abs(), (0, -k % 32)).view(a.shape[0], -1, 32)
        top = blocks.amax(dim=2)
        _, e = torch.frexp(top)                                # top = f 2^e, f in [0.5, 1)
        e = torch.where(top > 0, (e - 3).clamp_min(-127), torch.full_like(e, -127)).long()
        unit = _power64(e).repeat_interleave(32, dim=1)[:, :k]
        q = a.abs() / unit
        # the grid is 1/2 below 2, 1 up to 4 and 2 above; torch.round takes the even multiple between two
        grid = torch.where(q < 2, 0.5, torch.where(q < 4, 1.0, 2.0)).double()
        q = (torch.round(q / grid) * grid).clamp_max(6.0)
        out[r:r + step] = torch.copysign(q * unit, a)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    op, k = case["op"], case["k"]
    if op == "quantize":
        return _exact_quantized(s["x"])
    w = _exact_values(s["codes"], s["scales"], k)
    if op == "dequantize":
        return w
    x = s["x"].double() if op == "linear" else _exact_values(s["x_codes"], s["x_scales"], k)
    y = x @ w.t()
    return y + s["bias"].double() if s["bias"] is not None else y
