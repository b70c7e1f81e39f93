"""A feed-forward layer and a layer of experts with microscaled 4-bit weights, as measurable cases.

  act      aiq_mx_linear_act: y = act(x W^T + bias) + residual; gated: y = act(x G^T + bias_g) * (x U^T + bias_u) + residual,
           where G is the first half of the rows of W and U the second
  route    aiq_route_experts: the experts of every token, their weights, and the plan: all (token, expert) pairs sorted by expert
  experts  aiq_mx_linear_experts: act(x[row] W[expert of row]^T + bias[expert of row]) for the sorted rows
  combine  aiq_combine_experts: every token's weighted sum of its experts' rows, plus residual

W is held as in operators.py: blocks of 32 four-bit floating-point codes and one byte s that scales them by 2^(s - 127).
`run` computes them from elementary torch operations where `own` is false, and through the package's entry points where it is
true.  Everything is drawn on the GPU from the case's seed.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ACTIVATIONS = ["none", "relu", "relu6", "silu", "gelu", "gelu_tanh"]


def listed():
    return [
        # one row through MobileNetV2's head and its activation: nothing but latency
        dict(name="act_head_f32_m1", op="act", n=1280, k=320, m=1, dtype="f32", bias=True, act="relu6", gated=False, residual=False),
        # a single token through the gated half of a large feed-forward layer: the weight stream
        dict(name="act_gated_8192_bf16_m1", op="act", n=16384, k=4096, m=1, dtype="bf16", bias=False, act="silu", gated=True, residual=False),
        # a small ragged batch through a layer of odd sizes
        dict(name="act_ragged_f16_m37", op="act", n=5671, k=609, m=37, dtype="f16", bias=True, act="gelu_tanh", gated=False, residual=True),
        # a prompt through the gated half of a large feed-forward layer: the tensor cores
        dict(name="act_gated_8192_bf16_m2048", op="act", n=8192, k=8192, m=2048, dtype="bf16", bias=True, act="silu", gated=True, residual=True),
        # the experts of one token: nothing but latency
        dict(name="route_f32_t1", op="route", tokens=1, experts=32, top_k=4, dtype="f32", scoring="softmax", bias=False, groups=1,
             top_groups=1, group_best=1, renormalise=True, padded=0),
        # an odd number of tokens, some of them padding, and of experts
        dict(name="route_ragged_f16_t997", op="route", tokens=997, experts=60, top_k=6, dtype="f16", scoring="softmax", bias=True, groups=1,
             top_groups=1, group_best=1, renormalise=False, padded=41),
        # a long prompt among many experts in groups, with a bias for balance
        dict(name="route_grouped_bf16_t16384", op="route", tokens=16384, experts=256, top_k=8, dtype="bf16", scoring="sigmoid", bias=True,
             groups=8, top_groups=4, group_best=2, renormalise=True, padded=0),
        # one token through its four experts: their weights' stream
        dict(name="experts_bf16_t1", op="experts", tokens=1, experts=32, top_k=4, n=4096, k=2048, dtype="bf16", bias=False, act="silu",
             gated=True, sorted=False, padded=0),
        # a few requests at once, some of them padding, rows of odd sizes, almost every expert in use
        dict(name="experts_ragged_f16_t50", op="experts", tokens=50, experts=60, top_k=6, n=1411, k=1000, dtype="f16", bias=True, act="none",
             gated=False, sorted=True, padded=3),
        # a prompt: the tensor cores
        dict(name="experts_bf16_t4096", op="experts", tokens=4096, experts=32, top_k=4, n=4096, k=2048, dtype="bf16", bias=True, act="silu",
             gated=True, sorted=False, padded=0),
        # the weighted sum for one token
        dict(name="combine_bf16_t1", op="combine", tokens=1, experts=32, top_k=4, k=2048, dtype="bf16", residual=True, padded=0),
        # and for a prompt
        dict(name="combine_bf16_t4096", op="combine", tokens=4096, experts=64, top_k=8, k=4096, dtype="bf16", residual=True, padded=0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A row's length: half of them a multiple of 32, as layers usually are; the rest of any length."""
    k = _log_int(rng, lo, hi)
    return max(32, k // 32 * 32) if rng.random() < 0.5 else k


def draw(rng):
    op = rng.choice(["act", "act", "act", "route", "route", "experts", "experts", "experts", "combine"])
    dtype = rng.choice(sorted(TYPES))
    if op == "act":
        gated = rng.random() < 0.5
        n = _log_int(rng, 64, 8192)
        return dict(op=op, n=n + n % 2 if gated else n, k=_width(rng, 64, 8192), m=_log_int(rng, 1, 2048), dtype=dtype, bias=rng.random() < 0.5,
                    act=rng.choice(ACTIVATIONS), gated=gated, residual=rng.random() < 0.5)
    experts = _log_int(rng, 4, 256)
    if op == "route":
        tokens = _log_int(rng, 1, 16384)
        groups = rng.choice([1, 1, 2, 4, 8])
        experts = max(2, experts // groups) * groups
        top_groups = rng.randint(1, groups)
        top_k = rng.randint(1, min(8, experts // groups * top_groups))
        return dict(op=op, tokens=tokens, experts=experts, top_k=top_k, dtype=dtype, scoring=rng.choice(["softmax", "sigmoid"]),
                    bias=rng.random() < 0.5, groups=groups, top_groups=top_groups, group_best=rng.choice([1, 2]),
                    renormalise=rng.random() < 0.5, padded=rng.choice([0, tokens // 16]))
    tokens, top_k = _log_int(rng, 1, 4096), rng.randint(1, min(8, experts))
    padded = rng.choice([0, tokens // 16])
    if op == "combine":
        return dict(op=op, tokens=tokens, experts=experts, top_k=top_k, k=_width(rng, 64, 4096), dtype=dtype, residual=rng.random() < 0.5,
                    padded=padded)
    gated = rng.random() < 0.5
    experts, top_k = min(experts, 64), min(top_k, 4)
    n = _log_int(rng, 64, 4096)
    return dict(op=op, tokens=tokens, experts=experts, top_k=top_k, n=n + n % 2 if gated else n, k=_width(rng, 64, 2048), dtype=dtype,
                bias=rng.random() < 0.5, act=rng.choice(ACTIVATIONS), gated=gated, sorted=rng.random() < 0.5, padded=padded)


# ------------------------------------------------------------------------- microscaled weights
# Codes: rows of ceil(K / 128) * 64 bytes, element 2j in the low and 2j + 1 in the high nibble of byte j.  Scales: rows
# of ceil(K / 512) * 16 bytes, one for each block.  What lies behind K is zero.
def _row_bytes(k):
    return (k + 127) // 128 * 64


def _scale_row_bytes(k):
    return (k + 511) // 512 * 16


def _power(e):
    """2^e as float32 for whole numbers -126 <= e <= 127, from its bits."""
    return ((e + 127) << 23).int().view(torch.float32)


def _pack(x):
    """Codes and scales of float32 rows."""
    rows, k = x.shape
    x = torch.nn.functional.pad(x, (0, -k % 32)).view(rows, -1, 32)
    s = (((x.abs().amax(dim=2).view(torch.int32) >> 23) & 255) - 2).clamp_min(0)
    a = x.abs() * _power(127 - s)[:, :, None]
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    nibbles = (code | (torch.signbit(x).to(torch.uint8) << 3)).view(rows, -1)
    nibbles = torch.nn.functional.pad(nibbles, (0, 2 * _row_bytes(k) - nibbles.shape[1]))
    scales = torch.nn.functional.pad(s.to(torch.uint8), (0, _scale_row_bytes(k) - s.shape[1]))
    return (nibbles[:, 0::2] | (nibbles[:, 1::2] << 4)).contiguous(), scales.contiguous()


def _values(codes, scales, k):
    """The float32 values of rows of codes and scales, [rows][k]."""
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0],
                         dtype=torch.float32, device=codes.device)
    rows = codes.shape[0]
    v = table[torch.stack((codes & 15, codes >> 4), dim=2).view(rows, -1).int()].view(rows, -1, 32)
    s = scales[:, :v.shape[1]].int()
    return (v * 0.5 * _power(s - 126)[:, :, None]).view(rows, -1)[:, :k]


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


def _logits(tokens, experts, padded, seed):
    """A router's logits: normal, some experts more popular than others; -inf in the rows of the padding at the end."""
    l = _randn((tokens, experts), seed) + 0.5 * _randn((1, experts), seed + 1)
    if padded:
        l[tokens - padded:] = -math.inf
    return l


def _sorted_pairs(ids, experts):
    """(offsets [experts + 1], slots, positions) of ids [tokens][top_k]: slot t * top_k + j of token t, sorted by expert and then by slot;
    slots without an expert (-1) come behind all others in `slots`, as -1, and have position -1."""
    flat = ids.reshape(-1).long()
    key = torch.where(flat < 0, experts, flat)
    order = torch.sort(key, stable=True).indices
    counts = torch.zeros(experts + 1, dtype=torch.int64, device=ids.device).scatter_add_(0, key, torch.ones_like(key))
    ends = torch.cumsum(counts[:experts], 0)
    offsets = torch.cat((torch.zeros_like(ends[:1]), ends))
    at = torch.arange(len(flat), device=ids.device)
    positions = torch.empty_like(at).scatter_(0, order, at)
    return offsets.int(), torch.where(at < offsets[-1], order, -1).int(), torch.where(flat < 0, -1, positions).int().view(ids.shape)


def _ids(case, seed):
    """Experts of every token, from the logits of a router."""
    l = _logits(case["tokens"], case["experts"], case["padded"], seed)
    top = torch.sort(l, dim=1, descending=True, stable=True)
    k = case["top_k"]
    return torch.where(top.values[:, :k] == -math.inf, -1, top.indices[:, :k]).int().contiguous()


def prepare(case, seed):
    base = 16 * seed
    aiq = None
    if own:
        from paper_2512_14090_b200 import binding as aiq
    s = dict(case=case, aiq=aiq)
    op, dtype = case["op"], TYPES[case["dtype"]]
    if op == "route":
        t, e, k = case["tokens"], case["experts"], case["top_k"]
        s["logits"] = _logits(t, e, case["padded"], base).to(dtype)
        s["bias"] = 0.1 * _randn((e,), base + 2) if case["bias"] else None
        if own:
            s["ids"] = torch.empty((t, k), dtype=torch.int32, device="cuda")
            s["weights"] = torch.empty((t, k), dtype=torch.float32, device="cuda")
            s["plan"] = torch.empty(aiq.aiq_expert_plan_bytes(t, k, e), dtype=torch.uint8, device="cuda")
        return s
    if op in ("experts", "combine"):
        t, e, k = case["tokens"], case["experts"], case["top_k"]
        ids = _ids(case, base)
        s["offsets"], s["slots"], s["positions"] = _sorted_pairs(ids, e)
        if own:
            s["plan"] = torch.empty(aiq.aiq_expert_plan_bytes(t, k, e), dtype=torch.uint8, device="cuda")
            aiq.aiq_plan_experts(ids, e, s["plan"])
    if op == "combine":
        w = torch.exp(_randn((t, k), base + 2))
        s["weights"] = w / w.sum(dim=1, keepdim=True)
        s["z"] = _randn((t * k, case["k"]), base + 3).to(dtype)
        s["residual"] = _randn((t, case["k"]), base + 4).to(dtype) if case["residual"] else None
        s["y"] = torch.empty((t, case["k"]), dtype=dtype, device="cuda")
        return s
    n, width = case["n"], case["k"]
    outputs = n // 2 if case["gated"] else n
    if op == "act":
        m = case["m"]
        s["codes"], s["scales"] = _pack(_weights(n, width, base))
        s["bias"] = 0.1 * _randn((n,), base + 2) if case["bias"] else None
        s["x"] = _activations(m, width, base + 4).to(dtype)
        s["residual"] = _randn((m, outputs), base + 6).to(dtype) if case["residual"] else None
        s["y"] = torch.empty((m, outputs), dtype=dtype, device="cuda")
        if own:
            s["ws"] = torch.empty(aiq.aiq_mx_linear_workspace_bytes(n, width, m, dtype), dtype=torch.uint8, device="cuda")
        return s
    held = [_pack(_weights(n, width, base + (j << 20) + 3)) for j in range(e)]
    s["codes"], s["scales"] = torch.stack([h[0] for h in held]), torch.stack([h[1] for h in held])
    s["bias"] = 0.1 * _randn((e, n), base + 6) if case["bias"] else None
    s["x"] = _activations(t * k if case["sorted"] else t, width, base + 8).to(dtype)
    s["y"] = torch.zeros((t * k, outputs), dtype=dtype, device="cuda")             # rows that no expert has stay as they are
    if own:
        s["ws"] = torch.empty(aiq.aiq_mx_linear_experts_workspace_bytes(e, n, width, t * k, dtype), dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------------- one pass
def _activate(v, name):
    if name == "relu":
        return v.clamp_min(0)
    if name == "relu6":
        return v.clamp(0, 6)
    if name == "silu":
        return v / (1 + torch.exp(-v))
    if name == "gelu":
        return 0.5 * v * (1 + torch.erf(v * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * v * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v * v * v)))
    return v


def _layer(x, w, bias, case):
    v = x @ w.t()
    if bias is not None:
        v = v + bias
    if not case["gated"]:
        return _activate(v, case["act"])
    half = v.shape[1] // 2
    return _activate(v[:, :half], case["act"]) * v[:, half:]


def _route(logits, bias, case):
    """Scores and choices in 64 bits: two experts' scores can be as close as float32 rounding."""
    l = logits.double()
    masked = l == -math.inf
    if case["scoring"] == "softmax":
        top = l.amax(dim=1, keepdim=True)
        p = torch.exp(l - torch.where(top == -math.inf, 0, top))
        total = p.sum(dim=1, keepdim=True)
        p = torch.where(total > 0, p / total, 0)
    else:
        p = 1 / (1 + torch.exp(-l))
    # without a bias the scores' order is that of the logits
    choice = p if bias is None else p + bias.double()
    order = torch.where(masked, -math.inf, l if bias is None else choice)
    t, e = l.shape
    g = case["groups"]
    if g > 1:
        best = torch.where(masked, -math.inf, choice).view(t, g, e // g).sort(dim=2, descending=True).values
        score = best[:, :, 0]
        if case["group_best"] == 2:
            score = torch.where(best[:, :, 1] == -math.inf, score, score + best[:, :, 1])
        taken = torch.sort(score, dim=1, descending=True, stable=True).indices[:, :case["top_groups"]]
        open_ = torch.zeros((t, g), dtype=torch.bool, device=l.device).scatter_(1, taken, True)
        order = torch.where(open_.repeat_interleave(e // g, dim=1), order, -math.inf)
    first = torch.sort(order, dim=1, descending=True, stable=True)
    k = case["top_k"]
    none = first.values[:, :k] == -math.inf
    ids = first.indices[:, :k]
    w = torch.where(none, 0, p.gather(1, ids))
    if case["renormalise"]:
        total = w.sum(dim=1, keepdim=True)
        w = torch.where(total > 0, w / total, 0)
    return torch.where(none, -1, ids).int(), w.float()


def run(s):
    case, aiq = s["case"], s["aiq"]
    op = case["op"]
    if own:
        if op == "act":
            aiq.aiq_mx_linear_act(s["codes"], s["scales"], s["bias"], s["x"], s["y"], case["act"], gated=case["gated"], residual=s["residual"],
                                  workspace=s["ws"])
            return s["y"]
        if op == "route":
            aiq.aiq_route_experts(s["logits"], s["ids"], s["weights"], bias=s["bias"], scoring=case["scoring"], groups=case["groups"],
                                  top_groups=case["top_groups"], group_best=case["group_best"], renormalise=case["renormalise"], plan=s["plan"])
            return [s["ids"], s["weights"], *aiq.aiq_expert_plan_parts(s["plan"], case["tokens"], case["top_k"], case["experts"])]
        if op == "experts":
            aiq.aiq_mx_linear_experts(s["codes"], s["scales"], s["bias"], s["x"], s["plan"], case["top_k"], s["y"], case["act"],
                                      gated=case["gated"], x_sorted=case["sorted"], workspace=s["ws"])
            return s["y"]
        aiq.aiq_combine_experts(s["z"], s["weights"], s["plan"], case["experts"], s["y"], residual=s["residual"])
        return s["y"]
    if op == "route":
        ids, weights = _route(s["logits"], s["bias"], case)
        return [ids, weights, *_sorted_pairs(ids, case["experts"])]
    if op == "combine":
        at = s["positions"].long()
        v = (s["z"][at.clamp_min(0)].float() * torch.where(at < 0, 0, s["weights"])[:, :, None]).sum(dim=1)
        if s["residual"] is not None:
            v = v + s["residual"].float()
        return v.to(s["z"].dtype)
    dtype, k = s["x"].dtype, case["k"]
    if op == "act":
        v = _layer(s["x"].float(), _values(s["codes"], s["scales"], k), s["bias"], case)
        if s["residual"] is not None:
            v = v + s["residual"].float()
        return v.to(dtype)
    y = torch.zeros_like(s["y"])
    ends = s["offsets"].tolist()
    for e in range(case["experts"]):
        a, b = ends[e], ends[e + 1]
        if a < b:
            x = s["x"][a:b] if case["sorted"] else s["x"][s["slots"][a:b].long() // case["top_k"]]
            y[a:b] = _layer(x.float(), _values(s["codes"][e], s["scales"][e], k), s["bias"][e] if s["bias"] is not None else None, case).to(dtype)
    return y


def work(case):
    op, size = case["op"], {"f32": 4, "f16": 2, "bf16": 2}[case["dtype"]]
    if op == "route":                                          # logits in; ids, weights, slots and positions, four bytes each, out
        t, e, k = case["tokens"], case["experts"], case["top_k"]
        return dict(bytes=t * e * size + 16 * t * k + 4 * (e + 1) + (4 * e if case["bias"] else 0), flops=10 * t * e)
    if op == "combine":
        rows, pairs, k = case["tokens"], (case["tokens"] - case["padded"]) * case["top_k"], case["k"]
        return dict(bytes=(pairs + rows * (2 if case["residual"] else 1)) * k * size + 8 * rows * case["top_k"], flops=2 * pairs * k)
    n, k = case["n"], case["k"]
    held, outputs = k / 2 + k / 32, n // 2 if case["gated"] else n
    if op == "act":
        m = case["m"]
        return dict(bytes=n * held + m * (k + outputs * (2 if case["residual"] else 1)) * size + (4 * n if case["bias"] else 0), flops=2 * m * n * k)
    tokens = case["tokens"] - case["padded"]
    rows = tokens * case["top_k"]
    used = case["experts"] * (1 - (1 - case["top_k"] / case["experts"]) ** tokens)      # experts that some token has, were all alike
    x = rows if case["sorted"] else tokens
    return dict(bytes=used * n * held + (x * k + rows * outputs) * size + (4 * n * used if case["bias"] else 0) + 4 * rows, flops=2 * rows * n * k)


# ------------------------------------------------------------------------- in 64 bits
def _exact_values(codes, scales, k):
    """Sign, exponent and mantissa of every code, put together in float64."""
    c = torch.empty((codes.shape[0], 2 * codes.shape[1]), dtype=torch.int64, device=codes.device)
    c[:, 0::2] = codes.long() % 16
    c[:, 1::2] = codes.long() // 16
    c = c[:, :k]
    e, mantissa = c // 2 % 4, (c % 2).double()
    v = torch.where(e == 0, mantissa / 2, (1 + mantissa / 2) * ((e - 1 + 1023) << 52).view(torch.float64))
    v = v * ((scales.long() - 127 + 1023) << 52).view(torch.float64)[:, torch.arange(k, device=codes.device) // 32]
    return torch.where(c >= 8, -v, v)


def _exact_act(v, name):
    if name == "none":
        return v
    if name == "relu":
        return torch.where(v > 0, v, 0)
    if name == "relu6":
        return torch.where(v > 6, 6, torch.where(v > 0, v, 0))
    if name == "silu":
        return v * torch.sigmoid(v)
    if name == "gelu":
        return v * torch.special.ndtr(v)
    return v * torch.sigmoid(2 * (2 / math.pi) ** 0.5 * (v + 0.044715 * v ** 3))


def _exact_layer(x, w, bias, case):
    v = x.double() @ w.t()
    if bias is not None:
        v += bias.double()
    if case["gated"]:
        gate, up = v.chunk(2, dim=1)
        return _exact_act(gate, case["act"]) * up
    return _exact_act(v, case["act"])


def _exact_route(logits, bias, case):
    """One choice after the other: the largest, the first of equals."""
    l = logits.double()
    t, e = l.shape
    never = torch.isneginf(l)
    p = torch.sigmoid(l) if case["scoring"] == "sigmoid" else torch.nan_to_num(torch.softmax(l, dim=1))
    biased = p if bias is None else p + bias.double()
    left = (l if bias is None else biased).masked_fill(never, -math.inf)
    size, at = e // case["groups"], torch.arange(e, device=l.device)

    def first_of_largest(v):
        index = torch.arange(v.shape[1], device=v.device)
        return torch.where(v == v.amax(dim=1, keepdim=True), index, v.shape[1]).amin(dim=1)

    if case["groups"] > 1:
        scores = []
        for group in range(case["groups"]):
            v = biased.masked_fill(never, -math.inf)[:, group * size:(group + 1) * size]
            top = v.amax(dim=1)
            if case["group_best"] == 2 and size > 1:
                second = v.scatter(1, first_of_largest(v)[:, None], -math.inf).amax(dim=1)
                top = torch.where(torch.isneginf(second), top, top + second)
            scores.append(top)
        scores = torch.stack(scores, dim=1)
        closed = torch.ones_like(never)
        for _ in range(case["top_groups"]):
            group = first_of_largest(scores)
            closed &= at[None] // size != group[:, None]
            scores = scores.scatter(1, group[:, None], -math.inf)
        left = left.masked_fill(closed, -math.inf)
    ids, w = [], []
    for _ in range(case["top_k"]):
        i = first_of_largest(left)[:, None]
        some = ~torch.isneginf(left.gather(1, i))
        ids.append(torch.where(some, i, -1))
        w.append(torch.where(some, p.gather(1, i), 0))
        left = left.scatter(1, i, -math.inf)
    ids, w = torch.cat(ids, dim=1), torch.cat(w, dim=1)
    if case["renormalise"]:
        w = torch.nan_to_num(w / w.sum(dim=1, keepdim=True))
    return ids.int(), w


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "route":
        ids, w = _exact_route(s["logits"], s["bias"], case)
        return [ids, w, None, None, None]
    if op == "combine":
        y = s["residual"].double() if s["residual"] is not None else torch.zeros(s["y"].shape, dtype=torch.float64, device="cuda")
        for j in range(case["top_k"]):
            at = s["positions"][:, j].long()
            live = torch.nonzero(at >= 0)[:, 0]
            y[live] += s["weights"][live, j, None].double() * s["z"][at[live]].double()
        return y
    k = case["k"]
    if op == "act":
        y = _exact_layer(s["x"], _exact_values(s["codes"], s["scales"], k), s["bias"], case)
        return y + s["residual"].double() if s["residual"] is not None else y
    y = torch.zeros(s["y"].shape, dtype=torch.float64, device="cuda")
    for e in range(case["experts"]):
        rows = torch.arange(int(s["offsets"][e]), int(s["offsets"][e + 1]), device="cuda")
        if len(rows):
            of = rows if case["sorted"] else torch.div(s["slots"][rows].long(), case["top_k"], rounding_mode="floor")
            y[rows] = _exact_layer(s["x"][of], _exact_values(s["codes"][e], s["scales"][e], k), None if s["bias"] is None else s["bias"][e], case)
    return y
