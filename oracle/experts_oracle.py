"""Plain NumPy oracle of the feed-forward layer's way out and of a layer of experts (include/aiq.h), in float64 and integers; shares no code
with the CUDA library."""
import math

import numpy as np

_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def activate(v, name):
    with np.errstate(over="ignore", invalid="ignore"):
        if name == "relu":
            return np.where(v < 0, 0.0, v)
        if name == "relu6":
            return np.where(v < 0, 0.0, np.where(v > 6, 6.0, v))
        if name == "silu":
            return v / (1.0 + np.exp(-v))
        if name == "gelu":
            return 0.5 * v * _erfc(-v / math.sqrt(2.0))
        if name == "gelu_tanh":
            return v / (1.0 + np.exp(-2.0 * math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3)))
    return v


def tail(v, name, gated, residual=None):
    """act(v), or act(first half) * second half, plus residual; v [M][N] with its bias."""
    half = v.shape[1] // 2
    y = activate(v[:, :half], name) * v[:, half:] if gated else activate(v, name)
    return y if residual is None else y + residual


def route(logits, bias, scoring, top_k, groups=1, top_groups=1, group_best=1, renormalise=True, scale=1.0):
    """(ids int32 [T][top_k], weights float64 [T][top_k]) by sorting, one token after the other."""
    logits = np.asarray(logits, np.float64)
    t, e = logits.shape
    ids, weights = np.full((t, top_k), -1, np.int32), np.zeros((t, top_k))
    b = np.zeros(e) if bias is None else np.asarray(bias, np.float64)
    size = e // groups
    for i, l in enumerate(logits):
        if np.isnan(l).any() or np.isnan(b).any() or (scoring == "softmax" and l.max() == np.inf):
            weights[i] = np.nan
            continue
        on = (l != -np.inf) & (b != -np.inf)
        if l.max() == -np.inf:
            continue
        with np.errstate(over="ignore"):
            p = 1.0 / (1.0 + np.exp(-l)) if scoring == "sigmoid" else np.exp(l - l.max()) / np.exp(l - l.max()).sum()
        choice = p + b
        order = l if bias is None else choice              # without a bias the choices' order is the logits', and so is that of a group's best
        if groups > 1:
            ranked = []
            for g in range(groups):
                best = sorted(((order if group_best == 1 else choice)[x] for x in range(g * size, (g + 1) * size) if on[x]), reverse=True)[:group_best]
                if best:
                    ranked.append((-sum(best), g))
            taken = [g for _, g in sorted(ranked)[:top_groups]]
            on = on & np.isin(np.arange(e) // size, taken)
        chosen = sorted(np.flatnonzero(on), key=lambda x: (-order[x], x))[:top_k]
        ids[i, :len(chosen)] = chosen
        if renormalise:
            w = (l[chosen] if scoring == "softmax" else np.minimum(l[chosen], 0) - np.log1p(np.exp(-np.abs(l[chosen]))))     # logarithms
            w = np.exp(w - w.max()) if len(chosen) else w
            weights[i, :len(chosen)] = w / w.sum() * scale if len(chosen) else 0.0
        else:
            weights[i, :len(chosen)] = p[chosen] * scale
    return ids, weights


def plan(ids, e):
    """(offsets, slots, positions) of ids [T][top_k]."""
    flat = ids.reshape(-1)
    slots = [i for x in range(e) for i in np.flatnonzero(flat == x)]
    offsets = np.concatenate(([0], np.cumsum([(flat == x).sum() for x in range(e)])))
    positions = np.full(flat.shape, -1, np.int32)
    positions[slots] = np.arange(len(slots))
    return offsets.astype(np.int32), np.array(slots + [-1] * (len(flat) - len(slots)), np.int32), positions.reshape(ids.shape)
