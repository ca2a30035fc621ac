"""Plain references of the decoder layer's operators, in numpy's 64 bits, from their definitions in include/ifq.h."""
import math

import numpy as np

ACTS = {"silu": 1, "gelu": 2, "gelu_tanh": 3}


def round_to(x, dtype):
    """float64 -> the nearest value of "f16", "bf16" or "f32" (ties to even), in float64"""
    x = np.asarray(x, np.float64)
    with np.errstate(all="ignore"):
        if dtype == "f16":
            return x.astype(np.float16).astype(np.float64)
        if dtype == "f32":
            return x.astype(np.float32).astype(np.float64)
        _, e = np.frexp(np.where(np.isfinite(x), x, 0.0))
        step = np.ldexp(1.0, np.maximum(e, -125) - 8)
        y = np.where(np.isfinite(x), np.rint(x / step) * step, x)
        return np.where(np.abs(y) >= 2.0 ** 128, np.copysign(np.inf, y), y)


def half_step(dtype):
    """how far one rounding may be off, relative to the value"""
    return {"f16": 2.0 ** -11, "bf16": 2.0 ** -8, "f32": 2.0 ** -24}[dtype]


def weights(codes, scales, mins, group, dtype):
    """codes uint8 [rows][k / 2], scales and mins float64 [rows][groups] -> float64 [rows][k]"""
    rows, half = codes.shape
    c = np.empty((rows, 2 * half))
    c[:, 0::2], c[:, 1::2] = codes & 15, codes >> 4
    at = np.arange(2 * half) // group
    with np.errstate(all="ignore"):
        return round_to(c * scales[:, at] + mins[:, at], dtype)


def act(name, a):
    if name == "silu":
        return a / (1 + np.exp(-a))
    if name == "gelu":
        return 0.5 * a * np.vectorize(math.erfc)(-a / math.sqrt(2))
    with np.errstate(over="ignore"):   # 1 + tanh u = 2 / (1 + e^-2u), which does not cancel
        return a / (1 + np.exp(-2 * math.sqrt(2 / math.pi) * (a + 0.044715 * a ** 3)))


def products(x, w, truncated=True):
    """x w^T and how far sums in single precision may be off: 2^-24 of the terms' absolute sum for each addition, twice
    that where the sums may truncate."""
    y, t = x @ w.T, np.abs(x) @ np.abs(w).T
    return y, (x.shape[1] + 16) * (2.0 ** -23 if truncated else 2.0 ** -24) * t


def gated(x, wg, wu, name, dtype):
    """act(x wg^T) (x wu^T) and its tolerance: the two sums' (an activation's slope is at most 1.13), 2^-18 of the
    result for the single-precision activation (a few roundings and exponentials of arguments up to 88, whose
    rounding moves e^-a by 88 2^-24), and the rounding."""
    a, da = products(x, wg)
    b, db = products(x, wu)
    with np.errstate(over="ignore"):
        y = act(name, a) * b
    return y, 1.13 * da * (np.abs(b) + db) + np.abs(act(name, a)) * db + (2.0 ** -18 + half_step(dtype)) * np.abs(y) + 1e-37


def rms_norm(x, residual, weight, eps, dtype):
    """float64 inputs that are values of dtype -> (out, sum); sum is exact to its one rounding (in single precision first)"""
    h = x if residual is None else round_to(round_to(x + residual, "f32"), dtype)
    r = np.sqrt(np.mean(h * h, -1, keepdims=True) + eps)
    with np.errstate(all="ignore"):
        return h / r * weight, h


def scores(logits, tokens, scale, top):
    """float64 logits [rows][vocab] -> dict of logprobs, lse, entropy, top_ids, top_logprobs"""
    out = {"logprobs": [], "lse": [], "entropy": [], "top_ids": [], "top_logprobs": []}
    for row, token in zip(logits, tokens):
        z = row * scale
        m = z.max() if len(z) else -np.inf
        with np.errstate(all="ignore"):
            if m == -np.inf:
                lse, ent, lp = -np.inf, 0.0, np.full(len(z), -np.inf)
            else:
                e = np.exp(z - m)
                lse = m + np.log(e.sum()) if np.isfinite(m) else m
                lp = z - m - np.log(e.sum()) if np.isfinite(m) else z - m   # (not z - lse: a large m swallows the logarithm)
                ent = -np.sum(np.where(e > 0, e / e.sum() * lp, e))
        key = np.where(np.isnan(row), np.inf, row)
        order = np.lexsort((np.arange(len(z)), -key, ~np.isnan(row)))[:top]
        out["lse"].append(lse)
        out["entropy"].append(ent)
        out["logprobs"].append(0.0 if token < 0 else np.nan if token >= len(z) else lp[token])
        out["top_ids"].append(order)
        out["top_logprobs"].append(lp[order])
    return {k: np.array(v) for k, v in out.items()}


def scores_tolerance(logits, scale):
    """[rows]: z and the differences from the largest are rounded (2^-24 of |z| each); an exponential is off by 2^-22 and the
    rounding of its argument, weighted by p, at most 16 2^-24; sums of single precision by 2^-24 a step of a chain, of which
    a row's split over at least 256 threads has vocab / 256 + 16."""
    z = np.where(np.isfinite(logits), np.abs(logits) * scale, 0.0)
    return 2.0 ** -22 * (8 + z.max(-1)) + (logits.shape[1] / 256 + 32) * 2.0 ** -24
