"""Plain 64-bit forms of the answers' operators (quantised rows, layers on codes, log probabilities and
their gradient), and how far an fp32 evaluation of them may be off.

Error terms are counted in half steps of fp32, U = 2^-24 relative to the value (a rounding is off by at most one),
from the formulas and from CUDA's documented bounds of its functions (in steps of 2 U): expf 2, logf 1, tanhf 2,
erfcf 4, ex2.approx 2."""
import math

import numpy as np

U = 2.0 ** -24
HALF_STEP = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}
TINY = {"float32": 2.0 ** -149, "float16": 2.0 ** -24, "bfloat16": 2.0 ** -133}


def quantize(x):
    """x: [rows, cols] float64 holding values of the input type."""
    with np.errstate(invalid="ignore", over="ignore"):
        top = np.abs(x).max(axis=1).astype(np.float32)
        bad = ~np.isfinite(x).all(axis=1)
        scale = np.where(bad, np.float32(np.nan), top / np.float32(127.0)).astype(np.float32)
        ok = scale > 0
        q = np.rint(np.where(ok[:, None], x / np.where(ok, scale, 1.0).astype(np.float64)[:, None],
                             0.0))
    return np.clip(q, -127, 127).astype(np.int8), scale


def _erfc(z):
    try:
        import torch
        return torch.erfc(torch.from_numpy(np.ascontiguousarray(z))).numpy()
    except ImportError:
        return np.vectorize(math.erfc)(z)


def act(name, z, g):
    """The transfer function, and its largest slope."""
    if name == "tanh":
        return np.tanh(z), 1.0
    if name == "sigmoid":
        return 1.0 / (1.0 + np.exp(-z)), 0.25
    if name == "relu":
        return np.maximum(z, 0.0), 1.0
    if name == "gaussian":
        return np.exp(-g * z * z), math.sqrt(2.0 * g / math.e)
    if name == "gelu":
        return 0.5 * z * _erfc(-z / math.sqrt(2.0)), 1.13
    return z, 1.0


def code_linear(xq, xs, wq, ws, bias, name, g, dtype):
    """(y, how far an output may be off)."""
    return code_fields(xq.astype(np.int64) @ wq.astype(np.int64).T, xs, ws, bias, name, g, dtype)


def code_fields(s, xs, ws, bias, name, g, dtype):
    """The same from the integer sums."""
    z0 = s.astype(np.float64) * xs.astype(np.float64)[:, None] * ws.astype(np.float64)
    z = z0 if bias is None else z0 + bias.astype(np.float64)
    # the sum to fp32, two products, one addition
    dz = 3.01 * U * np.abs(z0) + (0 if bias is None else 1.01 * U * np.abs(z))
    y, slope = act(name, z, g)
    own = {"identity": 0.0, "relu": 0.0, "tanh": 4.0,
           # expf, the addition and the quotient
           "sigmoid": 4.0 + 1.0 + 1.0,
           # erfcf 8, its argument's product and constant: |z erfc'/erfc| <= z^2 + 1 each, two products
           "gelu": 8.0 + 2.0 + 2.0 * (np.minimum(z * z, 200.0) + 1.0),
           # expf, the argument's two products: relative to the argument
           "gaussian": 4.0 + 2.0 * np.abs(g) * z * z}[name]
    tol = slope * dz + 1.01 * own * U * np.abs(y)
    return y, tol + HALF_STEP[dtype] * (np.abs(y) + tol) * (0 if dtype == "float32" else 1) + \
        TINY[dtype]


def logprobs(x, targets, top):
    """x: [rows, vocab] float64. Returns a dict, with 'tol' per row for lse, logprob, entropy."""
    rows, vocab = x.shape
    r = {k: np.zeros(rows) for k in ("logprob", "entropy", "lse", "tol_lse", "tol_logprob",
                                     "tol_entropy")}
    r["top_logprob"] = np.full((rows, top), -np.inf)
    r["top_index"] = np.full((rows, top), -1, np.int64)
    # additions that a sum's term goes through: a thread's share of the row, then the threads'
    n_add = vocab / 256 + 64
    for i in range(rows):
        v = x[i]
        t = int(targets[i])
        if not (v < np.inf).all():
            r["lse"][i] = r["entropy"][i] = np.nan
            r["logprob"][i] = 0.0 if t == -1 else np.nan
            r["top_logprob"][i] = np.nan
            continue
        m = v.max()
        if m == -np.inf:
            r["lse"][i] = -np.inf
            r["logprob"][i] = 0.0 if t == -1 else np.nan if not 0 <= t < vocab else -np.inf
            continue
        live = v > -np.inf
        d = v[live] - m
        e = np.exp(d)
        s = e.sum()
        ls = math.log(s)
        p = e / s
        r["lse"][i] = m + ls
        r["entropy"][i] = ls - (p * d).sum()
        # a term: the difference and its product with log2 e, each U |d| in the exponent, ex2 4 U (and a
        # changed maximum's rescaling the same once more)
        term = 2 * (2.0 * np.abs(d) + 4.0) + n_add
        rel_s = (p * term).sum() * U
        r["tol_lse"][i] = 1.01 * (rel_s + 3 * U * abs(ls) + U * abs(m + ls))
        at = 0.0 if t == -1 else v[t] - m if 0 <= t < vocab else np.nan
        r["logprob"][i] = 0.0 if t == -1 else at - ls
        fin = at if np.isfinite(at) else 0.0
        r["tol_logprob"][i] = 1.01 * (rel_s + 3 * U * abs(ls) + U * abs(fin) + U * abs(fin - ls))
        # sum e d / s: the terms' errors times |d|, one more rounding each, the quotient
        r["tol_entropy"][i] = 1.01 * (rel_s + 3 * U * abs(ls) +
                                      ((p * np.abs(d)) * (term + 4.0)).sum() * U +
                                      (p * np.abs(d)).sum() * rel_s + U * abs(r["entropy"][i]))
        k = min(top, int(live.sum()))
        order = np.lexsort((np.arange(vocab), -v))[:k]
        r["top_index"][i, :k] = order
        r["top_logprob"][i, :k] = (v[order] - m) - ls
    return r


def backward(x, targets, lse, entropy, gl, ge, dtype):
    """(gradient, how far an element may be off)."""
    rows, vocab = x.shape
    out, tol = np.zeros_like(x), np.zeros_like(x)
    for i in range(rows):
        if lse[i] == -np.inf:
            continue
        t = -1 if gl is None else int(targets[i])
        g = 0.0 if t == -1 else float(gl[i])
        if not -1 <= t < vocab or np.isnan(lse[i]):
            out[i] = np.nan
            continue
        h = 0.0 if ge is None else float(ge[i])
        H = 0.0 if ge is None else float(entropy[i])
        with np.errstate(invalid="ignore"):
            lp = x[i] - float(lse[i])
            p = np.exp(lp)
            lz = np.where(p > 0, lp, 0.0)
        c = g + h * (lz + H)
        out[i] = -p * c
        rel_p = (2.0 * np.abs(lz) + 4.0) * U          # difference, product, ex2
        # the difference again, + H, product with g_entropy, + g_logprob, product with p
        dc = U * (abs(h) * (np.abs(lz) + 2 * np.abs(lz + H)) + np.abs(c) + abs(g))
        tol[i] = p * (np.abs(c) * (rel_p + 2 * U) + 1.01 * dc)
        if t >= 0:
            out[i, t] += g
            tol[i, t] += U * abs(out[i, t])
    tol = 1.01 * tol
    return out, tol + HALF_STEP[dtype] * (np.abs(out) + tol) + TINY[dtype] + 2.0 ** -125
