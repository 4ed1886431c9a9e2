"""8-bit integers, the layer norm, the balance of experts and the gradients' norm in 64 bits (NumPy), written from the definitions; and what their fp32
forms may be off by: U is half a step of fp32, the most that one rounding changes a number by relative to it."""
import numpy as np

U = 2.0 ** -24
# half a step of each type, and of its subnormal numbers
HALF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -150, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}


def rounding(want, dtype):
    """What the rounding of values near `want` to a type changes them by, at most."""
    return HALF[dtype] * np.abs(want) + TINY[dtype]


def quantise(x):
    """(q int64, scale as fp32 numbers in fp64) of rows."""
    x = np.asarray(x, np.float64)
    top = np.abs(x).max(axis=1, initial=0.0)
    bad = ~np.isfinite(x).all(axis=1)
    with np.errstate(invalid="ignore", over="ignore"):
        scale = (top / 127).astype(np.float32).astype(np.float64)
    scale = np.where(top == 0, 1.0, np.maximum(scale, 2.0 ** -126))
    scale[bad] = np.nan
    # (a quotient of numbers of 24 digits that is not k + 1/2 is further from it than fp64 rounds)
    q = np.rint(np.where(bad[:, None], 0.0, x) / np.where(bad, 1.0, scale)[:, None]).astype(np.int64)
    return q, scale


def product(qa, sa, qb, sb, bias=None):
    """out, and what fp32 scales and sums leave it off by."""
    s = (qa @ qb.T).astype(np.float64)
    v = s * sa[:, None] * sb[None, :]
    out = v if bias is None else v + bias
    return out, 3.01 * U * np.abs(v) + (0 if bias is None else 1.01 * U * np.abs(out)) + 2.0 ** -148


def norm(x, weight, bias, eps, depth):
    """y, mean, rstd and bounds of their errors; depth: additions on the way of one element to a sum over its row."""
    x = np.asarray(x, np.float64)
    n = x.shape[1]
    mean = x.mean(1, keepdims=True)
    d = x - mean
    v = (d * d).mean(1, keepdims=True)
    r = 1 / np.sqrt(v + eps)
    h = d * r
    w = np.ones(n) if weight is None else weight.astype(np.float64)
    b = np.zeros(n) if bias is None else bias.astype(np.float64)
    y = h * w + b
    e_mean = (depth + 2) * U * np.abs(x).mean(1, keepdims=True)
    # d is off by e_mean and its own rounding; an offset of all d's adds its square to the variance, the roundings' squares likewise
    e_v = (depth + 6) * U * (v + e_mean ** 2) + 1.01 * e_mean ** 2 + 2 * U * v
    rel_r = 0.51 * e_v / (v + eps) + 4 * U
    e_h = 1.01 * ((e_mean + U * (np.abs(d) + e_mean)) * r + (np.abs(h) + e_mean * r) * (rel_r + U))
    e_y = 1.01 * (np.abs(w) * e_h + 2 * U * (np.abs(h) + e_h) * np.abs(w) + U * np.abs(y))
    return y, mean[:, 0], r[:, 0], e_y, e_mean[:, 0], (rel_r * r)[:, 0] * 1.01


def norm_gradient(g, x, mean, rstd, weight, depth, row_depth):
    """dx, dweight, dbias from the given statistics, and bounds of their errors; row_depth: additions on the way of a row to the sums over rows."""
    g, x, mean, rstd = (np.asarray(t, np.float64) for t in (g, x, mean, rstd))
    n = x.shape[1]
    w = np.ones(n) if weight is None else weight.astype(np.float64)
    r = rstd[:, None]
    h = (x - mean[:, None]) * r
    u = g * w
    su, suh = u.mean(1, keepdims=True), (u * h).mean(1, keepdims=True)
    dx = r * (u - su - h * suh)
    e_su = (depth + 3) * U * np.abs(u).mean(1, keepdims=True)
    e_suh = (depth + 7) * U * np.abs(u * h).mean(1, keepdims=True)
    parts = np.abs(u) + np.abs(su) + np.abs(h * suh)
    e_dx = 1.01 * np.abs(r) * (U * np.abs(u) + e_su + np.abs(h) * e_suh + 2 * U * np.abs(h * suh) + 4 * U * parts)
    dweight, dbias = (g * h).sum(0), g.sum(0)
    e_w, e_b = 1.01 * (row_depth + 4) * U * np.abs(g * h).sum(0), 1.01 * row_depth * U * np.abs(g).sum(0)
    return dx, dweight, dbias, e_dx, e_w, e_b


def scores(logits, kind):
    """(scores, where a logit counts, relative bound of a score of the fp32 form)."""
    x = np.minimum(np.asarray(logits, np.float64), 3.4028234663852886e38)
    seen = x > -np.inf                                   # (False for NaN)
    with np.errstate(over="ignore", invalid="ignore"):
        if kind == "softmax":
            top = np.where(seen, x, -3.4e38).max(1, keepdims=True)
            off = np.where(seen, x - top, 0.0)
            # an exponential is off by 2 steps at most, its argument by one rounding
            return np.where(seen, np.exp(off), 0.0), seen, U * (np.minimum(np.abs(off), 110.0) + 5)
        return np.where(seen, 1 / (1 + np.exp(-x)), 0.0), seen, np.full(x.shape, 8 * U)


def balance(logits, ids, kind, factor):
    """loss, counts, push, p, and p's relative bound (without that of its sum's order)."""
    s, seen, rel = scores(logits, kind)
    T, E = s.shape
    total = s.sum(1, keepdims=True)
    p = np.divide(s, total, out=np.zeros_like(s), where=total > 0)
    chosen = ids[(ids >= 0) & (ids < E)]
    counts = np.bincount(chosen.ravel(), minlength=E)
    n, live = counts.sum(), int((total > 0).sum())
    push = factor * E * counts / (n * live) if n and live else np.zeros(E)
    return float((push * p.sum(0)).sum()), counts, push, p, s, seen, rel


def balance_gradient(p, s, seen, push, kind):
    d = p * (push - (p * push).sum(1, keepdims=True))
    return np.where(seen, d if kind == "softmax" else d * (1 - s), 0.0)
