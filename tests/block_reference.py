"""The 8-bit block format, the choice of experts and their gradients in 64 bits (NumPy), written from the definitions."""
import numpy as np

BLOCK = 128
# every finite E4M3 number from 0 up, by its byte
LEVELS = np.array([(b & 7) / 8 * 2.0 ** -6 if b < 8 else (1 + (b & 7) / 8) * 2.0 ** ((b >> 3) - 7) for b in range(127)])


def e4m3(v):
    """Nearest E4M3 byte of values of at most 448 (or NaN), ties to the even byte."""
    a = np.abs(v)
    hi = np.clip(np.searchsorted(LEVELS, np.where(np.isnan(a), 0, a)), 1, 126)
    lo = hi - 1
    up = (a - LEVELS[lo] > LEVELS[hi] - a) | ((a - LEVELS[lo] == LEVELS[hi] - a) & (hi % 2 == 0))
    byte = np.where(up, hi, lo).astype(np.uint8)
    return np.where(np.isnan(v), 127, byte | (np.signbit(v).astype(np.uint8) << 7)).astype(np.uint8)


def value(q, scale, tile):
    """What bytes and exponent bytes stand for."""
    R, C = q.shape[-2:]
    v = np.where(q & 127 == 127, np.nan, LEVELS[np.minimum(q & 127, 126)]) * np.where(q & 128, -1.0, 1.0)
    e = scale.astype(int)[..., np.arange(R) // tile, :][..., np.arange(C) // BLOCK] - 127
    return v * 2.0 ** e


def quantise(x, tile):
    """(bytes, exponent bytes) of a matrix (or a stack of them)."""
    x = np.asarray(x, np.float64)
    R, C = x.shape[-2:]
    rb, cb = -(-R // tile), -(-C // BLOCK)
    pad = np.zeros((*x.shape[:-2], rb * tile, cb * BLOCK))
    pad[..., :R, :C] = x
    blocks = pad.reshape(*x.shape[:-2], rb, tile, cb, BLOCK)
    top = np.where(np.isfinite(blocks), np.abs(blocks), 0).max(axis=(-3, -1))
    e = np.zeros(top.shape, int)
    some = top > 0
    e[some] = np.ceil(np.log2(top[some] / 448)).astype(int)
    e[some & (448 * 2.0 ** (e - 1) >= top)] -= 1
    e[some & (448 * 2.0 ** e < top)] += 1
    e = np.where(some, np.clip(e, -126, 126), 0)
    with np.errstate(invalid="ignore"):
        scaled = np.where(np.isfinite(blocks), blocks, np.nan) * 2.0 ** -e[..., :, None, :, None]
    q = e4m3(scaled).reshape(pad.shape)[..., :R, :C]
    return q, (e + 127).astype(np.uint8)


def scores(logits, kind):
    x = np.minimum(np.asarray(logits, np.float64), 3.4028234663852886e38)
    seen = x > -np.inf                                   # (False for NaN)
    s = np.zeros_like(x)
    for t in range(x.shape[0]):
        v = seen[t]
        if not v.any():
            continue
        if kind == "softmax":
            p = np.exp(x[t, v] - x[t, v].max())
            s[t, v] = p / p.sum()
        else:
            with np.errstate(over="ignore"):
                s[t, v] = 1 / (1 + np.exp(-x[t, v]))
    return s, seen


def route(logits, k, kind, bias=None, groups=1, kept=1, renormalise=True, factor=1.0):
    """ids, weights, and the smallest distance between a choice's keys that decided it (ties and near ties cannot be compared)."""
    s, seen = scores(logits, kind)
    key = np.where(seen, s + (0 if bias is None else np.asarray(bias, np.float64)), -np.inf)
    key[np.isnan(key)] = -np.inf
    T, E = key.shape
    ids, w, gap = np.full((T, k), -1), np.zeros((T, k)), np.full(T, np.inf)
    for t in range(T):
        mine = key[t].copy()
        if groups > 1:
            value = np.full(groups, -np.inf)
            for g in range(groups):
                part = np.sort(mine[g * E // groups:(g + 1) * E // groups])[::-1][:2]
                if part[0] > -np.inf:
                    value[g] = part[part > -np.inf].sum()
            order = np.argsort(-value, kind="stable")
            if kept < groups and value[order[kept]] > -np.inf:
                gap[t] = value[order[kept - 1]] - value[order[kept]]
            for g in range(groups):
                if g not in order[:kept]:
                    mine[g * E // groups:(g + 1) * E // groups] = -np.inf
        order = np.argsort(-mine, kind="stable")
        best = mine[order]
        n = min(k, int((best > -np.inf).sum()))
        ids[t, :n] = order[:n]
        for j in range(n):
            # (equal logits without a bias are a tie on every machine: the lower index)
            if j + 1 < E and best[j + 1] > -np.inf and not (bias is None and logits[t, order[j]] == logits[t, order[j + 1]]):
                gap[t] = min(gap[t], best[j] - best[j + 1])
        w[t, :n] = s[t, order[:n]]
        if renormalise:
            w[t] = w[t] / w[t].sum() if w[t].sum() > 0 else 0
    return ids, w * factor, gap


def weights_of(logits, ids, kind, renormalise, factor):
    """The weights as a function of the logits for a given choice: what the gradient is taken of."""
    s, _ = scores(logits, kind)
    w = np.where((ids >= 0) & (ids < logits.shape[1]), np.take_along_axis(s, np.clip(ids, 0, logits.shape[1] - 1), 1), 0.0)
    if renormalise:
        total = w.sum(1, keepdims=True)
        w = np.divide(w, total, out=np.zeros_like(w), where=total > 0)
    return factor * w


def route_gradient(logits, ids, dw, kind, renormalise, factor):
    s, seen = scores(logits, kind)
    T, E = s.shape
    dx = np.zeros((T, E))
    for t in range(T):
        there = [j for j in range(ids.shape[1]) if 0 <= ids[t, j] < E]
        total = sum(s[t, ids[t, j]] for j in there)
        for j in there:
            e = ids[t, j]
            if not renormalise:
                g = factor * dw[t, j]
            elif total > 0:
                g = factor * sum(s[t, ids[t, i]] * (dw[t, j] - dw[t, i]) for i in there) / total ** 2
            else:
                g = 0.0
            # d s_e / d x_f = s_e (1[e = f] - s_f) for the softmax, s_e (1 - s_e) 1[e = f] for the sigmoid
            if kind == "softmax":
                dx[t] -= g * s[t, e] * s[t]
                dx[t, e] += g * s[t, e]
            else:
                dx[t, e] += g * s[t, e] * (1 - s[t, e])
    return np.where(seen, dx, 0.0)
