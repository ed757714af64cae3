"""The router's and the experts' arithmetic in 64 bits, from the definitions in include/hiermoe.h; numpy on the CPU."""
from __future__ import annotations

import numpy as np

NONE = -np.inf


def up(n, m):
    return (n + m - 1) // m * m


# ---- routing --------------------------------------------------------------------------------------------------------
def usable(x):
    """Logits as they count: never chosen ones as -inf, +inf as the largest finite number."""
    x = np.where(np.isnan(x), NONE, x.astype(np.float64))
    return np.minimum(x, float(np.finfo(np.float32).max))


def scores(x, kind):
    x = usable(x)
    if kind == "sigmoid":
        with np.errstate(over="ignore"):
            return np.where(x == NONE, 0.0, 1.0 / (1.0 + np.exp(-x)))
    best = x.max(axis=1, keepdims=True)
    e = np.where(x == NONE, 0.0, np.exp(np.where(x == NONE, 0.0, x - np.where(best == NONE, 0.0, best))))
    return e / np.maximum(e.sum(axis=1, keepdims=True), 1e-300)


def choose(choice, group_choice, K, groups, top_groups, group_best):
    """(ids, the smallest gap between two unequal numbers that decided)."""
    T, E = choice.shape
    ids, gap, per = np.full((T, K), -1, dtype=np.int64), np.inf, E // groups
    for t in range(T):
        c = choice[t].copy()
        if groups > 1:
            total = np.full(groups, NONE)
            for g in range(groups):
                v = np.sort(group_choice[t, g * per:(g + 1) * per][c[g * per:(g + 1) * per] > NONE])[::-1]
                if len(v):
                    total[g] = v[:group_best].sum()
            order = np.argsort(-total, kind="stable")
            if top_groups < groups:
                a, b = total[order[top_groups - 1]], total[order[top_groups]]
                if a > b > NONE:
                    gap = min(gap, a - b)
            for g in order[top_groups:]:
                c[g * per:(g + 1) * per] = NONE
        order = np.argsort(-c, kind="stable")[:K + 1]
        v = c[order]
        for a, b in zip(v[:-1], v[1:]):
            if a > b > NONE:
                gap = min(gap, a - b)
        for k in range(K):
            if v[k] > NONE:
                ids[t, k] = order[k]
    return ids, gap


def route(x, bias, K, kind, groups=1, top_groups=1, group_best=1, renormalise=True, scale=1.0):
    """ids, weights, gap."""
    s, u = scores(x, kind), usable(x)
    c = u if bias is None else np.where(u == NONE, NONE, s + bias.astype(np.float64))
    ids, gap = choose(c, s if bias is None else c, K, groups, top_groups, group_best)
    w = np.where(ids >= 0, np.take_along_axis(s, np.maximum(ids, 0), axis=1), 0.0)
    if renormalise:
        total = w.sum(axis=1, keepdims=True)
        w = np.where(total > 0, w / np.where(total > 0, total, 1.0), 0.0)
    return ids, scale * w, gap


def weights_of(x, ids, kind, renormalise, scale):
    """The weights as a function of finite logits with the choice held fixed (ids of -1: no slot)."""
    s = scores(x, kind)
    w = np.where(ids >= 0, np.take_along_axis(s, np.maximum(ids, 0), axis=1), 0.0)
    return scale * (w / w.sum(axis=1, keepdims=True) if renormalise else w)


def route_backward(x, ids, g, kind, renormalise, scale):
    """(gradient, bound of its terms' magnitude)."""
    T, E = x.shape
    s = scores(x, kind)
    there = (ids >= 0) & (ids < E)
    at = np.where(there, ids, 0)
    there &= np.take_along_axis(usable(x), at, axis=1) > NONE
    g = np.where(there, g.astype(np.float64), 0.0)
    p = np.where(there, np.take_along_axis(s, at, axis=1), 0.0)
    total = p.sum(axis=1, keepdims=True) if renormalise else np.ones((T, 1))
    total = np.where(total > 0, total, 1.0)
    mean, size = (g * p).sum(axis=1, keepdims=True) / total, (np.abs(g) * p).sum(axis=1, keepdims=True) / total
    dp, bound = ((g - mean) / total, (np.abs(g) + size) / total) if renormalise else (g, np.abs(g))
    slope = p * (1.0 - p) if kind == "sigmoid" else p
    if kind == "sigmoid":   # 1 - s without cancellation
        u = np.take_along_axis(usable(x), at, axis=1)
        with np.errstate(over="ignore"):
            slope = np.where(there, p / (1.0 + np.exp(u)), 0.0)
    dx, size_x = np.zeros((T, E)), np.zeros((T, E))
    for t in range(T):
        np.add.at(dx[t], at[t][there[t]], (scale * dp * slope)[t][there[t]])
        np.add.at(size_x[t], at[t][there[t]], (scale * bound * slope)[t][there[t]])
    if kind == "softmax" and not renormalise:
        dx -= scale * s * (g * p).sum(axis=1, keepdims=True)
        size_x += scale * s * (np.abs(g) * p).sum(axis=1, keepdims=True)
    return dx, size_x


# ---- 8 bits ---------------------------------------------------------------------------------------------------------
def code_of(amax):
    """Least exponent e >= -127 with amax <= 448 * 2^e, + 127; any shape."""
    m, e = np.frexp(amax.astype(np.float64))
    return np.where(amax > 0, np.maximum(np.where(m <= 0.875, e - 9, e - 8), -127), -127) + 127


def e4m3(v):
    """Nearest e4m3 value, ties to even, of |v| <= 448; NaN stays."""
    step = np.ldexp(1.0, np.maximum(np.frexp(np.abs(np.where(np.isfinite(v), v, 1.0)))[1] - 1, -6) - 3)
    return np.where(np.isfinite(v), np.rint(v / step) * step, np.nan)


def in_blocks(x, axes):
    """Values in 8 bits (as numbers) and codes, a block being the given axes."""
    x = x.astype(np.float64)
    code = code_of(np.where(np.isfinite(x), np.abs(x), 0.0).max(axis=axes, keepdims=True))
    return e4m3(np.where(np.isfinite(x), x, np.nan) * np.ldexp(1.0, 127 - code)), code


def rows8(x):
    R, C = x.shape
    v = np.zeros((R, up(C, 128)))
    v[:, :C] = x
    q, code = in_blocks(v.reshape(R, -1, 128), 2)
    out = np.zeros((R, up(C, 512) // 128), dtype=np.int64)
    out[:, :code.shape[1]] = code[:, :, 0]
    return q.reshape(R, -1), out


def columns8(x, offsets):
    """(values, codes, which blocks belong to a segment)."""
    R, C = x.shape
    S = len(offsets) - 1
    B = R // 128 + S
    q, out, there = np.zeros((C, 128 * B)), np.zeros((B, C), dtype=np.int64), np.zeros(B, dtype=bool)
    for e in range(S):
        for i, r in enumerate(range(offsets[e], offsets[e + 1], 128)):
            b = offsets[e] // 128 + e + i
            assert not there[b]
            there[b] = True
            part = x[r:min(r + 128, offsets[e + 1])]
            v, code = in_blocks(part, 0)
            q[:, 128 * b:128 * b + len(part)] = v.T
            out[b] = code[0]
    return q, out, there


def weights8(w):
    E, N, C = w.shape
    v = np.zeros((E, up(N, 128), up(C, 128)))
    v[:, :N, :C] = w
    q, code = in_blocks(v.reshape(E, v.shape[1] // 128, 128, v.shape[2] // 128, 128), (2, 4))
    q = q.reshape(v.shape)
    code = code[:, :, 0, :, 0]

    def codes(c, cols):
        out = np.zeros(c.shape[:2] + (up(cols, 512) // 128,), dtype=np.int64)
        out[:, :, :c.shape[2]] = c
        return out
    return q[:, :N], codes(code, C), np.swapaxes(q, 1, 2)[:, :C], codes(np.swapaxes(code, 1, 2), N)


def row_values(q, code):
    R, W = q.shape
    return (q.reshape(R, -1, 128) * np.ldexp(1.0, code[:, :W // 128, None] - 127)).reshape(R, W)


def column_values(q, code):
    """[place, column]."""
    return (q.reshape(q.shape[0], -1, 128) * np.ldexp(1.0, code.T[:, :, None] - 127)).reshape(q.shape).T


def weight_values(q, code):
    E, N, W = q.shape
    s = np.ldexp(1.0, code[:, :, :W // 128] - 127)
    return q * np.repeat(np.repeat(s, 128, axis=1)[:, :N], 128, axis=2)


def product(a, b, steps):
    """a b^T, the sum of the magnitudes, and for every block of 128 the largest product, added up."""
    size, largest = np.zeros((len(a), len(b))), np.zeros((len(a), len(b)))
    for k in range(steps):
        p = np.abs(a[:, None, 128 * k:128 * k + 128]) * np.abs(b[None, :, 128 * k:128 * k + 128])
        size += p.sum(axis=2)
        largest += p.max(axis=2, initial=0.0)
    return a @ b.T, size, largest
