"""The norm, the gated activation and the layer for a few tokens in 64 bits, from the definitions in include/hiermoe.h, with what
their fp32 arithmetic may be off; numpy on the CPU."""
from __future__ import annotations

import numpy as np

import layer_reference as R

U = 2.0 ** -24          # half a step of fp32, relative
HALF = {"bf16": 2.0 ** -8, "f32": U}   # of a rounded result
TINY = 1.2e-38          # the least normal number: below it steps are absolute


# ---- norm -----------------------------------------------------------------------------------------------------------
def rms_norm(s, w, eps):
    """(y, what fp32 may be off before the result is rounded).  A row's squares are added by a thread (up to 32), over 64 lanes (6)
    and up to 16 waves: half of 54 roundings in the root, three for mean, eps and root, one for the inverse, two products."""
    s, w = s.astype(np.float64), w.astype(np.float64)
    y = s / np.sqrt((s * s).mean(axis=1, keepdims=True) + eps) * w
    return y, 36 * U * np.abs(y)


def rms_norm_backward(gy, s, w, eps, gtotal, parts):
    """gx, gw and what they may be off.  The two sums of a row as above (60 roundings each); `parts`: rows of a part of gw."""
    gy, s, w = (t.astype(np.float64) for t in (gy, s, w))
    m = (s * s).mean(axis=1, keepdims=True) + eps
    u = gy * w
    mean, size = (u * s).mean(axis=1, keepdims=True), np.abs(u * s).mean(axis=1, keepdims=True)
    gx = (u - s * mean / m) / np.sqrt(m)
    off = 40 * U * np.abs(u) / np.sqrt(m) + np.abs(s) * m ** -1.5 * (80 * U * np.abs(mean) + 60 * U * size)
    if gtotal is not None:
        gx = gx + gtotal
        off = off + U * np.abs(gx)
    terms = gy * s / np.sqrt(m)
    rows = len(gy)
    return gx, off, terms.sum(axis=0), (rows / parts + parts / 16 + 16 + 40 + 1) * U * np.abs(terms).sum(axis=0)


# ---- gated activation -----------------------------------------------------------------------------------------------
def sigmoid(x):
    with np.errstate(over="ignore"):
        return np.where(x >= 0, 1.0 / (1.0 + np.exp(-np.abs(x))), np.exp(-np.abs(x)) / (1.0 + np.exp(-np.abs(x))))


def gated(h):
    """(a, what fp32 may be off): exp to two steps (4), the sum, the quotient, the product, and where exp(-gate) overflows a is 0."""
    F = h.shape[1] // 2
    gate, up = h[:, :F].astype(np.float64), h[:, F:].astype(np.float64)
    a = gate * sigmoid(gate) * up
    return a, 8 * U * np.abs(a) + (90 * TINY) * (1 + np.abs(up))


def gated_backward(h, ga):
    """(gradient of h, what fp32 may be off).  s is off by 7 roundings, 1 - s by as many of s; three products and the sum."""
    F = h.shape[1] // 2
    gate, up = h[:, :F].astype(np.float64), h[:, F:].astype(np.float64)
    ga = ga.astype(np.float64)
    s = sigmoid(gate)
    g = np.concatenate([ga * up * s * (1 + gate * sigmoid(-gate)), ga * gate * s], axis=1)
    off = np.concatenate([np.abs(ga * up) * s * (1 + np.abs(gate)) * 16 * U, 10 * U * np.abs(ga * gate * s)], axis=1)
    return g, off + 90 * TINY * (1 + np.abs(np.concatenate([ga * up, ga], axis=1)))


# ---- 8 bits ---------------------------------------------------------------------------------------------------------
def check_rows8(q, code, v, off):
    """Values in 8 bits (as numbers) and codes of rows v known to `off`: the code is that of a value within `off`, and every value is
    within a rounding (2^-4 of it, 2^-10 of the scale below the normal numbers) of one."""
    R_, C = v.shape
    W = R.up(C, 128)
    pad = lambda t: np.pad(t, ((0, 0), (0, W - C))).reshape(R_, W // 128, 128)
    v, off = pad(v), pad(off)
    code = code.astype(np.int64)
    assert not code[:, W // 128:].any() and not q[:, C:].any()
    code = code[:, :W // 128]
    low, high = R.code_of(np.maximum(np.abs(v) - off, 0).max(axis=2)), R.code_of((np.abs(v) + off).max(axis=2))
    assert ((code >= low) & (code <= high)).all()
    scale = np.ldexp(1.0, code - 127)[:, :, None]
    got = q.reshape(R_, W // 128, 128) * scale
    assert (np.abs(got - v) <= 2.0 ** -4 * (np.abs(v) + off) + 2.0 ** -10 * scale + off).all()


# ---- a layer for a few tokens ---------------------------------------------------------------------------------------
def layer_few(x, ids, weights, w13, w2, first, planes):
    """x [T,H], ids and weights [T,K], w13 [E,2F,H], w2 [E,H,F] as the numbers that 8 bits stand for; (out, what it may be off).

    A wave adds every fourth step of 128, four products of 32 a step: H / 128 sums and 32 inside a product, four waves.  The
    activation's derivative by gate is at most 1.1 |up|, by up silu.  Each plane of the activation leaves 2^-8 of what it rounds.
    The second product adds 4 `planes` a step, then K experts and 8 waves, the last two in parts."""
    x, weights = x.astype(np.float64), weights.astype(np.float64)
    T, K = ids.shape
    E, H, F = w2.shape
    out, off = np.zeros((T, H)), np.zeros((T, H))
    n1, n2 = H / 128 + 32 + 4 + 4, 4 * planes * (F / 128 + 1) + 32 + K + 16
    for t in range(T):
        for k in range(K):
            e = ids[t, k] - first
            if ids[t, k] < 0 or not 0 <= e < E:
                continue
            h, size = w13[e] @ x[t], np.abs(w13[e]) @ np.abs(x[t])
            gate, up, d = h[:F], h[F:], n1 * U * size
            a = gate * sigmoid(gate) * up
            da = 1.1 * (np.abs(up) + d[F:]) * d[:F] + np.abs(gate * sigmoid(gate)) * d[F:] + (8 * U + 2.0 ** (-8 * planes)) * np.abs(a)
            y, dy = w2[e] @ a, np.abs(w2[e]) @ da + n2 * U * (np.abs(w2[e]) @ np.abs(a))
            out[t] += weights[t, k] * y
            off[t] += np.abs(weights[t, k]) * (dy + 2 * U * np.abs(y))
    return out, off
