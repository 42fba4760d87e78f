"""Float64 oracle of what stands beside the pruned products: low-rank adapters,
their gradients, the gradient of the pruned product with respect to its input,
and the norm and rotation of heads. Loops over tokens, adapters and heads;
shares no code with the library. Test infrastructure only.

Where a function also returns a bound, it holds for fp32 sums in any order: a
sum of n products has an error of at most 2 n 2^-24 times the sum of their
magnitudes (twice the half-step of a rounding per addition, for accumulators
that truncate).
"""

from __future__ import annotations

import numpy as np

U32 = 2.0 ** -24  # half a step of fp32, relative
SPLIT = 2.0 ** -21  # two fp16 in the place of an fp32: 22 bits, and the scaled product's own rounding
TINY = 2.0 ** -36  # ... and what the second one's last bit is of the largest


def half_step(y):
    """Half a step of fp16 at y: relative 2^-11, absolute 2^-25 below 2^-14;
    past the largest number (65504) a rounding may give infinity."""
    y = np.abs(y)
    return np.where(y > 65504.0, np.inf, np.maximum(2.0 ** -11 * y, 2.0 ** -25))


def adapters_of(ids, n, count):
    """Each token's adapter, -1 for none."""
    if ids is None:
        return np.zeros(n, dtype=np.int64)
    i = np.asarray(ids, dtype=np.int64)
    return np.where((i >= 0) & (i < count), i, -1)


def _low_rank(x, ids, base, a, b, scale):
    x, a, b = (np.asarray(v, dtype=np.float64) for v in (x, a, b))
    base, scale = np.asarray(base, dtype=np.float64), np.asarray(scale, dtype=np.float64)
    count, rank, cols = a.shape
    y, h = base.copy(), np.zeros((x.shape[0], rank))
    y_err, h_err = np.zeros_like(y), np.zeros_like(h)
    for t, i in enumerate(adapters_of(ids, x.shape[0], count)):
        if i < 0:
            continue
        h[t] = a[i] @ x[t]
        h_err[t] = 2 * cols * U32 * (np.abs(a[i]) @ np.abs(x[t]))
        part = scale[i] * (h[t] @ b[i])
        y[t] += part
        size = np.abs(h[t]) + h_err[t]
        y_err[t] = abs(scale[i]) * ((h_err[t] + (SPLIT + 2 * (2 * rank + 2) * U32) * size + TINY * size.max()) @ np.abs(b[i])
                                    + 2 * U32 * np.abs(h[t] @ b[i]))
        y_err[t] += 2 * U32 * np.abs(y[t])
    return y, y_err, h, h_err


def adapt(x, ids, base, a, b, scale):
    """(y, bound on fp16 y's error, h, bound on h's): base + scale b (a x) of
    each token's own adapter; b is [count, rank, rows]."""
    y, e, h, he = _low_rank(x, ids, base, a, b, scale)
    return y, e + half_step(np.abs(y) + e), h, he


def adapt_grad(x, ids, h, dy, base, a, b, scale):
    """((dx, bound), (da, bound), (db, bound)) for dy."""
    x, h, dy = (np.asarray(v, dtype=np.float64) for v in (x, h, dy))
    dx, dx_err, u, u_err = _low_rank(dy, ids, base, b, a, scale)
    which = adapters_of(ids, x.shape[0], a.shape[0])
    out = [(dx, dx_err + half_step(np.abs(dx) + dx_err))]
    for act, err, z, like in ((u, u_err, x, a), (h, np.zeros_like(h), dy, b)):
        d, e = np.zeros(like.shape), np.zeros(like.shape)
        for i in range(like.shape[0]):
            at = np.flatnonzero(which == i)
            if at.size == 0:
                continue
            s = float(scale[i])
            d[i] = s * (act[at].T @ z[at])
            size = np.abs(act[at]) + err[at]
            e[i] = abs(s) * ((err[at] + (SPLIT + 2 * (2 * at.size + 2) * U32) * size + TINY * size.max()).T @ np.abs(z[at]))
            e[i] += 4 * U32 * np.abs(d[i]) + 2.0 ** -149
        out.append((d, e))
    return tuple(out)


def spmm_grad(w, dy):
    """(dy w, bound on the fp16 result's error) for w [rows, cols]."""
    w, dy = np.asarray(w, dtype=np.float64), np.asarray(dy, dtype=np.float64)
    dx = dy @ w
    e = 2 * w.shape[0] * U32 * (np.abs(dy) @ np.abs(w))
    return dx, e + half_step(np.abs(dx) + e)


def _turn(v, cos, sin, interleaved):
    """v [dim]: the leading 2 len(cos) numbers' pairs rotated."""
    out = v.copy()
    half = len(cos)
    for i in range(half):
        p, q = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        out[p] = v[p] * cos[i] - v[q] * sin[i]
        out[q] = v[q] * cos[i] + v[p] * sin[i]
    return out


def heads(x, dim, pos, cos, sin, weight, eps, interleaved, y):
    """(heads, bound): x [tokens, heads * dim]; padding tokens keep y's rows."""
    x = np.asarray(x, dtype=np.float64)
    out, err = np.asarray(y, dtype=np.float64).copy(), np.zeros(x.shape)
    w = None if weight is None else np.asarray(weight, dtype=np.float64)
    for t in range(x.shape[0]):
        if not 0 <= pos[t] < cos.shape[0]:
            continue
        c, s = cos[pos[t]].astype(np.float64), sin[pos[t]].astype(np.float64)
        for k in range(0, x.shape[1], dim):
            v = x[t, k:k + dim]
            n = v if w is None else v / np.sqrt((v * v).sum() / dim + eps) * w
            out[t, k:k + dim] = _turn(n, c, s, interleaved)
            size = _turn(np.abs(n), np.abs(c), -np.abs(s), interleaved)
            # sums of the pair, and the norm's squares, root, quotient and products
            size = np.maximum(size, _turn(np.abs(n), np.abs(c), np.abs(s), interleaved))
            err[t, k:k + dim] = (2 * dim + 12) * U32 * np.abs(size) if w is not None else 6 * U32 * np.abs(size)
    return out, err + np.where(err > 0, half_step(np.abs(out) + err), 0.0)


def heads_grad(x, dim, pos, cos, sin, dy, weight, eps, interleaved):
    """((dx, bound), (dweight, bound) or None)."""
    x, dy = np.asarray(x, dtype=np.float64), np.asarray(dy, dtype=np.float64)
    dx, err = np.zeros(x.shape), np.zeros(x.shape)
    dw, dw_err = np.zeros(dim), np.zeros(dim)
    w = None if weight is None else np.asarray(weight, dtype=np.float64)
    terms = 0
    for t in range(x.shape[0]):
        if not 0 <= pos[t] < cos.shape[0]:
            continue
        c, s = cos[pos[t]].astype(np.float64), sin[pos[t]].astype(np.float64)
        for k in range(0, x.shape[1], dim):
            v, d = x[t, k:k + dim], dy[t, k:k + dim]
            g = _turn(d, c, -s, interleaved)
            size = np.maximum(np.abs(_turn(np.abs(d), np.abs(c), np.abs(s), interleaved)),
                              np.abs(_turn(np.abs(d), np.abs(c), -np.abs(s), interleaved)))
            terms += 1
            if w is None:
                dx[t, k:k + dim], err[t, k:k + dim] = g, 6 * U32 * size
                continue
            r = 1.0 / np.sqrt((v * v).sum() / dim + eps)
            dx[t, k:k + dim] = r * (w * g - v * r * r * (w * g * v).sum() / dim)
            mag = r * (np.abs(w) * size + np.abs(v) * r * r * (np.abs(w) * size * np.abs(v)).sum() / dim)
            err[t, k:k + dim] = (8 * dim + 40) * U32 * mag
            dw += g * v * r
            dw_err += size * np.abs(v) * r
    dw_err *= (2 * terms + 2 * dim + 20) * U32
    return (dx, err + half_step(np.abs(dx) + err)), None if w is None else (dw, dw_err)
