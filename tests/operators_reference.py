"""Plain 64-bit forms of the operators on four-bit matrices and routed experts (numpy, from their definitions)."""
import math

import numpy as np

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}      # half a step, relative to the value


def blocks(n):
    return (n + 31) // 32


def quantise(x):
    """x [..., n] (float64 holding values of the source type) -> codes [..., 16 blocks], scale bytes [..., blocks]."""
    n, nb = x.shape[-1], blocks(x.shape[-1])
    v = np.zeros(x.shape[:-1] + (32 * nb,))
    v[..., :n] = x
    v = v.reshape(x.shape[:-1] + (nb, 32))
    bad = ~np.isfinite(v).all(-1)
    v = np.where(bad[..., None], 0.0, v)
    top = np.abs(v).max(-1)
    shift = np.where(top > 0, np.frexp(top)[1] - 3, -127)
    shift = np.maximum(shift, -127)
    q = v / 2.0 ** shift[..., None]
    # the nearest of the eight values; of two equally near ones the one with the even code
    a = np.minimum(np.abs(q), 6.0)
    d = np.abs(a[..., None] - GRID)
    order = np.array([0, 2, 4, 6, 1, 3, 5, 7])
    code = order[np.argmin(d[..., order], -1)]
    code = (code + 8 * np.signbit(v)).astype(np.uint8)
    code[bad] = 0
    scale = np.where(bad, 255, shift + 127).astype(np.uint8)
    code = code.reshape(x.shape[:-1] + (32 * nb,))
    return code[..., 0::2] | (code[..., 1::2] << 4), scale


def values(codes, scales, n):
    code = np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[:-1] + (-1,))
    v = np.where(code >= 8, -1.0, 1.0) * GRID[code & 7]
    s = np.where(scales == 255, math.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return (v.reshape(scales.shape + (32,)) * s[..., None]).reshape(codes.shape[:-1] + (-1,))[..., :n]


_erf = np.vectorize(math.erf, otypes=[np.float64])


def act(v, name):
    if name == "relu":
        return np.maximum(v, 0)
    return 0.5 * v * (1 + _erf(v / math.sqrt(2))) if name == "gelu" else v


SLOPE = {"none": 1.0, "relu": 1.0, "gelu": 1.13}       # the steepest of each activation
ACT_ERR = {"none": 0.0, "relu": 0.0, "gelu": 2e-6}    # of the kernels' own, absolute and relative: the error function in single precision


def product(a, w, bias, name, kind):
    """act(a w^T + bias), and how far a result in single precision, rounded once to `kind`, may be from it: K additions that each are
    off by a step (2^-23) of at most the sum of the magnitudes, the activation, half a step of the result."""
    s = a @ w.T + (0 if bias is None else bias)
    size = np.abs(a) @ np.abs(w).T + (0 if bias is None else np.abs(bias))
    y = act(s, name)
    acc = (a.shape[1] + 2) * 2.0 ** -23 * size * SLOPE[name] + ACT_ERR[name] * (1 + np.abs(y))
    return y, acc + HALF[kind] * (np.abs(y) + acc) + 2.0 ** -126


def leaves(x, w1, b1, w2, b2, idx, weight, name):
    """The mixture of leaf networks and its tolerance: the hidden sums as in `product`, each hidden value rounded to bf16 (and
    scaled before it), then a sum over width, the mixture over k in single precision, half a step of bf16."""
    T, O = x.shape[0], w2.shape[1]
    y, tol = np.zeros((T, O)), np.zeros((T, O))
    for e in np.unique(idx):
        if e < 0 or e >= len(w1):
            continue
        t, i = np.nonzero(idx == e)
        h, he = product(x[t], w1[e], b1[e], name, "bf16")
        g = np.ones((len(t), 1)) if weight is None else weight[t, i][:, None]
        size = np.abs(h) @ np.abs(w2[e]).T + np.abs(b2[e])
        np.add.at(y, t, g * (h @ w2[e].T + b2[e]))
        np.add.at(tol, t, np.abs(g) * ((he + 2.0 ** -23 * np.abs(h)) @ np.abs(w2[e]).T + (w2.shape[2] * idx.shape[1] + 4) * 2.0 ** -23 * size))
    return y, tol + HALF["bf16"] * (np.abs(y) + tol) + 2.0 ** -126


def route(logits, k, mask=None, normalise=True):
    """idx, weight, count (tokens last), prob_mean, loss, and p, lse, on of the rows."""
    l = np.where(np.isnan(logits), -np.inf, logits.astype(np.float64))
    T, E = l.shape
    on = (np.ones(T, bool) if mask is None else mask.astype(bool)) & (l.max(1, initial=-np.inf) > -np.inf)
    order = np.argsort(-l, axis=1, kind="stable")[:, :k]
    found = (np.take_along_axis(l, order, 1) > -np.inf) & on[:, None]
    idx = np.where(found, order, -1).astype(np.int32)
    m = np.where(on, l.max(1, initial=-np.inf), 0.0)
    with np.errstate(invalid="ignore", over="ignore"):
        p = np.where(np.isinf(m)[:, None] & (m > 0)[:, None], (l == np.inf) * 1.0, np.exp(l - m[:, None]))
    p = np.where(on[:, None], p, 0.0)
    s = p.sum(1)
    lse = np.where(on, m + np.log(np.where(s > 0, s, 1)), 0.0)
    p = p / np.where(s > 0, s, 1)[:, None]
    w = np.where(found, np.take_along_axis(p, np.maximum(idx, 0), 1), 0.0)
    if normalise:
        w = w / np.where(w.sum(1) > 0, w.sum(1), 1)[:, None]
    n = int(on.sum())
    count = np.bincount(idx[idx >= 0], minlength=E)
    mean = p.sum(0) / max(n, 1)
    loss = np.array([E * (count / (max(n, 1) * k) * mean).sum(), (lse ** 2).sum() / max(n, 1)])
    return idx, w, np.append(count, n), mean, loss, p, lse, on


def route_backward(logits, idx, count, dweight, dloss, mask=None, normalise=True):
    """dlogits, and the sum of the magnitudes of the terms of each."""
    k = idx.shape[1]
    _, _, _, _, _, p, lse, on = route(logits, 1, mask)
    T, E = p.shape
    n = int(count[E])
    pull = np.zeros(E) if dloss is None or n == 0 else dloss[0] * E * count[:E] / (n * k) / n
    zz = np.zeros(T) if dloss is None or n == 0 else 2 * dloss[1] * lse / n
    dot = (p * pull).sum(1, keepdims=True)
    d = p * (pull - dot + zz[:, None])
    size = p * (np.abs(pull) + (p * np.abs(pull)).sum(1, keepdims=True) + np.abs(zz)[:, None])
    if dweight is not None:
        good = (idx >= 0) & (idx < E) & on[:, None]
        at = np.where(good, idx, 0)
        q = np.where(good, np.take_along_axis(p, at, 1), 0.0)
        g = np.where(good, dweight, 0.0)
        total = np.where(q.sum(1) > 0, q.sum(1), 1)[:, None] if normalise else 1.0
        w = q / total
        mean, mean_size = (w * g).sum(1, keepdims=True), (w * np.abs(g)).sum(1, keepdims=True)
        rows = np.arange(T)[:, None].repeat(k, 1)
        if normalise:
            np.add.at(d, (rows, at), w * (g - mean))
            np.add.at(size, (rows, at), w * (np.abs(g) + mean_size))
        else:
            d -= p * mean
            size += p * mean_size
            np.add.at(d, (rows, at), w * g)
            np.add.at(size, (rows, at), w * np.abs(g))
    return d, size
