"""Plain 64-bit forms of the last stage's operators (MXFP4 rounding and products,
sampling, the walk of a drafted tree), on the CPU, for the tests."""
from __future__ import annotations

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = 32


def mx4_encode(x):
    """(codes [m, k] in 0..15, scale bytes [m, ceil(k / 32)]) of float64 rows."""
    x = np.asarray(x, np.float64)
    m, k = x.shape
    nb = -(-k // BLOCK)
    codes, scales = np.zeros((m, k), np.uint8), np.zeros((m, nb), np.uint8)
    for r in range(m):
        for b in range(nb):
            v = x[r, b * BLOCK:(b + 1) * BLOCK]
            if not np.isfinite(v).all():
                scales[r, b] = 255
                continue
            top = np.abs(v).max()
            if top == 0:
                codes[r, b * BLOCK:b * BLOCK + len(v)] = np.signbit(v) * 8
                continue
            e = max(int(np.frexp(top)[1]) - 1 - 2, -127)
            scales[r, b] = e + 127
            a = np.abs(v) / 2.0 ** e
            d = np.abs(a[:, None] - GRID[None])
            best = d.min(1)
            near = d == best[:, None]
            # of two equally near the even code; everything above 6 is nearest to 6
            even = near & (np.arange(8) % 2 == 0)[None]
            c = np.where(near.sum(1) > 1, even.argmax(1), near.argmax(1))
            codes[r, b * BLOCK:b * BLOCK + len(v)] = c + np.signbit(v) * 8
    return codes, scales


def mx4_values(codes, scales):
    """float64 [m, k] of unpacked codes and scale bytes."""
    v = GRID[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return v * np.repeat(s, BLOCK, axis=1)[:, : codes.shape[1]]


def mx4_pack(codes):
    m, k = codes.shape
    c = np.concatenate([codes, np.zeros((m, k % 2), np.uint8)], 1)
    return (c[:, 0::2] | (c[:, 1::2] << 4)).astype(np.uint8)


def ranking(z):
    """Ranked indices and their float64 logits: highest first, lowest index among equals; NaN and -inf out, +inf as the largest float."""
    z = np.asarray(z, np.float64)
    z = np.minimum(z, np.finfo(np.float32).max)
    ok = np.flatnonzero(~np.isnan(z) & (z > -np.inf))
    order = ok[np.lexsort((ok, -z[ok]))]
    return order, z[order]


def sample(z, temperature, top_k, top_p, min_p, u):
    """(token, p, how near the draw and the cuts came to another outcome, relative to the kept weight)."""
    f = lambda v: float(np.float32(v))  # noqa: E731
    temperature, top_p, min_p, u = f(temperature), f(top_p), f(min_p), f(u)
    order, s = ranking(z)
    if len(order) == 0:
        return -1, 0.0, 1.0
    if temperature == 0:
        return int(order[0]), 1.0, 1.0
    w = np.exp((s - s[0]) / temperature)
    if top_k:
        w = w[:top_k]
    near = 1.0
    tied = lambda v: bool(((v == 1.0) | (v == 0.0)).all())  # noqa: E731    sums of ones and zeros are exact: a border is no doubt
    if top_p < 1:
        run = np.cumsum(w)
        need = top_p * run[-1]
        n = int(np.searchsorted(run, need)) + 1
        if not tied(w):
            near = min(near, np.abs(run - need).min() / run[-1])
        w = w[:n]
    if min_p > 0:
        if not tied(w):
            # each weight is compared with min_p by itself: what could turn it is a relative error of that weight
            near = min(near, np.abs(w[w != 1.0] / min_p - 1).min())
        w = w[w >= min_p]
    run = np.cumsum(w)
    t = u * run[-1]
    i = min(int(np.searchsorted(run, t, side="right")), len(w) - 1)
    if not tied(w) and u > 0:
        near = min(near, np.abs(run - t).min() / run[-1])
    return int(order[i]), float(w[i] / run[-1]), float(near)


def tree_walk(parents, tokens, sampled):
    """(path, next token) of one tree."""
    n = len(parents)
    path = [0]
    while True:
        cur = path[-1]
        nxt = [c for c in range(cur + 1, n) if parents[c] == cur and tokens[c] == sampled[cur]]
        if not nxt:
            return path, int(sampled[cur])
        path.append(nxt[0])
