"""fp64 definition of causal linear attention with a decay for each head, of its gradients, and of rotary positions.

Test infrastructure: written from the formulas, dense, on the CPU; the product never imports it.  With every result comes a bound on how far a kernel may be from it that
rounds, at unit `u` (half a step relative to the value: 2^-8 for bf16), the factors of its products, and sums in fp32: each rounding moves a value by at most u times its
magnitude, so the bounds are the same sums over magnitudes.
"""
from __future__ import annotations

import numpy as np

FP32 = 2.0 ** -24


def weights(n, g):
    """lambda^(i - j) for j <= i, else 0; g may be -inf."""
    r = np.arange(n)[:, None] - np.arange(n)[None]
    if g == -np.inf:
        return np.where(r == 0, 1.0, 0.0)
    return np.where(r >= 0, np.exp(g * np.maximum(r, 0)), 0.0)


def powers(g, r):
    """lambda^r; 0^0 = 1."""
    r = np.asarray(r, dtype=np.float64)
    return np.where(r == 0, 1.0, 0.0) if g == -np.inf else np.exp(g * r)


def rows(a, b, c, g, x, from_x):
    """sum_{j <= i} lambda^(i-j) (a_i . b_j) c_j + lambda^from_x[i] a_i x"""
    return ((a @ b.T) * weights(len(a), g)) @ c + powers(g, from_x)[:, None] * (a @ x)


def forward(q, k, v, g, scale, state):
    """One head: q, k, v [n, d], state [d, d] -> out, state behind the last token."""
    n = len(q)
    out = scale * rows(q, k, v, g, state, np.arange(n) + 1)
    return out, powers(g, n) * state + (powers(g, n - 1 - np.arange(n))[:, None] * k).T @ v


def backward(q, k, v, g, scale, state, dout, dstate):
    """dq, dk, dv, gradient of the state before the first token."""
    n = len(q)
    i = np.arange(n)
    dq = scale * rows(dout, v, k, g, state.T, i + 1)
    dk = rows(v[::-1], scale * dout[::-1], q[::-1], g, dstate.T, i)[::-1]
    dv = rows(k[::-1], scale * q[::-1], dout[::-1], g, dstate, i)[::-1]
    return dq, dk, dv, powers(g, n) * dstate + scale * (powers(g, i + 1)[:, None] * q).T @ dout


def _sum_error(n, d, g):
    """Relative error of fp32 sums over n tokens and d channels, and of their weights."""
    return (2 * n + d + 128 + (min(abs(g) * n, 110.0) if n else 0.0)) * FP32


def forward_bounds(q, k, v, g, scale, state, u):
    """Of the rows, three roundings at u of which two meet at most in a product's path (the weights of a pair; or the weighted row and the state); of the state fp32 alone."""
    out, end = forward(np.abs(q), np.abs(k), np.abs(v), g, scale, np.abs(state))
    e = _sum_error(*q.shape, g)
    return (2 * u + u * u + e) * out, e * end


def backward_bounds(q, k, v, g, scale, state, dout, dstate, u):
    dq, dk, dv, ds = backward(*[np.abs(x) for x in (q, k, v)], g, scale, *[np.abs(x) for x in (state, dout, dstate)])
    e = _sum_error(*q.shape, g)
    return [(2 * u + u * u + e) * x for x in (dq, dk, dv)] + [e * ds]


def pairs(dims, kind):
    """[(first channel, second channel, axis, m, dims of the axis)] of a row."""
    got, off = [], 0
    for a, size in enumerate(dims):
        for m in range(size // 2):
            got.append((off + 2 * m, off + 2 * m + 1, a, m, size) if kind == "adjacent" else (off + m, off + m + size // 2, a, m, size))
        off += size
    return got


def grid_positions(n, grid, first):
    """[n, axes]"""
    got = []
    for i in range(n):
        at, x = [], i
        for size in list(grid)[:0:-1]:
            at.append(x % size)
            x //= size
        got.append([a + f for a, f in zip([x] + at[::-1], first)])
    return np.array(got, dtype=np.int64).reshape(n, len(grid))


def rotary(x, pos, dims, kind, base, inverse):
    """x [..., n, d], pos [n, axes] -> turned x, and a bound on its error before it is rounded to its type: sine and cosine to 2^-22 (the fraction of a turn and
    the function), two products and a sum."""
    y, err = x.copy(), np.zeros_like(x)
    for one, two, a, m, size in pairs(dims, kind):
        t = pos[:, a] * base ** (-2.0 * m / size)
        c, s = np.cos(t), np.sin(-t if inverse else t)
        x1, x2 = x[..., one], x[..., two]
        y[..., one], y[..., two] = x1 * c - x2 * s, x1 * s + x2 * c
        # (cos and sin of the angle in fp64 are off by its rounding, below 2^-52 |t|)
        err[..., one] = err[..., two] = (2.0 ** -22 + 4 * FP32 + 2.0 ** -52 * np.abs(t)) * (np.abs(x1) + np.abs(x2))
    return y, err
