"""fp64 definition of softmax attention with a sliding window and first tokens, of its gradients, and of the quantised cache row.

Test infrastructure: written from the formulas, dense, on the CPU; the product never imports it.  With every result comes a bound on
how far a kernel may be from it that rounds, at unit `u` (half a step relative to the value: 2^-8 for bf16), the stored result and the operands
of the products, and sums in fp32: each rounding moves a value by at most u times its magnitude, so the bounds are the same sums over
magnitudes.
"""
from __future__ import annotations

import numpy as np

LEAST_EXP = -117
FP32 = 2.0 ** -24


def seen(pos, keys, length, left, right, sinks):
    """[queries, keys]: whether the query at pos[i] sees key keys[j] of a sequence of `length` tokens."""
    p, j = np.asarray(pos)[:, None], np.asarray(keys)[None, :]
    ok = np.broadcast_to(j < length, (p.shape[0], j.shape[1])).copy()
    if right >= 0:
        ok &= j <= p + right
    if left >= 0:
        ok &= (j >= p - left) | (j < sinks)
    return ok


def forward(q, k, v, ok, scale):
    """One head: q [m, d], k, v [n, d], ok [m, n] -> out, lse, p.  Rows of ok without a key: zeros, -inf.  Keys that no query sees are not looked at."""
    used = ok.any(0)
    k, v = np.where(used[:, None], k, 0.0), np.where(used[:, None], v, 0.0)
    s = np.where(ok, scale * (q @ k.T), -np.inf)
    top = s.max(1, initial=-np.inf)
    e = np.exp(s - np.where(np.isneginf(top), 0.0, top)[:, None])
    total = e.sum(1)
    some = total > 0
    p = e / np.where(some, total, 1.0)[:, None]
    lse = np.where(some, top + np.log(np.where(some, total, 1.0)), -np.inf)
    return p @ v, lse, p


def slack(q, k, ok, scale):
    """Relative error of a probability from fp32 scores: the exponent's rounding, at the magnitude of the terms it is summed from."""
    terms = abs(scale) * (np.abs(q) @ np.abs(np.where(ok.any(0)[:, None], k, 0.0)).T)
    return 8 * FP32 * (1.0 + np.where(ok, terms, 0.0).max(initial=0.0))


def forward_bounds(q, k, v, ok, scale, u):
    out, lse, p = forward(q, k, v, ok, scale)
    e = slack(q, k, ok, scale)
    v = np.where(ok.any(0)[:, None], v, 0.0)
    return u * np.abs(out) + (u + 2 * e) * (p @ np.abs(v)), np.where(np.isfinite(lse), e + 4 * FP32 * np.abs(np.where(np.isfinite(lse), lse, 0.0)), 0.0)


def backward(q, k, v, ok, scale, dout):
    """dq, dk, dv of one head."""
    out, _, p = forward(q, k, v, ok, scale)
    ds = p * (dout @ v.T - (dout * out).sum(1)[:, None])
    return scale * (ds @ k), scale * (ds.T @ q), p.T @ dout


def backward_bounds(q, k, v, ok, scale, dout, u, u_out):
    """u: rounding of operands and results; u_out: of the forward's result, from which the row sums dout . out may be taken."""
    out, _, p = forward(q, k, v, ok, scale)
    dq, dk, dv = backward(q, k, v, ok, scale, dout)
    e = slack(q, k, ok, scale)
    dp_mag = np.abs(dout) @ np.abs(v).T
    delta_err = (u_out * np.abs(dout) * np.abs(out)).sum(1) + (u_out + 4 * e) * ((np.abs(dout) * (p @ np.abs(v))).sum(1))
    ds = p * (dout @ v.T - (dout * out).sum(1)[:, None])
    ds_err = u * np.abs(ds) + p * (delta_err[:, None] + 4 * e * (dp_mag + (np.abs(dout) * np.abs(out)).sum(1)[:, None]))
    return (u * np.abs(dq) + abs(scale) * (ds_err @ np.abs(k)) + 4 * FP32 * abs(scale) * (np.abs(ds) @ np.abs(k)),
            u * np.abs(dk) + abs(scale) * (ds_err.T @ np.abs(q)) + 4 * FP32 * abs(scale) * (np.abs(ds).T @ np.abs(q)),
            u * np.abs(dv) + (u + 4 * e) * (p.T @ np.abs(dout)))


def e4m3_numbers():
    """The non-negative numbers of e4m3 (no infinities, 448 the largest) in the order of their codes."""
    small = [m / 8 * 2.0 ** -6 for m in range(8)]
    return np.array(small + [(1 + m / 8) * 2.0 ** (e - 7) for e in range(1, 16) for m in range(8)][:-1])


def quantise(row):
    """Row of finite or infinite or NaN numbers -> (values that the cache holds, exponent)."""
    row = np.asarray(row, dtype=np.float64)
    amax = np.abs(row[np.isfinite(row)]).max(initial=0.0)
    e = LEAST_EXP
    while amax > 448.0 * 2.0 ** e:
        e += 1
    grid = e4m3_numbers()
    grid = grid[grid * 2.0 ** e < 2.0 ** 128]          # what bf16 can hold
    got = np.empty_like(row)
    for i, x in enumerate(row):
        if not np.isfinite(x):
            got[i] = np.nan
            continue
        y = abs(x) * 2.0 ** -e
        dist = np.abs(grid - y)
        best = np.flatnonzero(dist == dist.min())
        code = best[0] if len(best) == 1 else [c for c in best if c % 2 == 0][0]
        got[i] = np.copysign(grid[code] * 2.0 ** e, x)
    return got, e
