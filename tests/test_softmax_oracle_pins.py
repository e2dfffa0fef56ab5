"""Pins of oracle/softmax_oracle.py: the formulas written out, finite differences, planted mistakes, e4m3 by hand."""
import math

import numpy as np
import pytest

from oracle import softmax_oracle as S


def _rand(shape, seed):
    return np.random.default_rng(seed).standard_normal(shape)


@pytest.mark.parametrize("left,right,sinks", [(-1, -1, 0), (2, 0, 1), (0, 3, 2), (-1, 0, 0), (1, 1, 9)])
def test_seen_is_the_rule_written_out(left, right, sinks):
    n, length = 9, 7
    ok = S.seen(range(n), range(n), length, left, right, sinks)
    for i in range(n):
        for j in range(n):
            window = (right < 0 or j <= i + right) and (left < 0 or j >= i - left or j < sinks)
            assert ok[i, j] == (j < length and window)


def test_forward_of_two_keys_by_hand():
    # scores 0 and ln 3 -> weights 1/4, 3/4
    out, lse, p = S.forward(np.array([[1.0]]), np.array([[0.0], [math.log(3.0)]]), np.array([[4.0], [8.0]]), np.ones((1, 2), bool), 1.0)
    assert np.allclose(p, [[0.25, 0.75]]) and np.allclose(out, 7.0) and np.allclose(lse, math.log(4.0))


def test_a_row_without_keys_and_keys_without_a_row():
    q, k, v = _rand((2, 4), 1), _rand((3, 4), 2), _rand((3, 4), 3)
    ok = np.array([[True, False, True], [False, False, False]])
    v[1], k[1] = np.nan, np.inf
    out, lse, _ = S.forward(q, k, v, ok, 0.5)
    assert np.isfinite(out).all() and (out[1] == 0).all() and lse[1] == -np.inf and np.isfinite(lse[0])


def _loss(q, k, v, ok, scale, dout):
    return float((S.forward(q, k, v, ok, scale)[0] * dout).sum())


def _differences(q, k, v, ok, scale, dout, h=1e-5):
    res = []
    for x in (q, k, v):
        g = np.zeros_like(x)
        for at in np.ndindex(x.shape):
            keep = x[at]
            x[at] = keep + h
            up = _loss(q, k, v, ok, scale, dout)
            x[at] = keep - h
            g[at] = (up - _loss(q, k, v, ok, scale, dout)) / (2 * h)
            x[at] = keep
        res.append(g)
    return res


def test_gradients_match_finite_differences():
    q, k, v, do = _rand((6, 4), 1), _rand((6, 4), 2), _rand((6, 4), 3), _rand((6, 4), 4)
    ok = S.seen(range(6), range(6), 5, 2, 0, 1)
    ok[4] = False
    for a, b in zip(S.backward(q, k, v, ok, 0.7, do), _differences(q, k, v, ok, 0.7, do)):
        assert np.abs(a - b).max() < 1e-8


def test_planted_mistakes_are_caught_by_the_differences():
    q, k, v, do = _rand((6, 4), 1), _rand((6, 4), 2), _rand((6, 4), 3), _rand((6, 4), 4)
    ok, scale = S.seen(range(6), range(6), 6, 2, 0, 1), 0.7
    want = _differences(q, k, v, ok, scale, do)
    out, _, p = S.forward(q, k, v, ok, scale)
    dp, delta = do @ v.T, (do * out).sum(1)[:, None]
    for wrong in (scale * ((p * dp) @ k), (p * (dp - delta)) @ k, scale * ((p * (dp - delta.T)) @ k)):
        assert np.abs(wrong - want[0]).max() > 1e-3


def test_bounds_hold_for_rounded_operands():
    """Rounding P and dS to 8 bits in every way keeps the results inside the bounds."""
    q, k, v, do = _rand((20, 8), 1), _rand((20, 8), 2), _rand((20, 8), 3), _rand((20, 8), 4)
    ok, scale, u = S.seen(range(20), range(20), 20, 6, 0, 2), 0.4, 2.0 ** -8
    out, _, p = S.forward(q, k, v, ok, scale)
    rng = np.random.default_rng(5)
    wobble = lambda x: x * (1 + u * rng.choice((-1.0, 1.0), x.shape))
    assert (np.abs(wobble(wobble(p) @ v) - out) <= S.forward_bounds(q, k, v, ok, scale, u)[0] * (1 + u)).all()
    dq, dk, dv = S.backward(q, k, v, ok, scale, do)
    bq, bk, bv = S.backward_bounds(q, k, v, ok, scale, do, u, u)
    ds = wobble(p * (do @ v.T - (do * wobble(out)).sum(1)[:, None]))
    for got, want, bound in ((scale * ds @ k, dq, bq), (scale * ds.T @ q, dk, bk), (wobble(p).T @ do, dv, bv)):
        assert (np.abs(wobble(got) - want) <= bound * (1 + u)).all()


def test_e4m3_by_hand():
    g = S.e4m3_numbers()
    assert len(g) == 127 and g[0] == 0 and g[1] == 2.0 ** -9 and g[8] == 2.0 ** -6 and g[-1] == 448.0 and (np.diff(g) > 0).all()
    # amax 448 -> e 0; 17 lies between 16 (even code) and 18; 19 between 18 and 20: ties to the even codes
    v, e = S.quantise([448.0, 17.0, 19.0, -17.5, 2.0 ** -10, 3 * 2.0 ** -10])
    assert e == 0 and list(v) == [448.0, 16.0, 20.0, -18.0, 0.0, 2.0 ** -8]
    assert S.quantise([449.0])[1] == 1 and S.quantise([0.0]) == (np.zeros(1), S.LEAST_EXP)
    v, e = S.quantise([np.inf, 3.0, np.nan])
    assert np.isnan(v[0]) and np.isnan(v[2]) and v[1] == 3.0 and e == -7
