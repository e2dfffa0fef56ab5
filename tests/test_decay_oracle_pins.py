"""The fp64 definition of causal linear attention with a decay and of rotary positions against the recurrence, differences and closed forms."""
import numpy as np
import pytest

from oracle import decay_oracle as O


def _case(n=23, d=8, seed=0):
    rng = np.random.default_rng(seed)
    return [rng.standard_normal(s) for s in ((n, d), (n, d), (n, d), (d, d), (n, d), (d, d))]


@pytest.mark.parametrize("g", [0.0, -0.3, -5.0, -np.inf])
def test_forward_is_the_recurrence(g):
    q, k, v, s, _, _ = _case()
    out, end = O.forward(q, k, v, g, 0.7, s)
    for i in range(len(q)):
        s = np.exp(g) * s + np.outer(k[i], v[i])
        assert np.allclose(out[i], 0.7 * q[i] @ s, rtol=1e-12, atol=1e-12)
    assert np.allclose(end, s, rtol=1e-12, atol=1e-12)


@pytest.mark.parametrize("g", [0.0, -0.3, -5.0])
def test_gradients_are_differences(g):
    q, k, v, s, do, ds = _case(n=7, d=4)

    def loss(q, k, v, s):
        out, end = O.forward(q, k, v, g, 0.7, s)
        return (out * do).sum() + (end * ds).sum()

    want = O.backward(q, k, v, g, 0.7, s, do, ds)
    for which, got in enumerate(want):
        x = [q, k, v, s]
        for at in np.ndindex(x[which].shape):
            moved = [y.copy() for y in x]
            moved[which][at] += 1e-6
            up = loss(*moved)
            moved[which][at] -= 2e-6
            assert abs((up - loss(*moved)) / 2e-6 - got[at]) < 1e-7


def test_pieces_join():
    """A sequence in two calls is the sequence in one."""
    q, k, v, s, _, _ = _case()
    out, end = O.forward(q, k, v, -0.2, 1.0, s)
    o1, s1 = O.forward(q[:9], k[:9], v[:9], -0.2, 1.0, s)
    o2, s2 = O.forward(q[9:], k[9:], v[9:], -0.2, 1.0, s1)
    assert np.allclose(np.concatenate((o1, o2)), out) and np.allclose(s2, end)


@pytest.mark.parametrize("kind", ["adjacent", "halves"])
def test_rotary_turns(kind):
    """Lengths stay, scores go by the difference of positions, and the inverse takes it back."""
    rng = np.random.default_rng(1)
    x, y = rng.standard_normal((2, 5, 12))
    pos = rng.integers(0, 50, (5, 2))
    dims = (6, 4)
    a, _ = O.rotary(x, pos, dims, kind, 100.0, False)
    assert np.allclose((a ** 2).sum(-1), (x ** 2).sum(-1)) and np.array_equal(a[:, 10:], x[:, 10:])
    assert np.allclose(O.rotary(a, pos, dims, kind, 100.0, True)[0], x)
    b, _ = O.rotary(y, pos + 3, dims, kind, 100.0, False)
    a2, _ = O.rotary(x, pos + 11, dims, kind, 100.0, False)
    b2, _ = O.rotary(y, pos + 14, dims, kind, 100.0, False)
    assert np.allclose((a * b).sum(-1), (a2 * b2).sum(-1))
    one, _ = O.rotary(np.eye(2)[:1], np.array([[1]]), (2,), kind, 100.0, False)
    assert np.allclose(one, [[np.cos(1), np.sin(1)]])


def test_grid_positions():
    assert O.grid_positions(7, (9, 2, 3), (10, 0, 5)).tolist() == [[10, 0, 5], [10, 0, 6], [10, 0, 7], [10, 1, 5], [10, 1, 6], [10, 1, 7], [11, 0, 5]]
    assert O.grid_positions(3, (1,), (4,)).tolist() == [[4], [5], [6]]
