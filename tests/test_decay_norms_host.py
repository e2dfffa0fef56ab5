"""What the 2-norms of test_decay_norms_gpu.py refuse: results of a definition with one mistake, and roundings that a kernel must not make, on the CPU."""
import pytest
import torch

from tests.test_decay_norms_gpu import BEFORE, SUMS, _near, _rows, _sum

G, CUT = -0.004, 128


def _case(n=320, d=64, seed=3):
    gen = torch.Generator().manual_seed(seed)
    q, k, v = [torch.randn((n, d), generator=gen).bfloat16().double() for _ in range(3)]
    return q, k, v, torch.randn((d, d), generator=gen).double()


def _pieced(q, k, v, s, g=G, at=CUT, fade=1.0, shift=0, rounded=lambda x: x):
    """out in two pieces that a state joins, with a mistake in what it carries."""
    c = q.shape[1] ** -0.5
    state = rounded(_sum(k[:at], v[:at], g, s) * fade * torch.exp(torch.tensor(g * shift, dtype=torch.float64)))
    return torch.cat((c * _rows(q[:at], k[:at], v[:at], g, s, 1), c * _rows(q[at:], k[at:], v[at:], g, state, 1)))


def _out(q, k, v, s):
    c = q.shape[1] ** -0.5
    return c * _rows(q, k, v, G, s, 1), c * c * _rows(q * q, k * k, v * v, 2 * G, s * s, 1)


def _bf16(x):
    return x.to(torch.bfloat16).double()


@pytest.mark.parametrize("mode,dtype", [("bf16", torch.bfloat16), ("f32math", torch.bfloat16), ("f32", torch.float32)])
def test_right_results_pass(mode, dtype):
    x = _case()
    want, squares = _out(*x)
    _near("out", mode, _pieced(*x).to(dtype), want, squares, dtype, BEFORE[mode])
    # factors in two pieces
    q, k, v, s = x
    two = lambda y: _bf16(y) + _bf16(y - _bf16(y))
    _near("out", "bf16", _pieced(*x, rounded=two).to(torch.bfloat16), want, squares, torch.bfloat16, BEFORE["bf16"])


@pytest.mark.parametrize("mode,dtype", [("bf16", torch.bfloat16), ("f32math", torch.bfloat16), ("f32", torch.float32)])
@pytest.mark.parametrize("mistake", [dict(fade=0.9), dict(fade=1.0 + 1 / 256), dict(shift=1), dict(shift=-1), dict(rounded=_bf16)])
def test_a_wrong_state_is_refused(mode, dtype, mistake):
    """A tenth of it lost, a factor off by one bit of bf16, a power off by one token, a rounding to bf16."""
    x = _case()
    want, squares = _out(*x)
    with pytest.raises(AssertionError):
        _near("out", mode, _pieced(*x, **mistake).to(dtype), want, squares, dtype, BEFORE[mode])


def test_weights_rounded_once_are_refused():
    q, k, v, s = _case()
    want, squares = _out(q, k, v, s)
    i = torch.arange(len(q)).double()
    gap = i[:, None] - i[None]
    p = _bf16((q @ k.T) * torch.where(gap >= 0, torch.exp(G * gap.clamp(min=0)), 0.0) / 8)
    got = (p @ v + torch.exp(G * (i + 1))[:, None] * (q @ s) / 8).to(torch.bfloat16)
    with pytest.raises(AssertionError):
        _near("out", "bf16", got, want, squares, torch.bfloat16, BEFORE["bf16"])


@pytest.mark.parametrize("pieces,passes", [(1, False), (2, True), (3, True)])
def test_states_handed_out_are_whole(pieces, passes):
    """Weighted rows as one bf16 number are refused in a state.  Two, off by 1.66e-3 squared, 2.8e-6, are inside of 2^-18, 3.8e-6; three are fp32."""
    q, k, v, s = _case(n=2000)
    n = len(k)
    w = torch.exp(G * (n - 1 - torch.arange(n).double()))[:, None] * v
    rows, rest = torch.zeros_like(w), w
    for _ in range(pieces):
        piece = _bf16(rest)
        rows, rest = rows + piece, rest - piece
    got = k.T @ rows
    want, squares = _sum(k, v, G, None), _sum(k * k, v * v, 2 * G, None)
    if passes:
        _near("state", "bf16", got, want, squares, torch.float32, SUMS)
    else:
        with pytest.raises(AssertionError):
            _near("state", "bf16", got, want, squares, torch.float32, SUMS)
