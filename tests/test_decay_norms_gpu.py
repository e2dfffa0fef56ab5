"""linattn_decay_fwd and linattn_decay_bwd against the definition in 64 bits, by 2-norms: every head, every 64 rows, every state.  The elementwise bounds of test_decay_gpu.py hold
for any order and sign of the roundings, and are as large as the results where many tokens are seen; errors of 2-norms are far smaller, since roundings are as often up as down, and
a state with a wrong weight, or one rounded where it should not be, is far outside.  Their tolerances:

results in the tensors' type: the error of the definition's own result after its one rounding, s = |round(y) - y|, is there for every kernel.  A kernel that is off by e |y| before it
    rounds is at most e |y| + s' away, s' the rounding of a value that close to y.  bf16: factors in two pieces, each off by at most 2^-16 of it; their signs vary, and a row has at least 64
    channels of many pairs, so that the sum is off by a fraction of 2^-16 |y|, and e = 2^-13 leaves a factor of eight and more.  fp32: e = 2^-18, below.
sums in fp32: an element is a sum over 64 or 128 channels, 32 or 64 tokens of a chunk, and the chunks and segments before it: at most 400 roundings in a row in the sizes here, each at most
    2^-24 of a partial sum that is at most a few times the result in the 2-norm; sqrt(400) 2^-24 = 2^-19.7, and 2^-18 leaves a factor of three.
|y| is the 2-norm of the result or, where that is larger, of the root of the sum of its terms' squares.  Partial sums are as large as the latter, whatever is left of them: of one token without a
    state, out = scale (q . k) v, where q . k of 64 or 128 products with random signs is as often as not below two thirds of the root of the sum of their squares, in one of a hundred below an
    eightieth, and its roundings are those of the partial sums.  The terms' squares are the same sums of squared numbers, the decay twice as fast.
states that are handed out are such sums, of bf16 tensors too.
"""
import pytest

pytestmark = pytest.mark.gpu

SUMS = 2.0 ** -18
BEFORE = {"bf16": 2.0 ** -13, "f32math": SUMS, "f32": SUMS}
CODE = {"bf16": 1, "f32": 2, "f32math": 3}


def _make(mode, B, H, HK, n, d, layout, seed, state=True):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def t(heads):
        shape = (B, n, heads, d) if layout == "bnhd" else (B, heads, n, d)
        return torch.randn(shape, generator=gen, device="cuda").to(torch.float32 if mode == "f32" else torch.bfloat16)
    s = [torch.randn((B, H, d, d), generator=gen, device="cuda") if state else None for _ in range(2)]
    return t(H), t(HK), t(HK), t(H), *s


def _decays(H):
    """None, memories of thousands of tokens, of hundreds, of ten, of one."""
    import torch
    return torch.tensor([(0.0, -0.0004, -0.004, -0.1, -1.5)[h % 5] for h in range(H)], device="cuda")


def _rows(a, b, c, g, x, start):
    """One head in 64 bits: sum_{j <= i} lambda^(i-j) (a_i . b_j) c_j + lambda^(i+start) a_i x, 1024 rows at a time."""
    import torch
    n, out = len(a), torch.empty_like(a)
    i = torch.arange(n, device=a.device, dtype=torch.float64)
    for r in range(0, n, 1024):
        e = min(n, r + 1024)
        gap = i[r:e, None] - i[None, :e]
        out[r:e] = ((a[r:e] @ b[:e].T) * torch.where(gap >= 0, torch.exp(g * gap.clamp(min=0)), 0.0)) @ c[:e]
    return out if x is None else out + torch.exp(g * (i + start))[:, None] * (a @ x)


def _sum(b, c, g, x):
    """The state behind the last token."""
    import torch
    n = len(b)
    i = torch.arange(n, device=b.device, dtype=torch.float64)
    s = (torch.exp(g * (n - 1 - i))[:, None] * b).T @ c
    return s if x is None else s + torch.exp(torch.tensor(g * n, dtype=torch.float64)).item() * x


def _definition(q, k, v, do, g, c, s, ds):
    """out, state, dq, dk, dv, dstate of one head."""
    T = lambda x: None if x is None else x.T
    f = lambda x: x.flip(0)
    return (c * _rows(q, k, v, g, s, 1), _sum(k, v, g, s), c * _rows(do, v, k, g, T(s), 1), f(_rows(f(v), c * f(do), f(q), g, T(ds), 0)),
            f(_rows(f(k), c * f(q), f(do), g, ds, 0)), _dstate(q, do, g, c, ds))


def _dstate(q, do, g, c, ds):
    import math
    import torch
    i = torch.arange(len(q), device=q.device, dtype=torch.float64)
    x = c * (torch.exp(g * (i + 1))[:, None] * q).T @ do
    return x if ds is None else x + math.exp(g * len(q)) * ds


def _near(name, mode, got, want, squares, dtype, before):
    """Blocks of 64 rows; want, and the sums of its terms' squares, in 64 bits."""
    s = (want.to(dtype).double() - want)
    for r in range(0, len(want), 64):
        e = slice(r, r + 64)
        err, tol = (got[e].double() - want[e]).norm(), 1.03 * s[e].norm() + before * max(want[e].norm(), squares[e].sum().sqrt())
        assert err <= tol, (name, mode, r, (err / want[e].norm()).item(), (tol / want[e].norm()).item())


def check(mode, B, H, HK, n, d, layout="bhnd", lengths=None, state=True, train=True, seed=1, heads=None, segments=None):
    """segments: (least, most) of the forward, by its workspace."""
    import torch
    from paper_2510_08318_amd import binding as L, torch_glue as G
    q, k, v, do, s0, ds1 = _make(mode, B, H, HK, n, d, layout, seed, state)
    if segments:
        w = L.DecayDesc(CODE[mode], B, H, HK, n, d, 0, 0.0, 256, None, None, 0, None, 0)
        got = L.linattn_decay_workspace_bytes(w) // (B * H * d * d * 4) or 1
        assert segments[0] <= got <= segments[1], got
    g = _decays(H)
    kw = dict(state=s0, layout=layout, lengths=None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda"), f32_math=mode == "f32math")
    out, end = G.decay_attention(q, k, v, g, **kw)
    only, _ = G.decay_attention(q, k, v, g, state_out=False, **kw)
    got = dict(out=out, only=only)
    if train:
        got["dq"], got["dk"], got["dv"], dstate = G.decay_attention_backward(q, k, v, g, do, dstate=ds1, **kw)
    first = (lambda x: x.transpose(1, 2)) if layout == "bnhd" else (lambda x: x)
    q, k, v, do = [first(x) for x in (q, k, v, do)]
    got = {name: first(x) for name, x in got.items()}
    R = H // HK
    for b in range(B):
        m = n if lengths is None else lengths[b]
        for j in range(HK):
            if heads is not None and (b, j) not in heads:
                continue
            dk = dv = dk2 = dv2 = 0.0
            for h in range(j * R, j * R + R):
                x = [None if t is None else t.double() for t in (q[b, h, :m], k[b, j, :m], v[b, j, :m], do[b, h, :m], None if s0 is None else s0[b, h],
                                                                 None if ds1 is None else ds1[b, h])]
                w = _definition(*x[:4], float(g[h].double()), d ** -0.5, *x[4:])
                z = _definition(*[t * t for t in x[:4]], 2 * float(g[h].double()), 1 / d, *[None if t is None else t * t for t in x[4:]])
                _near(f"out {b} {h}", mode, got["out"][b, h, :m], w[0], z[0], out.dtype, BEFORE[mode])
                _near(f"out alone {b} {h}", mode, got["only"][b, h, :m], w[0], z[0], out.dtype, BEFORE[mode])
                _near(f"state {b} {h}", mode, end[b, h], w[1], z[1], torch.float32, SUMS)
                assert not got["out"][b, h, m:].any() and not got["only"][b, h, m:].any()
                if train:
                    _near(f"dq {b} {h}", mode, got["dq"][b, h, :m], w[2], z[2], out.dtype, BEFORE[mode])
                    dk, dv, dk2, dv2 = dk + w[3], dv + w[4], dk2 + z[3], dv2 + z[4]
                    if state:
                        _near(f"dstate {b} {h}", mode, dstate[b, h], w[5], z[5], torch.float32, SUMS)
            if train:
                for name, x, x2 in (("dk", dk, dk2), ("dv", dv, dv2)):
                    _near(f"{name} {b} {j}", mode, got[name][b, j, :m], x, x2, out.dtype, BEFORE[mode])
                    assert not got[name][b, j, m:].any()


MODES = ("bf16", "f32", "f32math")


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("state", [False, True])
def test_one_chunk_and_several(mode, d, state):
    for n in (9, 33, 64, 65, 200):
        check(mode, 1, 5, 5, n, d, state=state, seed=n)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("d", [64, 128])
def test_several_segments(mode, d):
    check(mode, 1, 5, 5, 1300, d, "bnhd", segments=(6, 64))
