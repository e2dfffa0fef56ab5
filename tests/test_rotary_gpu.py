"""linattn_rotary against the fp64 definition, element by element, inside bounds that count the roundings (oracle/decay_oracle.py)."""
import numpy as np
import pytest

from oracle import decay_oracle as O

pytestmark = pytest.mark.gpu

U = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def _tensor(mode, shape, seed):
    import torch
    gen = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=gen).to(torch.float32 if mode == "f32" else torch.bfloat16)


def _check(mode, B, H, HK, n, d, dims, kind, layout, grid=None, first=None, positions=None, base=10000.0, inverse=False, lengths=None, in_place=False, seed=1):
    import torch
    from paper_2510_08318_amd import torch_glue as G
    shape = lambda heads: (B, n, heads, d) if layout == "bnhd" else (B, heads, n, d)
    q, k = _tensor(mode, shape(H), seed), _tensor(mode, shape(HK), seed + 1) if HK else None
    host = [G.to_host_f64(x) if x is not None else None for x in (q, k)]
    if lengths is not None:
        for t in (q, k):
            for b, length in enumerate(lengths):
                t[b].narrow(0 if layout == "bnhd" else 1, length, n - length).fill_(float("nan"))
    q, k = q.cuda(), k.cuda() if HK else None
    L = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    P = None if positions is None else torch.tensor(positions, dtype=torch.int32, device="cuda")
    out = dict(q_out=q, k_out=k) if in_place else {}
    got = G.rotary(q, k, dims=dims, grid=grid, first=first, positions=P, base=base, pairs=kind, inverse=inverse, layout=layout, lengths=L, **out)
    torch.cuda.synchronize()
    assert (got[1] is None) == (not HK)
    if in_place:
        assert got[0] is q and got[1] is k
    where = O.grid_positions(n, grid or (1,), first or (0,) * len(dims)) if positions is None else np.asarray(positions)
    for x, y in zip(host, got):
        if x is None:
            continue
        y = G.to_host_f64(y)
        if layout == "bnhd":
            x, y = np.swapaxes(x, 1, 2), np.swapaxes(y, 1, 2)
        for b in range(B):
            want, err = O.rotary(x[b], where if where.ndim == 2 else where[b], dims, kind, base, inverse)
            live = n if lengths is None else lengths[b]
            over = np.abs(y[b] - want) - err - U[mode] * np.abs(want)
            assert (over[:, :live] <= 0).all(), (b, over[:, :live].max())
            assert (y[b][:, live:] == 0).all()
            used = sum(dims)
            assert np.array_equal(y[b][:, :live, used:], x[b][:, :live, used:])


CASES = [(128, (128,), None), (128, (44, 42, 42), (2, 3, 5)), (128, (32, 48, 48), (2, 3, 5)), (128, (64, 32), (2, 7)), (64, (32, 16, 16), (1, 4, 4)),
         (64, (24, 20, 20), (9, 1, 6)), (64, (16, 12, 10), (1, 2, 40)), (64, (2,), None), (64, (64,), None), (128, (48, 16), (1, 4)), (128, (2, 124), (1, 300))]


@pytest.mark.parametrize("mode", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["adjacent", "halves"])
@pytest.mark.parametrize("d,dims,grid", CASES)
def test_axes(mode, kind, d, dims, grid):
    _check(mode, 2, 3, 2, 31, d, dims, kind, "bnhd", grid=grid, first=tuple(range(5, 5 + len(dims))))


@pytest.mark.parametrize("layout", ["bhnd", "bnhd"])
@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("n,H,HK", [(1, 1, 1), (1, 40, 8), (17, 5, 0), (300, 9, 4), (1000, 12, 12)])
def test_lengths_and_heads(layout, inverse, n, H, HK):
    _check("bf16", 2, H, HK, n, 128, (44, 42, 42), "adjacent", layout, grid=(1, 5, 7), inverse=inverse)


@pytest.mark.parametrize("mode", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["adjacent", "halves"])
@pytest.mark.parametrize("shared", [False, True])
def test_explicit_positions(mode, kind, shared):
    """Far ones, negative ones, and the ends of their range; the first and the last frequency."""
    rng = np.random.default_rng(3)
    pos = rng.integers(-1000, 1 << 20, (2, 40, 2))
    pos[:, 0], pos[:, 1] = (1 << 31) - 1, -(1 << 31)
    _check(mode, 2, 3, 1, 40, 64, (32, 32), kind, "bhnd", positions=(pos[0] if shared else pos).tolist(), base=500.0,
           grid=(1, 3) if shared else None, first=(7, 9))      # (not looked at)


@pytest.mark.parametrize("mode", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["bhnd", "bnhd"])
def test_padded_batch_in_place(mode, layout):
    _check(mode, 4, 3, 3, 70, 64, (24, 20, 20), "halves", layout, grid=(1, 6, 6), lengths=[0, 1, 33, 70], in_place=True)
    _check(mode, 4, 3, 3, 70, 64, (24, 20, 20), "adjacent", layout, grid=(1, 6, 6), lengths=[70, 0, 0, 69], in_place=True)


@pytest.mark.parametrize("kind", ["adjacent", "halves"])
def test_channels_without_an_axis_stay_beside_infinities(kind):
    import torch
    from paper_2510_08318_amd import torch_glue as G
    q = _tensor("bf16", (1, 2, 9, 64), 4)
    q[..., 38] = float("inf")
    q[..., 40:] = float("nan")
    got, _ = G.rotary(q.cuda(), dims=(20, 18), grid=(1, 3), pairs=kind)
    assert torch.isfinite(got[..., :38]).all() and torch.isinf(got[..., 38]).all() and torch.isnan(got[..., 40:]).all()
    assert torch.equal(got[..., 39].cpu(), q[..., 39])


def test_rows_behind_32_bits():
    """A tensor of more than 2^31 elements."""
    import torch
    from paper_2510_08318_amd import torch_glue as G
    n, d = (1 << 25) + 77, 64
    q = torch.zeros((1, 1, n, d), dtype=torch.bfloat16, device="cuda")
    q[0, 0, -3:] = 1.0
    got, _ = G.rotary(q, dims=(64,), q_out=q)
    tail = G.to_host_f64(got[0, 0, -3:])
    want, err = O.rotary(np.ones((3, d)), np.arange(n - 3, n)[:, None], (64,), "adjacent", 10000.0, False)
    assert (np.abs(tail - want) <= err + U["bf16"] * np.abs(want)).all()
    assert not got[0, 0, : 1000].any() and not got[0, 0, -1000: -3].any()


@pytest.mark.parametrize("kind,layout", [("adjacent", "bnhd"), ("halves", "bhnd")])
def test_full_size(kind, layout):
    """A layer's size at 832x480, more than the last-level cache has room for: tokens here and there."""
    import torch
    from paper_2510_08318_amd import torch_glue as G
    H, n, d, dims, grid = 12, 32760, 128, (44, 42, 42), (21, 30, 52)
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, k = [torch.randn((1, n, H, d) if layout == "bnhd" else (1, H, n, d), generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2)]
    got = G.rotary(q, k, dims=dims, grid=grid, pairs=kind, layout=layout)
    rows = np.array([0, 1, 51, 52, 1559, 1560, 20000, 32759])
    at = torch.tensor(rows, device="cuda")
    pos = np.stack((rows // 1560, rows // 52 % 30, rows % 52), 1)
    for x, y in zip((q, k), got):
        x, y = [G.to_host_f64(t[0, at].transpose(0, 1) if layout == "bnhd" else t[0][:, at]) for t in (x, y)]
        want, err = O.rotary(x, pos, dims, kind, 10000.0, False)
        assert (np.abs(y - want) <= err + U["bf16"] * np.abs(want)).all()


def test_gradient_by_differences():
    """The inverse of an upstream gradient is the gradient of the sum that it weighs."""
    import torch
    from paper_2510_08318_amd import torch_glue as G
    x, g = _tensor("f32", (1, 1, 3, 64), 5).cuda(), _tensor("f32", (1, 1, 3, 64), 6).cuda()
    kw = dict(dims=(24, 20, 20), grid=(1, 2, 2), first=(3, 1, 0))
    dx, _ = G.rotary(g, inverse=True, **kw)
    for at in [(0, 0, 1, 0), (0, 0, 2, 23), (0, 0, 2, 44), (0, 0, 1, 63)]:
        y = x.clone()
        y[at] += 1.0                                    # the operator is linear: differences are exact but for roundings
        diff = ((G.rotary(y, **kw)[0].double() - G.rotary(x, **kw)[0].double()) * g.double()).sum().item()
        assert abs(diff - dx[at].item()) < 64 * 2.0 ** -22 * 8


def test_streams_and_captured_graphs():
    import torch
    from paper_2510_08318_amd import torch_glue as G
    q, k = _tensor("bf16", (2, 50, 6, 128), 7).cuda(), _tensor("bf16", (2, 50, 2, 128), 8).cuda()
    pos = torch.arange(100, dtype=torch.int32, device="cuda").view(2, 50, 1)
    want = G.rotary(q, k, positions=pos, layout="bnhd")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = G.rotary(q, k, positions=pos, layout="bnhd")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            held = G.rotary(q, k, positions=pos, layout="bnhd")
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    for step in range(3):
        pos += 5 * step
        graph.replay()
        torch.cuda.synchronize()
        now = G.rotary(q, k, positions=pos, layout="bnhd")
        assert all(torch.equal(a, b) for a, b in zip(held, now)), step
