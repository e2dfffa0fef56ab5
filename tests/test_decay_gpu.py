"""linattn_decay_fwd and linattn_decay_bwd against the fp64 definition, element by element, inside bounds that count the roundings (oracle/decay_oracle.py)."""
import numpy as np
import pytest

from oracle import decay_oracle as O

pytestmark = pytest.mark.gpu

STORE = {"bf16": 2.0 ** -8, "f32math": 2.0 ** -8, "f32": 2.0 ** -24}        # of the results
FACTOR = {"bf16": 2.0 ** -8, "f32math": 2.0 ** -22, "f32": 2.0 ** -22}      # of the products' factors
MODES = ("bf16", "f32", "f32math")


def _make(mode, B, H, HK, n, d, layout, seed):
    import torch
    gen = torch.Generator().manual_seed(seed)
    dt = torch.float32 if mode == "f32" else torch.bfloat16

    def t(heads, mul=1.0):
        x = (torch.randn((B, heads, n, d), generator=gen) * mul).to(dt)
        return (x.transpose(1, 2) if layout == "bnhd" else x).contiguous().cuda()
    states = [torch.randn((B, H, d, d), generator=gen) for _ in range(2)]
    return t(H), t(HK), t(HK), t(H, 0.3), states[0].cuda(), (states[1] * 0.3).cuda()


def _decays(H):
    """No decay, memories of a hundred tokens, of a few, of less than one, and none."""
    import torch
    return torch.tensor([(0.0, -0.01, -0.3, -4.0, -0.0005, -float("inf"))[h % 6] for h in range(H)], dtype=torch.float32, device="cuda")


def _host(x, layout):
    from paper_2510_08318_amd import torch_glue as G
    a = G.to_host_f64(x)
    return np.swapaxes(a, 1, 2) if layout == "bnhd" else a


def _inside(name, got, want, bound):
    assert np.isfinite(got).all(), name
    over = np.abs(got - want) - bound - 1e-28
    assert (over <= 0).all(), (name, np.unravel_index(over.argmax(), over.shape), over.max(), bound.max())


def _check(mode, B, H, HK, n, d, layout="bhnd", lengths=None, state=True, train=True, seed=1, g=None, scale=0.0, edit=None):
    """edit(q, k, v, dout): changes to tokens that no result may depend on."""
    import torch
    from paper_2510_08318_amd import torch_glue as G
    q, k, v, do, s0, ds1 = _make(mode, B, H, HK, n, d, layout, seed)
    hq, hk, hv, hd = [_host(x, layout) for x in (q, k, v, do)]
    if edit:
        edit(q, k, v, do)
    if not state:
        s0 = ds1 = None
    hs, he = [np.zeros((B, H, d, d)) if x is None else G.to_host_f64(x) for x in (s0, ds1)]
    g = _decays(H) if g is None else g
    hg = g.cpu().double().numpy()
    L = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    kw = dict(state=s0, layout=layout, lengths=L, f32_math=mode == "f32math", scale=scale)
    out, end = G.decay_attention(q, k, v, g, **kw)
    only, none = G.decay_attention(q, k, v, g, **{**kw, "state_out": False})
    assert none is None
    grads = G.decay_attention_backward(q, k, v, g, do, dstate=ds1, **kw) if train else ()
    torch.cuda.synchronize()
    c, u, f = scale or d ** -0.5, STORE[mode], FACTOR[mode]
    out, only, end = _host(out, layout), _host(only, layout), G.to_host_f64(end)
    if train:
        dq, dk, dv = [_host(x, layout) for x in grads[:3]]
        assert (grads[3] is None) == (s0 is None)
        dstate = None if grads[3] is None else G.to_host_f64(grads[3])
    for b in range(B):
        m = n if lengths is None else lengths[b]
        sums = {name: np.zeros((HK, m, d)) for name in ("dk", "dv", "ek", "ev")}
        for h in range(H):
            j = h // (H // HK)
            args = (hq[b, h, :m], hk[b, j, :m], hv[b, j, :m], hg[h], c, hs[b, h])
            want, after = O.forward(*args)
            eo, es = O.forward_bounds(*args, f)
            for x in (out, only):
                _inside(f"out {b} {h}", x[b, h, :m], want, eo + u * np.abs(want))
                assert (x[b, h, m:] == 0).all()
            _inside(f"state {b} {h}", end[b, h], after, es)
            if not train:
                continue
            rq, rk, rv, rs = O.backward(*args, hd[b, h, :m], he[b, h])
            eq, ek, ev, es = O.backward_bounds(*args, hd[b, h, :m], he[b, h], f)
            _inside(f"dq {b} {h}", dq[b, h, :m], rq, eq + u * np.abs(rq))
            assert (dq[b, h, m:] == 0).all()
            if dstate is not None:
                _inside(f"dstate {b} {h}", dstate[b, h], rs, es)
            for name, x in (("dk", rk), ("dv", rv), ("ek", ek), ("ev", ev)):
                sums[name][j] += x
        if train:
            _inside(f"dk {b}", dk[b][:, :m], sums["dk"], sums["ek"] + u * np.abs(sums["dk"]))
            _inside(f"dv {b}", dv[b][:, :m], sums["dv"], sums["ev"] + u * np.abs(sums["dv"]))
            assert (dk[b][:, m:] == 0).all() and (dv[b][:, m:] == 0).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 128, 129, 200, 333])
def test_lengths(n, d):
    _check("bf16", 1, 6, 6, n, d)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("layout", ["bhnd", "bnhd"])
@pytest.mark.parametrize("state", [False, True])
def test_types_widths_and_layouts(mode, d, layout, state):
    _check(mode, 2, 6, 2, 150, d, layout, state=state)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("n", [1, 5, 40, 65, 130])
def test_fp32_arithmetic_lengths(mode, n):
    _check(mode, 3, 3, 3, n, 64, "bnhd", scale=0.37)


@pytest.mark.parametrize("H,HK", [(8, 1), (6, 3), (5, 5)])
@pytest.mark.parametrize("mode", ["bf16", "f32"])
def test_shared_key_heads(H, HK, mode):
    _check(mode, 2, H, HK, 210, 64, "bnhd")


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("n", [9, 150])
def test_padded_batch(mode, n):
    """Items of no token, of one, of all; the padding holds NaN."""
    lengths = [0, 1, n - 1, n, n // 2]

    def edit(q, k, v, do):
        for t in (q, k, v, do):
            for b, length in enumerate(lengths):
                t[b, :, length:] = float("nan")
    _check(mode, 5, 6, 3, n, 64, lengths=lengths, edit=edit)


@pytest.mark.parametrize("mode", ["bf16", "f32"])
@pytest.mark.parametrize("n", [700, 1300])
def test_longer_sequences(mode, n):
    """Several workgroups to a head."""
    _check(mode, 1, 3, 1, n, 128 if mode == "bf16" else 64, g=__import__("torch").tensor([0.0, -0.003, -0.2], device="cuda"))


@pytest.mark.parametrize("mode,d", [("f32", 128), ("f32math", 128), ("f32math", 64), ("bf16", 64)])
def test_longer_sequences_other_types(mode, d):
    _check(mode, 1, 2, 2, 900, d, "bnhd", g=__import__("torch").tensor([-0.0004, -0.05], device="cuda"))


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("d", [64, 128])
def test_padded_batch_over_segments(mode, d):
    """Items that end in a segment, at its end, before the last ones; shared key heads."""
    n, lengths = 1000, [1000, 512, 513, 63, 960, 0]

    def edit(q, k, v, do):
        for t in (q, k, v, do):
            for b, length in enumerate(lengths):
                t[b, length:] = float("inf")
    _check(mode, 6, 2, 1, n, d, "bnhd", lengths=lengths, edit=edit, g=__import__("torch").tensor([-0.002, -0.1], device="cuda"))


def test_full_size():
    """A layer's size at 832x480 and more heads than the last-level cache has room for: rows of a few heads, here and there, and their states, against the definition in 64 bits."""
    import torch
    from paper_2510_08318_amd import torch_glue as G
    H, n, d = 18, 32760, 128
    gen = torch.Generator(device="cuda").manual_seed(12)
    q, k, v, do = [torch.randn((1, H, n, d), generator=gen, device="cuda").to(torch.bfloat16) for _ in range(4)]
    g = -torch.exp2(-8.0 * torch.arange(1, H + 1, device="cuda") / H)
    out, end = G.decay_attention(q, k, v, g)
    dq, dk, dv, _ = G.decay_attention_backward(q, k, v, g, do)
    rows = torch.tensor([0, 1, 63, 64, 127, 831, 832, 5000, 16383, 16384, 20001, 32700, 32759], device="cuda")
    for h in (0, 7, 16, 17):
        Q, K, V, D = [x[0, h].double() for x in (q, k, v, do)]
        i, c, gh = torch.arange(n, device="cuda").double(), d ** -0.5, float(g[h].double())

        def near(name, got, a, b, x, back):
            gap = (i[None] - i[rows, None]) * (1 if back else -1)
            w = torch.where(gap >= 0, torch.exp(gh * gap.clamp(min=0)), 0.0)
            want, mass = c * (((a[rows] @ b.T) * w) @ x), c * (((a[rows].abs() @ b.T.abs()) * w) @ x.abs())
            err = FACTOR["bf16"] * 2.01 + (2 * n + d + 128 + 110) * O.FP32
            over = (got[0, h, rows].double() - want).abs() - err * mass - STORE["bf16"] * want.abs()
            assert (over <= 0).all(), (name, h, over.max())
        near("out", out, Q, K, V, False)
        near("dq", dq, D, V, K, False)
        near("dk", dk, V, D, Q, True)
        near("dv", dv, K, Q, D, True)
        w = torch.exp(gh * (n - 1 - i))[:, None]
        over = (end[0, h].double() - (w * K).T @ V).abs() - (2 * n + d + 128 + 110) * O.FP32 * ((w * K.abs()).T @ V.abs())
        assert (over <= 0).all(), (h, over.max())


@pytest.mark.parametrize("mode", ["bf16", "f32"])
def test_many_heads(mode):
    """As many heads as fill the chip: a workgroup takes all of a head's tokens."""
    _check(mode, 24, 24, 24, 70, 64, train=mode == "bf16", lengths=[70, 1, 0, 64] * 6)


def test_decays_out_of_range_count_as_none():
    import torch
    from paper_2510_08318_amd import torch_glue as G
    q, k, v, do, s, ds = _make("bf16", 1, 3, 3, 80, 64, "bhnd", 2)
    bad = torch.tensor([0.5, float("nan"), float("inf")], device="cuda")
    a = G.decay_attention(q, k, v, bad, state=s)
    b = G.decay_attention(q, k, v, torch.zeros(3, device="cuda"), state=s)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("n,at", [(130, 70), (12, 5), (64, 63), (200, 100)])
def test_what_is_not_finite_reaches_only_what_sees_it(mode, n, at):
    """out and dq before token `at`, dk and dv behind it, other columns of v: as they are without the infinities and NaN."""
    import torch
    from paper_2510_08318_amd import torch_glue as G
    q, k, v, do, s, ds = _make(mode, 1, 2, 2, n, 64, "bhnd", 5)
    g = torch.tensor([-0.02, -0.5], device="cuda")
    kw = dict(state=s, f32_math=mode == "f32math")
    for which, value in ((0, "nan"), (1, "inf"), (2, "nan"), (2, "-inf"), (3, "nan"), (1, "nan")):
        x = [t.clone() for t in (q, k, v, do)]
        x[which][:, 1, at, 3] = float(value)
        clean = [t.clone() for t in (q, k, v, do)]
        clean[which][:, 1, at, 3] = 0.0
        got, want = [(G.decay_attention(*y[:3], g, **kw)[0], *G.decay_attention_backward(*y[:3], g, y[3], dstate=ds, **kw)[:3]) for y in (x, clean)]
        close = lambda a, b: b.numel() == 0 or torch.allclose(a.float(), b.float(), rtol=2.0 ** -6, atol=2.0 ** -6 * float(b.float().abs().amax()))
        for name, a, b in zip(("out", "dq", "dk", "dv"), got, want):
            assert torch.equal(a[:, 0], b[:, 0]), (name, which, value)
            seen = a[:, 1, :at] if name in ("out", "dq") else a[:, 1, at + 1:]
            clear = b[:, 1, :at] if name in ("out", "dq") else b[:, 1, at + 1:]
            assert torch.isfinite(seen).all() and close(seen, clear), (name, which, value)
        if which == 2:
            assert not torch.isfinite(got[0][:, 1, at:, 3]).any()
            rest = [c for c in range(64) if c != 3]
            assert close(got[0][:, 1, :, rest], want[0][:, 1, :, rest])


def test_large_and_small_magnitudes():
    import torch
    _check("bf16", 1, 3, 3, 100, 64, scale=2.0 ** 60)
    _check("f32", 1, 3, 3, 100, 64, scale=2.0 ** -60)


# ---- states: pieces of a sequence, slots, in place ---------------------------------------------------------------------------


@pytest.mark.parametrize("mode", MODES)
def test_pieces_of_a_sequence(mode):
    """A prompt, a chunk, tokens one by one: what one call gives, and what the definition gives."""
    import torch
    from paper_2510_08318_amd import torch_glue as G
    n, cuts = 260, [0, 170, 250, 251, 252, 260]
    q, k, v, _, s, _ = _make(mode, 2, 4, 2, n, 64, "bnhd", 6)
    g = _decays(4)
    kw = dict(layout="bnhd", f32_math=mode == "f32math")
    state, parts = s.clone(), []
    for a, b in zip(cuts, cuts[1:]):
        out, same = G.decay_attention(*[x[:, a:b].contiguous() for x in (q, k, v)], g, state=state, state_out=state, **kw)
        assert same is state
        parts.append(out)
    got = _host(torch.cat(parts, 1), "bnhd")
    hq, hk, hv = [_host(x, "bnhd") for x in (q, k, v)]
    for b in range(2):
        for h in range(4):
            args = (hq[b, h], hk[b, h // 2], hv[b, h // 2], float(g[h].double()), 0.125, G.to_host_f64(s)[b, h])
            want, end = O.forward(*args)
            eo, es = O.forward_bounds(*args, FACTOR[mode])
            _inside("out", got[b, h], want, eo + STORE[mode] * np.abs(want))
            _inside("state", G.to_host_f64(state)[b, h], end, es)


@pytest.mark.parametrize("n", [1, 7, 90])
@pytest.mark.parametrize("B", [3, 80])
def test_slots(n, B):
    """States by slot, in place and from one pool to another; a slot that is none reads zeros and writes nothing; other rows stay."""
    import torch
    from paper_2510_08318_amd import torch_glue as G
    H, d = 8, 64
    q, k, v, do, _, ds = _make("bf16", B, H, 4, n, d, "bnhd", 7)
    pool = torch.randn((B + 4, H, d, d), generator=torch.Generator().manual_seed(3)).cuda()
    slots = torch.randperm(B + 4, generator=torch.Generator().manual_seed(4))[:B].int()
    slots[1], slots[2] = -1, B + 4
    lengths = torch.tensor([n - (b % 3 == 0 and n > 1) for b in range(B)], dtype=torch.int32)
    real = [(b, int(x)) for b, x in enumerate(slots) if 0 <= x < B + 4]
    state = torch.zeros((B, H, d, d), device="cuda")
    for b, x in real:
        state[b] = pool[x]
    kw = dict(layout="bnhd", lengths=lengths.cuda())
    want, end = G.decay_attention(q, k, v, _decays(H), state=state, **kw)
    at = slots.cuda()
    other = torch.full_like(pool, 7.0)
    out, res = G.decay_attention(q, k, v, _decays(H), state=pool, slots=at, state_out=other, **kw)
    assert res is other and torch.equal(out, want)
    used = torch.zeros(B + 4, dtype=torch.bool)
    for b, x in real:
        assert torch.equal(other[x], end[b])
        used[x] = True
    assert (other[~used.cuda()] == 7.0).all()
    grads = G.decay_attention_backward(q, k, v, _decays(H), do, state=pool, dstate=ds, slots=at, **kw)
    same = G.decay_attention_backward(q, k, v, _decays(H), do, state=state, dstate=ds, **kw)
    assert all(torch.equal(a, b) for a, b in zip(grads, same))
    before = pool.clone()
    out, res = G.decay_attention(q, k, v, _decays(H), state=pool, slots=at, **kw)
    assert res is pool and torch.equal(out, want) and torch.equal(pool[used.cuda()], other[used.cuda()])
    assert torch.equal(pool[~used.cuda()], before[~used.cuda()])


def test_offsets_past_32_bits():
    """States and rows behind 2^31 elements."""
    import torch
    from paper_2510_08318_amd import torch_glue as G
    H, d, S = 4, 128, (1 << 31) // (4 * 128 * 128) + 5
    pool = torch.zeros((S, H, d, d), device="cuda")
    q, k, v, _, s, _ = _make("bf16", 1, H, H, 1, d, "bnhd", 8)
    pool[S - 2] = s[0]
    slots = torch.tensor([S - 2], dtype=torch.int32, device="cuda")
    want, end = G.decay_attention(q, k, v, _decays(H), state=s, layout="bnhd")
    out, _ = G.decay_attention(q, k, v, _decays(H), state=pool, slots=slots, layout="bnhd")
    assert torch.equal(out, want) and torch.equal(pool[S - 2], end[0]) and not pool[S - 1].any() and not pool[: S - 2].any()


def test_a_run_together():
    """Positions, attention, and their gradients back, as a layer does it; the same through the paged cache's branch."""
    import torch
    from paper_2510_08318_amd import torch_glue as G
    B, H, n, d = 1, 3, 90, 64
    q, k, v, do, s, ds = _make("f32", B, H, H, n, d, "bnhd", 9)
    g, turn = _decays(H), dict(dims=(24, 20, 20), grid=(1, 5, 6), layout="bnhd")

    def loss(q, k, v):
        a, b = G.rotary(q, k, **turn)
        out, end = G.decay_attention(a, b, v, g, state=s, layout="bnhd")
        return (out.double() * do.double()).sum() + (end.double() * ds.double()).sum()

    a, b = G.rotary(q, k, **turn)
    da, db, dv, _ = G.decay_attention_backward(a, b, v, g, do, state=s, dstate=ds, layout="bnhd")
    dq, dk = G.rotary(da, db, inverse=True, **turn)
    gen = torch.Generator().manual_seed(1)
    for which, grad in enumerate((dq, dk, dv)):
        step = torch.randn((B, n, H, d), generator=gen).cuda()
        up, down = [[x + (sign * 0.5 * step if i == which else 0.0) for i, x in enumerate((q, k, v))] for sign in (1, -1)]
        diff = (loss(*up) - loss(*down)).item()                      # linear in each of the three: exact but for roundings
        want = (grad.double() * step.double()).sum().item()
        # both are sums of at most 90 * 3 * 64 products whose factors are fp32 results of sums of some hundred terms
        mass = (grad.double() * step.double()).abs().sum().item()
        total = abs(loss(*up).item()) + abs(loss(*down).item())
        assert abs(diff - want) <= 2.0 ** -24 * 600 * (mass + total), which
    # the other branch reads the same turned keys: a prompt into the paged cache, one more token, and the window operator over both
    x = [t.to(torch.bfloat16) for t in (a, b, v)]
    cache = G.PagedCache.empty(8, 16, H, d, B, 8)
    cache.table.copy_(torch.arange(8, dtype=torch.int32, device="cuda").view(1, 8))
    cache.lengths.fill_(n)
    cache.write(x[1], x[2])
    out, _ = cache.attend(x[0])
    want, _ = G.window_attention(*x, right=0, layout="bnhd")
    assert torch.allclose(out.float(), want.float(), rtol=2.0 ** -6, atol=2.0 ** -6)


# ---- streams, graphs, repeats ------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("n", [1, 400])
def test_streams_and_captured_graphs(n):
    """A training step on a stream of its own, captured while an eager one lives, replayed with eager work in between; two graphs side by side."""
    import torch
    from paper_2510_08318_amd import torch_glue as G
    q, k, v, do, s, ds = _make("bf16", 2, 4, 2, n, 64, "bnhd", 10)
    g = _decays(4)

    def step():
        out, end = G.decay_attention(q, k, v, g, state=s, layout="bnhd")
        return (out, end, *G.decay_attention_backward(q, k, v, g, do, state=s, dstate=ds, layout="bnhd"))

    eager = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = []
    with torch.cuda.stream(side):
        got = step()
        for _ in range(2):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                held = step()
            graphs.append((graph, held))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, eager))
    other = torch.cuda.Stream()
    for i in range(3):
        q.mul_(1.0 + 0.25 * i)
        s.add_(0.5 * i)
        torch.cuda.synchronize()
        graphs[0][0].replay()
        with torch.cuda.stream(other):
            graphs[1][0].replay()
        now = step()
        torch.cuda.synchronize()
        for _, held in graphs:
            assert all(torch.equal(a, b) for a, b in zip(held, now)), i


@pytest.mark.parametrize("mode", MODES)
def test_results_repeat(mode):
    import torch
    from paper_2510_08318_amd import torch_glue as G
    q, k, v, do, s, ds = _make(mode, 2, 6, 2, 900, 64, "bhnd", 11)
    runs = []
    for _ in range(3):
        junk = torch.full((1 << 22,), float("nan"), device="cuda")      # what a workspace may hold
        del junk
        runs.append((*G.decay_attention(q, k, v, _decays(6), state=s, f32_math=mode == "f32math"),
                     *G.decay_attention_backward(q, k, v, _decays(6), do, state=s, dstate=ds, f32_math=mode == "f32math")))
    for r in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(runs[0], r))
