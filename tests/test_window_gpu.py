"""Softmax attention with a sliding window and first tokens (linattn_window_fwd, linattn_window_bwd) against the fp64 definition, element by
element, inside bounds that count the roundings (oracle/softmax_oracle.py)."""
import numpy as np
import pytest

from oracle import softmax_oracle as S

pytestmark = pytest.mark.gpu

U = {"bf16": 2.0 ** -8, "f32math": 2.0 ** -8, "f32": 2.0 ** -24}
OPERAND = {"bf16": 2.0 ** -8, "f32math": 2.0 ** -22, "f32": 2.0 ** -22}      # what P and dS lose as operands


def _make(mode, B, H, HK, n, d, layout, seed, scale=1.0):
    import torch
    gen = torch.Generator().manual_seed(seed)
    dt = torch.float32 if mode == "f32" else torch.bfloat16

    def t(heads, mul):
        x = (torch.randn((B, heads, n, d), generator=gen) * mul).to(dt)
        return (x.transpose(1, 2) if layout == "bnhd" else x).contiguous().cuda()
    return t(H, scale), t(HK, scale), t(HK, 1.0), t(H, 0.1)


def _host(x, layout):
    from paper_2510_08318_amd import torch_glue as G
    a = G.to_host_f64(x)
    return np.swapaxes(a, 1, 2) if layout == "bnhd" else a


def _inside(name, got, want, bound, extra=1e-30):
    assert np.isfinite(got).all() == np.isfinite(want).all(), name
    over = np.abs(got - want) - bound - extra
    assert (over <= 0).all(), (name, np.unravel_index(over.argmax(), over.shape), over.max())


def _check(mode, B, H, HK, n, d, left, right, sinks, layout="bhnd", lengths=None, seed=1, train=True, scale=0.0, values=1.0, edit=None):
    """edit(q, k, v, dout): changes to tokens that no result may depend on."""
    import torch
    from paper_2510_08318_amd import torch_glue as G
    q, k, v, do = _make(mode, B, H, HK, n, d, layout, seed, values)
    hq, hk, hv, hd = [_host(x, layout) for x in (q, k, v, do)]
    if edit:
        edit(q, k, v, do)
    L = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    kw = dict(left=left, right=right, sinks=sinks, layout=layout, lengths=L, f32_math=mode == "f32math", scale=scale)
    out, lse = G.window_attention(q, k, v, **kw)
    grads = G.window_attention_backward(q, k, v, out, lse, do, **kw) if train else []
    torch.cuda.synchronize()
    got = [_host(x, layout) for x in (out, *grads)]
    lse = G.to_host_f64(lse)
    u, op, c = U[mode], OPERAND[mode], scale or d ** -0.5
    for b in range(B):
        length = n if lengths is None else lengths[b]
        ok = S.seen(range(n), range(n), length, left, right, sinks)
        ok[length:] = False
        live = np.arange(n) < length
        dk, dv, bk, bv = np.zeros((HK, n, d)), np.zeros((HK, n, d)), np.zeros((HK, n, d)), np.zeros((HK, n, d))
        for h in range(H):
            g = h // (H // HK)
            args = (hq[b, h] * live[:, None], hk[b, g], hv[b, g], ok, c)
            o, l, _ = S.forward(*args)
            bo, bl = S.forward_bounds(*args, op)
            _inside(f"out {b} {h}", got[0][b, h], o, bo + u * np.abs(o))
            assert np.array_equal(np.isneginf(lse[b, h]), np.isneginf(l)), (b, h)
            some = np.isfinite(l)
            _inside(f"lse {b} {h}", lse[b, h][some], l[some], bl[some])
            assert (got[0][b, h][~some] == 0).all()
            if not train:
                continue
            dout = hd[b, h] * live[:, None]
            rq, rk, rv = S.backward(*args, dout)
            eq, ek, ev = S.backward_bounds(*args, dout, op, u)
            _inside(f"dq {b} {h}", got[1][b, h], rq, eq + u * np.abs(rq))
            dk[g] += rk; dv[g] += rv; bk[g] += ek; bv[g] += ev
        if train:
            _inside(f"dk {b}", got[2][b], dk, bk + u * np.abs(dk))
            _inside(f"dv {b}", got[3][b], dv, bv + u * np.abs(dv))


MODES = ("bf16", "f32", "f32math")
SIGHTS = [(-1, -1, 0), (-1, 0, 0), (7, 0, 0), (0, 0, 0), (40, 25, 3), (0, 90, 70), (100, 0, 200), (1, -1, 5)]


@pytest.mark.parametrize("left,right,sinks", SIGHTS)
@pytest.mark.parametrize("n", [1, 2, 31, 64, 65, 130, 333])
def test_bf16_windows_and_lengths(n, left, right, sinks):
    _check("bf16", 1, 2, 2, n, 128, left, right, sinks)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("layout", ["bhnd", "bnhd"])
@pytest.mark.parametrize("left,right,sinks", [(-1, 0, 0), (50, 30, 4), (20, 0, 90)])
def test_types_widths_and_layouts(mode, d, layout, left, right, sinks):
    _check(mode, 2, 4, 2, 210, d, left, right, sinks, layout)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("left,right,sinks", [(-1, -1, 0), (33, 0, 2)])
def test_padded_batch(mode, left, right, sinks):
    """Items of no token, of one, of all; the padding holds NaN."""
    lengths = [0, 1, 97, 150, 64]

    def edit(q, k, v, do):
        for t in (q, k, v, do):
            for b, length in enumerate(lengths):
                t[b, :, length:] = float("nan")
    _check(mode, 5, 3, 3, 150, 64, left, right, sinks, lengths=lengths, edit=edit)


@pytest.mark.parametrize("H,HK", [(8, 1), (6, 3), (7, 7)])
def test_shared_key_heads(H, HK):
    _check("bf16", 1, H, HK, 280, 64, 60, 0, 5, "bnhd")


@pytest.mark.parametrize("left,right,sinks", SIGHTS)
@pytest.mark.parametrize("n", [31, 64, 130, 200])
def test_bf16_many_heads(n, left, right, sinks):
    """As many blocks as have the forward take rows, not keys, to a wavefront; items of unlike lengths."""
    _check("bf16", 10, 16, 8, n, 64, left, right, sinks, "bnhd", lengths=[n, 1, n // 2, n, n, n - 1, 0, n, n, 7 % n])


@pytest.mark.parametrize("d", [64, 128])
def test_bf16_many_heads_longer(d):
    _check("bf16", 3, 12, 12, 1000, d, 300, 0, 70)


@pytest.mark.parametrize("n,left,right,sinks", [(700, 150, 150, 40), (900, -1, 0, 0), (1100, 300, 0, 130)])
@pytest.mark.parametrize("d", [64, 128])
def test_longer_sequences(n, left, right, sinks, d):
    _check("bf16", 1, 2, 1, n, d, left, right, sinks)


@pytest.mark.parametrize("mode", MODES)
def test_first_tokens_that_everything_sees(mode):
    """Most of the first tokens' gradient comes from outside their window."""
    _check(mode, 1, 2, 2, 900 if mode == "bf16" else 400, 64, 10, 10, 70)


@pytest.mark.parametrize("mode", MODES)
def test_sharp_scores(mode):
    """Scores up to a few hundred: most probabilities vanish, the running maximum moves a lot."""
    _check(mode, 1, 2, 2, 300, 64, -1, 0, 0, values=4.0, scale=0.5)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_tokens_out_of_sight_do_not_matter(mode, value):
    """A window of 20 to the left: tokens from 200 on see nothing before 180, tokens before 100 nothing from 100 on (right = 0)."""
    import torch
    from paper_2510_08318_amd import torch_glue as G
    for d in (64, 128):
        q, k, v, do = _make(mode, 1, 2, 2, 260, d, "bhnd", 3)
        kw = dict(left=20, right=0, sinks=2, f32_math=mode == "f32math")
        out, lse = G.window_attention(q, k, v, **kw)
        grads = G.window_attention_backward(q, k, v, out, lse, do, **kw)
        bad = [t.clone() for t in (q, k, v, do)]
        for t in bad:
            t[:, :, 100:110] = value
        out2, lse2 = G.window_attention(*bad[:3], **kw)
        grads2 = G.window_attention_backward(*bad[:3], out2, lse2, bad[3], **kw)
        torch.cuda.synchronize()
        # rows that see one of the tokens 100..109: 100..129; keys that those see: 80.. and the first two
        for a, b, rows in ((out, out2, (100, 130)), (lse, lse2, (100, 130)), (grads[0], grads2[0], (100, 130))):
            keep = [i for i in range(260) if not rows[0] <= i < rows[1]]
            assert torch.isfinite(b[:, :, keep]).all()
            assert (a[:, :, keep].float() - b[:, :, keep].float()).abs().max() <= 2e-2 * a.float().abs().max()
        assert not torch.isfinite(out2[:, :, 100:130]).all(-1).any()
        for a, b in zip(grads[1:], grads2[1:]):
            keep = [j for j in range(2, 260) if not 80 <= j < 130]
            assert torch.isfinite(b[:, :, keep]).all()
            assert (a[:, :, keep].float() - b[:, :, keep].float()).abs().max() <= 2e-2 * a.float().abs().max()


def test_results_repeat_bit_for_bit():
    import torch
    from paper_2510_08318_amd import torch_glue as G
    q, k, v, do = _make("bf16", 2, 4, 2, 500, 128, "bhnd", 9)
    kw = dict(left=100, right=20, sinks=80)
    first = None
    for _ in range(3):
        out, lse = G.window_attention(q, k, v, **kw)
        res = [out, lse, *G.window_attention_backward(q, k, v, out, lse, do, **kw)]
        torch.cuda.synchronize()
        first = first or [t.clone() for t in res]
        assert all(torch.equal(a, b) for a, b in zip(first, res))


def test_captured_forward_and_backward_replay():
    """Two graphs and eager calls of the same leaves, replayed in turn: scratch is not shared."""
    import torch
    from paper_2510_08318_amd import torch_glue as G
    sets = [_make("bf16", 1, 3, 3, n, 64, "bhnd", 20 + n) for n in (300, 190)]
    kw = dict(left=60, right=0, sinks=70)

    def step(q, k, v, do):
        out, lse = G.window_attention(q, k, v, **kw)
        return [out, lse, *G.window_attention_backward(q, k, v, out, lse, do, **kw)]
    graphs, outs = [], []
    for s in sets:
        step(*s)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step(*s))
        graphs.append(g)
    for rep in range(4):
        for s in sets:
            for t in s:
                t.copy_(torch.roll(t, 1, 2))
        eager = [step(*s) for s in sets]
        for o in outs:
            for t in o:
                t.zero_()
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager, outs):
            assert all(torch.equal(x, y) for x, y in zip(a, b)), rep


def test_two_streams_at_once():
    import torch
    from paper_2510_08318_amd import torch_glue as G
    sets = [_make("bf16", 1, 4, 4, 600, 128, "bhnd", 30 + i) for i in range(2)]
    kw = dict(left=200, right=0, sinks=100)

    def step(q, k, v, do):
        out, lse = G.window_attention(q, k, v, **kw)
        return [out, lse, *G.window_attention_backward(q, k, v, out, lse, do, **kw)]
    want = [[t.clone() for t in step(*s)] for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(3):
        got = []
        for st, s in zip(streams, sets):
            with torch.cuda.stream(st):
                got.append(step(*s))
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_the_softmax_branch_of_a_mixed_layer():
    """Eq. 6 with this branch: its output goes in as blend_in, its upstream gradient is r times the layer's."""
    import torch
    from oracle import linattn_oracle as O
    from paper_2510_08318_amd import synth, torch_glue as G
    x = synth.generate("C5", n=300, H=2, d=64)
    q, k, v, do = [G.to_device(t) for t in (x.q, x.k, x.v, x.dout)]
    lay = G.Layer(G.to_device(x.wq), G.to_device(x.wk), x.B, x.n)
    r = 0.4
    kw = dict(left=40, right=40, sinks=8)
    s, lse = G.window_attention(q, k, v, **kw)
    rd, dr = torch.tensor([r], device="cuda"), torch.zeros(1, device="cuda")
    lay.set_blend(s, rd, dr)
    out = lay.forward(q, k, v)
    linear = lay.backward(q, k, v, do)
    soft = G.window_attention_backward(q, k, v, s, lse, (r * do.float()).to(do.dtype), **kw)
    torch.cuda.synchronize()
    lay.close()
    hq, hk, hv, hd = [O.to_f64(t) for t in (x.q, x.k, x.v, x.dout)]
    ok = S.seen(range(300), range(300), 300, 40, 40, 8)
    ref = np.stack([S.forward(hq[0, h], hk[0, h], hv[0, h], ok, 64 ** -0.5)[0] for h in range(2)])[None]
    blend = O.blend_fwd_bh(x.q, x.k, x.v, x.wq, x.wk, ref, r)
    assert O.err_metric(G.to_host_f64(out), blend)[0] <= 1e-2
    want = O.blend_bwd_bh(x.q, x.k, x.v, x.wq, x.wk, ref, r, x.dout)[:3]
    for i in range(3):
        sm = np.stack([S.backward(hq[0, h], hk[0, h], hv[0, h], ok, 64 ** -0.5, r * hd[0, h])[i] for h in range(2)])[None]
        total = G.to_host_f64(linear[i]) + G.to_host_f64(soft[i])
        scale = np.sqrt(np.mean(want[i] ** 2)) + np.sqrt(np.mean(sm ** 2))
        assert np.abs(total - want[i] - sm).max() <= 1e-2 * max(np.abs(want[i]).max() + np.abs(sm).max(), scale)


@pytest.mark.parametrize("mode", MODES)
def test_without_lse_and_without_workspace(mode):
    """The ABI's optional arguments: the forward without lse, and (fp32) without the workspace that its shared blocks need."""
    import torch
    from paper_2510_08318_amd import binding as L, torch_glue as G
    q, k, v, _ = _make(mode, 2, 2, 2, 100, 64, "bhnd", 3)
    kw = dict(left=30, right=0, sinks=2, f32_math=mode == "f32math")
    want, _ = G.window_attention(q, k, v, **kw)
    dtype = {"bf16": L.BF16, "f32math": L.BF16_F32MATH, "f32": L.F32}[mode]
    desc = L.WindowDesc(dtype, 2, 2, 2, 100, 64, 0, L.Sight(30, 0, 2, 0.0), None, None, 0)
    out = torch.empty_like(q)
    L.linattn_window_fwd(desc, q, k, v, out, None, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert (out.float() - want.float()).abs().max() <= 2 * U[mode] * want.float().abs().max()


def test_the_glue_refuses_what_the_library_cannot_see():
    import torch
    from paper_2510_08318_amd import binding as L, torch_glue as G
    q, k, v, do = _make("bf16", 1, 2, 2, 40, 64, "bhnd", 3)
    out, lse = G.window_attention(q, k, v)
    bad = [dict(q=q.transpose(1, 2)), dict(q=q.half()), dict(k=k.float()), dict(v=v[:, :, :20]), dict(k=k[:, :1]), dict(v=v.cpu()), dict(q=q[0])]
    for change in bad:
        with pytest.raises((ValueError, L.LinattnError)):
            G.window_attention(**{**dict(q=q, k=k, v=v), **change})
    for kw in (dict(layout="nbhd"), dict(lengths=torch.tensor([40], device="cuda")), dict(lengths=torch.tensor([40, 40], dtype=torch.int32, device="cuda")),
               dict(out=q.float()), dict(lse=lse[:, :1]), dict(sinks=-1), dict(scale=-1.0)):
        with pytest.raises((ValueError, L.LinattnError)):
            G.window_attention(q, k, v, **kw)
    for args in ((q, k, v, out.float(), lse, do), (q, k, v, out, lse[:, :1], do), (q, k, v, out, lse.double(), do), (q, k, v, out, lse, do[:, :, :3])):
        with pytest.raises(ValueError):
            G.window_attention_backward(*args)


def test_offsets_past_32_bits():
    """600000 tokens of 32 heads, 4.9 GB a tensor: the last tokens' results are those of the last tokens alone."""
    import torch
    from paper_2510_08318_amd import torch_glue as G
    n, H, d, tail = 600_000, 32, 128, 400
    gen = torch.Generator(device="cuda").manual_seed(1)
    ts = []
    for _ in range(4):
        t = torch.empty((1, n, H, d), dtype=torch.bfloat16, device="cuda")
        t.normal_(generator=gen)
        ts.append(t)
    q, k, v, do = ts
    kw = dict(left=60, right=0, layout="bnhd")
    out, lse = G.window_attention(q, k, v, **kw)
    grads = G.window_attention_backward(q, k, v, out, lse, do, **kw)
    s = [t[:, -tail:].contiguous() for t in ts]
    out2, lse2 = G.window_attention(*s[:3], **kw)
    grads2 = G.window_attention_backward(*s[:3], out2, lse2, s[3], **kw)
    torch.cuda.synchronize()
    assert (lse[:, :, -300:] - lse2[:, :, -300:]).abs().max() <= 1e-4
    for a, b in zip((out, *grads), (out2, *grads2)):
        x, y = a[:, -300:].float(), b[:, -300:].float()
        # two roundings of operands and one of the result on each side, of numbers as large as the largest
        assert (x - y).abs().max() <= 6 * 2.0 ** -8 * y.abs().max()


def test_inputs_made_on_another_stream():
    """The calls run on the current stream, after what it waited for."""
    import torch
    from paper_2510_08318_amd import torch_glue as G
    q, k, v, _ = _make("bf16", 1, 4, 4, 500, 64, "bhnd", 8)
    want, _ = G.window_attention(q, k, v, left=100)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(side):
            side.wait_stream(torch.cuda.default_stream())
            k2 = (k.float() * 2 - k.float()).to(k.dtype)
            got, _ = G.window_attention(q, k2, v, left=100)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(want, got)


def test_inputs_that_require_a_gradient():
    """Nothing is recorded for autograd: the same results, without a gradient; a Function around the two calls has autograd give what the backward call does."""
    import torch
    from paper_2510_08318_amd import torch_glue as G
    q, k, v, do = _make("bf16", 1, 2, 2, 100, 64, "bhnd", 3)
    kw = dict(left=30, right=0)
    out, lse = G.window_attention(q, k, v, **kw)
    grads = G.window_attention_backward(q, k, v, out, lse, do, **kw)

    class Recorded(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, v):
            out, lse = G.window_attention(q, k, v, **kw)
            ctx.save_for_backward(q, k, v, out, lse)
            return out

        @staticmethod
        def backward(ctx, dout):
            return G.window_attention_backward(*ctx.saved_tensors, dout.contiguous(), **kw)
    leaves = [t.clone().requires_grad_() for t in (q, k, v)]
    got, _ = G.window_attention(*leaves, **kw)
    assert torch.equal(got, out) and not got.requires_grad
    Recorded.apply(*leaves).backward(do)
    torch.cuda.synchronize()
    assert all(torch.equal(t.grad, g) for t, g in zip(leaves, grads))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,HK", [(4, 4), (8, 4), (8, 2)])
def test_f32_blocks_of_their_own(H, HK, d):
    """So many blocks of 32 rows that each has one workgroup, which stores its results itself; with eight heads on two, of the query side only.  A padded
    item, whose padding holds NaN."""
    lengths = [600, 333]

    def edit(q, k, v, do):
        for t in (q, k, v, do):
            t[1, :, 333:] = float("nan")
    _check("f32", 2, H, HK, 600, d, 100, 20, 5, lengths=lengths, edit=edit)


def _check_out_of_sight(mode, B, H, HK, n, d, left, right, sinks, bad, value):
    """Tokens `bad` hold `value` in q, k, v and dout: whatever does not depend on them is what it is without them, whatever does is not finite."""
    import torch
    from paper_2510_08318_amd import torch_glue as G
    q, k, v, do = _make(mode, B, H, HK, n, d, "bhnd", 6)
    hq, hk, hv, hd = [_host(x, "bhnd") for x in (q, k, v, do)]
    for t in (q, k, v, do):
        t[:, :, bad] = value
    kw = dict(left=left, right=right, sinks=sinks, f32_math=mode == "f32math")
    out, lse = G.window_attention(q, k, v, **kw)
    grads = G.window_attention_backward(q, k, v, out, lse, do, **kw)
    torch.cuda.synchronize()
    got, lse = [_host(x, "bhnd") for x in (out, *grads)], G.to_host_f64(lse)
    ok = S.seen(range(n), range(n), n, left, right, sinks)
    rows = ~ok[:, bad].any(1)                  # rows that see no such token, and keys that only such rows see
    keys = ~ok[~rows].any(0)
    assert 40 < rows.sum() < n and 40 < keys.sum() < n
    u, op = U[mode], OPERAND[mode]
    for b in range(B):
        sums = [np.zeros((HK, n, d)) for _ in range(4)]
        for h in range(H):
            g = h // (H // HK)
            args, dout = (hq[b, h], hk[b, g], hv[b, g], ok, d ** -0.5), hd[b, h]
            o, l, _ = S.forward(*args)
            bo, bl = S.forward_bounds(*args, op)
            _inside(f"out {b} {h}", got[0][b, h][rows], o[rows], (bo + u * np.abs(o))[rows])
            _inside(f"lse {b} {h}", lse[b, h][rows], l[rows], bl[rows])
            assert not np.isfinite(got[0][b, h][~rows]).all(-1).any()
            grad, bound = S.backward(*args, dout), S.backward_bounds(*args, dout, op, u)
            _inside(f"dq {b} {h}", got[1][b, h][rows], grad[0][rows], (bound[0] + u * np.abs(grad[0]))[rows])
            for i, x in enumerate((grad[1], grad[2], bound[1], bound[2])):
                sums[i][g] += x
        for g in range(HK):
            for i, name in enumerate(("dk", "dv")):
                _inside(f"{name} {b} {g}", got[2 + i][b, g][keys], sums[i][g][keys], (sums[2 + i][g] + u * np.abs(sums[i][g]))[keys])


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("d", [64, 128])
def test_tokens_out_of_sight_of_long_windows(mode, d, value):
    """Windows of more than 256 keys, key blocks that several workgroups share, of first tokens and of the window: rows and keys next to tokens that they do not
    see are done again from the stored output's row sums, and into the parts of a sum."""
    _check_out_of_sight(mode, 1, 4, 2, 900, d, 300, 0, 0, slice(450, 453), value)
    _check_out_of_sight(mode, 1, 4, 2, 900, d, 290, 30, 0, slice(560, 570), value)
    _check_out_of_sight(mode, 1, 4, 2, 900, d, 300, 0, 70, slice(450, 453), value)


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("d", [64, 128])
def test_f32_tokens_out_of_sight_of_many_blocks(d, value):
    """As many blocks as have one workgroup each do such rows again themselves."""
    _check_out_of_sight("f32", 2, 4, 4, 600, d, 90, 10, 0, slice(300, 304), value)
