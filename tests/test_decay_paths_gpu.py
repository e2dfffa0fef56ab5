"""linattn_decay_* where real calls go: segments of several chunks, one segment of many chunks, the ends of the token-by-token form, a layer's full size, all by 2-norms
(test_decay_norms_gpu.py); and infinities and NaN that pass from chunk to chunk and from segment to segment, what they reach and what they do not."""
import pytest

from tests.test_decay_norms_gpu import MODES, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("state", [False, True])
def test_one_segment_of_many_chunks(mode, d, state):
    """512 heads fill the chip: a workgroup takes a head's 16 or 32 chunks, the last partial, and hands the state out."""
    check(mode, 16, 32, 32, 1000, d, "bnhd" if state else "bhnd", state=state, heads=[(0, 0), (0, 1), (3, 12), (15, 28), (15, 31)], segments=(1, 1))


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("d", [64, 128])
def test_one_segment_padded_with_shared_heads(mode, d):
    lengths = [1000, 0, 1, 63, 64, 65, 127, 128, 129, 500, 960, 961, 992, 999, 33, 32]
    check(mode, 16, 32, 8, 1000, d, "bnhd", lengths=lengths, heads=[(b, j) for b in (0, 2, 4, 5, 9, 10, 11, 13, 15) for j in (b % 8,)], segments=(1, 1))


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("state", [False, True])
def test_segments_of_several_chunks(mode, d, state):
    check(mode, 2, 12, 4, 4133, d, "bhnd" if state else "bnhd", lengths=[4133, 2817], state=state, heads=[(0, 0), (1, 1), (1, 3)], segments=(9, 40))


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("d", [64, 128])
def test_segments_of_a_batch(mode, d):
    """Lengths at a segment's end, one before it and one behind it, where segments are of 4, 5, 8 or 10 chunks."""
    check(mode, 4, 16, 16, 2500, d, lengths=[2500, 1280, 1279, 1281], heads=[(b, 4 * b + x) for b in range(4) for x in (0, 3)], segments=(4, 16))


@pytest.mark.parametrize("mode,n", [("bf16", 8), ("bf16", 9), ("f32", 12), ("f32", 13), ("f32", 31), ("f32", 32), ("f32math", 16), ("f32math", 17), ("f32math", 63)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("state", [False, True])
def test_ends_of_the_token_by_token_form(mode, n, d, state):
    check(mode, 3, 5, 5, n, d, "bnhd", lengths=[n, n - 1, 1], state=state)
    check(mode, 70, 8, 4, n, d, state=state, heads=[(0, 0), (33, 2), (69, 3)])


@pytest.mark.parametrize("mode", MODES)
def test_full_size(mode):
    """A layer's size at 832x480, with more heads than the last-level cache has room for in bf16: every row of some heads."""
    check(mode, 1, 18, 18, 32760, 128, state=mode == "bf16", heads=[(0, 0), (0, 7), (0, 16)])


# ---- infinities and NaN ------------------------------------------------------------------------------------------------------

# relative 2-norm of what one of them does not reach, beside the same call without it.  A row's own chunk may then be worked out pair by pair: bf16 results go to the next value where
# that moves them over the middle between two, which happens to few (a move of 2^-16 on a step of 2^-8), so that 2^-10 is far above; fp32 sums in another order, SUMS of test_decay_norms_gpu.py twice
APART = {"bf16": 2.0 ** -10, "f32math": 2.0 ** -10, "f32": 2.0 ** -17}


def _reach(which, at, n, ch):
    """Elements of a result that a value in channel `ch` of token `at` of q, k, v or dout reaches: {name: (rows, channels)}; None: all."""
    after, before = slice(at, None), slice(0, at + 1)
    return {"q": dict(out=(slice(at, at + 1), None), dk=(before, ch), dv=(before, None), dstate=(ch, None)),
            "k": dict(out=(after, None), dq=(after, ch), dv=(slice(at, at + 1), None), state=(ch, None)),
            "v": dict(out=(after, ch), dq=(after, None), dk=(slice(at, at + 1), None), state=(None, ch)),
            "do": dict(dq=(slice(at, at + 1), None), dk=(before, None), dv=(before, ch), dstate=(None, ch))}[which]


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,H,n,at", [(1, 2, 900, 0), (1, 2, 900, 63), (1, 2, 900, 500), (1, 2, 900, 899), (2, 12, 1500, 700), (8, 64, 300, 130), (8, 64, 300, 299), (1, 2, 7, 3)])
def test_what_is_not_finite(mode, d, B, H, n, at):
    import torch
    from paper_2510_08318_amd import torch_glue as G
    gen = torch.Generator(device="cuda").manual_seed(at + n)
    dt = torch.float32 if mode == "f32" else torch.bfloat16
    q, k, v, do = [torch.randn((B, H, n, d), generator=gen, device="cuda").to(dt) for _ in range(4)]
    s, ds = [torch.randn((B, H, d, d), generator=gen, device="cuda") for _ in range(2)]
    g = torch.tensor([(-0.001, -0.3)[h % 2] for h in range(H)], device="cuda")
    kw = dict(state=s, f32_math=mode == "f32math")

    def run(x):
        out, end = G.decay_attention(x["q"], x["k"], x["v"], g, **kw)
        dq, dk, dv, first = G.decay_attention_backward(x["q"], x["k"], x["v"], g, x["do"], dstate=ds, **kw)
        return dict(out=out, state=end, dq=dq, dk=dk, dv=dv, dstate=first)

    b, h = B - 1, 1
    for which, value, ch in (("q", "nan", 3), ("q", "inf", d - 1), ("k", "-inf", 33), ("k", "nan", 0), ("v", "inf", d // 2 + 5), ("v", "nan", 2), ("do", "nan", d - 9), ("do", "inf", 17)):
        x = dict(q=q, k=k, v=v, do=do)
        old = x[which][b, h, at, ch].clone()
        x[which][b, h, at, ch] = 0.0
        want = run(x)
        x[which][b, h, at, ch] = float(value)
        got = run(x)
        x[which][b, h, at, ch] = old
        reach = _reach(which, at, n, ch)
        for name in got:
            a, c = got[name], want[name]
            assert torch.isfinite(c).all()
            others = torch.ones((B, H), dtype=torch.bool)
            others[b, h] = False
            assert torch.equal(a[others.cuda()], c[others.cuda()]), (name, which, value)
            a, c = a[b, h].double(), c[b, h].double()
            hit = torch.zeros(a.shape, dtype=torch.bool, device="cuda")
            if name in reach:
                rows, columns = [slice(None) if i is None else i for i in reach[name]]
                hit[rows, columns] = True
            assert not torch.isfinite(a[hit]).any(), (name, which, value)
            clear, whole = a[~hit], c[~hit]
            assert torch.isfinite(clear).all(), (name, which, value)
            assert (clear - whole).norm() <= APART[mode] * whole.norm(), (name, which, value, ((clear - whole).norm() / whole.norm()).item())


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("n", [5, 300, 1500])
def test_states_that_are_not_finite(mode, n):
    """A NaN in the state that came before reaches its column of every row, an infinity in dstate its own; other heads and columns stay."""
    import torch
    from paper_2510_08318_amd import torch_glue as G
    H, d = 3, 128
    gen = torch.Generator(device="cuda").manual_seed(n)
    dt = torch.float32 if mode == "f32" else torch.bfloat16
    q, k, v, do = [torch.randn((1, H, n, d), generator=gen, device="cuda").to(dt) for _ in range(4)]
    g = torch.tensor([-0.001, -0.01, -0.0003], device="cuda")
    s, ds = [torch.randn((1, H, d, d), generator=gen, device="cuda") for _ in range(2)]
    s[0, 1, 40, 70], ds[0, 2, 100, 5] = float("nan"), float("inf")
    kw = dict(f32_math=mode == "f32math")
    out, end = G.decay_attention(q, k, v, g, state=s, **kw)
    dq, dk, dv, first = G.decay_attention_backward(q, k, v, g, do, state=s, dstate=ds, **kw)

    def only(x, rows, columns, head):
        bad = ~torch.isfinite(x[0])
        want = torch.zeros_like(bad)
        want[head][rows, columns] = True
        assert torch.equal(bad, want)
    every = slice(None)
    only(out, every, 70, 1)
    only(end, 40, 70, 1)
    only(dq, every, 40, 1)
    only(dk, every, 100, 2)
    only(dv, every, 5, 2)
    only(first, 100, 5, 2)
