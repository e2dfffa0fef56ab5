"""linattn_decay_* at the ends of its sizes: rows behind 2^31 elements, as many heads and sequences as there may be, states that several sequences read."""
import pytest

from tests.test_decay_norms_gpu import BEFORE, _definition, _near

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mode", ["bf16", "f32"])
def test_rows_behind_32_bits(mode):
    """33 million tokens.  The decay forgets 400 tokens (exp(-200)), so that the last rows of out and dq, and the first of dk and dv, are those of a sequence of their own."""
    import torch
    from paper_2510_08318_amd import torch_glue as G
    n, d, m = (1 << 25) + 77, 64, 400
    dt = torch.float32 if mode == "f32" else torch.bfloat16
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, k, v, do = [torch.empty((1, n, 1, d), dtype=dt, device="cuda").normal_(generator=gen) for _ in range(4)]
    g = torch.tensor([-0.5], device="cuda")
    out, end = G.decay_attention(q, k, v, g, layout="bnhd")
    dq, dk, dv, _ = G.decay_attention_backward(q, k, v, g, do, layout="bnhd")
    for part in (slice(n - 2 * m, n), slice(0, 2 * m), slice((1 << 24) - m, (1 << 24) + m)):
        x = [t[0, part, 0].double() for t in (q, k, v, do)]
        w = _definition(*x, -0.5, d ** -0.5, None, None)
        z = _definition(*[t * t for t in x], -1.0, 1 / d, None, None)
        a, b = (0 if part.start == 0 else m), (2 * m if part.stop == n else m)      # rows from a on see 400 tokens before them, rows up to b 400 behind
        for name, got, i in (("out", out, 0), ("dq", dq, 2)):
            _near(name, mode, got[0, part, 0][a:], w[i][a:], z[i][a:], dt, BEFORE[mode])
        for name, got, i in (("dk", dk, 3), ("dv", dv, 4)):
            _near(name, mode, got[0, part, 0][:b], w[i][:b], z[i][:b], dt, BEFORE[mode])
        if part.stop == n:
            _near("state", mode, end[0, 0], w[1], z[1], torch.float32, 2.0 ** -18)
    del q, k, v, do, out, dq, dk, dv
    torch.cuda.empty_cache()


@pytest.mark.parametrize("mode,n", [("bf16", 1), ("bf16", 9), ("f32", 13), ("f32math", 17)])
@pytest.mark.parametrize("B,H,HK", [(1, 65535, 65535), (65535, 1, 1), (32767, 2, 1)])
def test_most_heads_and_sequences(mode, n, B, H, HK):
    """The same bits as calls of a few of them: a chunk and one segment in all of these.  (A single token of few heads is summed in another order, fp32 sums of 64 products, which may
    take a row's store to the next bf16 value, 2^-7.)"""
    import torch
    from paper_2510_08318_amd import torch_glue as G
    d, dt = 64, torch.float32 if mode == "f32" else torch.bfloat16
    gen = torch.Generator(device="cuda").manual_seed(B)

    def t(*shape):
        return torch.empty(shape, dtype=dt, device="cuda").normal_(generator=gen)
    q, k, v, do = t(B, H, n, d), t(B, HK, n, d), t(B, HK, n, d), t(B, H, n, d)
    s, ds = [torch.empty((B, H, d, d), device="cuda").normal_(generator=gen) for _ in range(2)]
    g = -torch.rand((H,), generator=gen, device="cuda")
    kw = dict(f32_math=mode == "f32math")
    out, end = G.decay_attention(q, k, v, g, state=s, **kw)
    grads = G.decay_attention_backward(q, k, v, g, do, state=s, dstate=ds, **kw)
    for i in (0, max(B, H) // 2, max(B, H) - 3):
        b, h = (slice(i, i + 3), slice(None)) if B > 1 else (slice(None), slice(i, i + 3))
        c = lambda x: x[b, h].contiguous()
        a = [c(x) for x in (q, k, v)]
        few, after = G.decay_attention(*a, g[h].contiguous(), state=c(s), **kw)
        same = G.decay_attention_backward(*a, g[h].contiguous(), c(do), state=c(s), dstate=c(ds), **kw)
        assert torch.equal(end[b, h], after), i
        for x, y in zip((out, *grads), (few, *same)):
            assert torch.allclose(x[b, h].float(), y.float(), rtol=2.0 ** -7, atol=2.0 ** -16) if n == 1 else torch.equal(x[b, h], y), i


@pytest.mark.parametrize("n", [1, 40, 700])
def test_a_state_that_several_sequences_read(n):
    """The same slot twice, in calls that write no states: a prompt's continuations, and their gradients, by item."""
    import torch
    from paper_2510_08318_amd import torch_glue as G
    gen = torch.Generator(device="cuda").manual_seed(n)
    q, k, v, do = [torch.randn((4, n, 3, 64), generator=gen, device="cuda").to(torch.bfloat16) for _ in range(4)]
    pool, ds = torch.randn((5, 3, 64, 64), generator=gen, device="cuda"), torch.randn((4, 3, 64, 64), generator=gen, device="cuda")
    slots, g = torch.tensor([2, 2, 0, 2], dtype=torch.int32, device="cuda"), torch.tensor([-0.01, -0.2, 0.0], device="cuda")
    before = pool.clone()
    out, none = G.decay_attention(q, k, v, g, state=pool, slots=slots, state_out=False, layout="bnhd")
    grads = G.decay_attention_backward(q, k, v, g, do, state=pool, dstate=ds, slots=slots, layout="bnhd")
    state = pool[slots.long()]
    want, _ = G.decay_attention(q, k, v, g, state=state, state_out=False, layout="bnhd")
    same = G.decay_attention_backward(q, k, v, g, do, state=state, dstate=ds, layout="bnhd")
    assert none is None and torch.equal(out, want) and all(torch.equal(a, b) for a, b in zip(grads, same)) and torch.equal(pool, before)


def test_two_calls_at_once():
    """Two streams, calls with workspaces, and one state that both read."""
    import torch
    from paper_2510_08318_amd import torch_glue as G
    gen = torch.Generator(device="cuda").manual_seed(4)
    q, k, v, do = [torch.randn((1, 6, 3000, 64), generator=gen, device="cuda").to(torch.bfloat16) for _ in range(4)]
    s, g = torch.randn((1, 6, 64, 64), generator=gen, device="cuda"), torch.full((6,), -0.01, device="cuda")

    def step(q):
        out, end = G.decay_attention(q, k, v, g, state=s)
        return (out, end, *G.decay_attention_backward(q, k, v, g, do, state=s))
    inputs = [q, q * 2, q * 0.5, -q]
    want = [step(x) for x in inputs]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for i in range(12):
        with torch.cuda.stream(streams[i % 2]):
            got.append(step(inputs[i % 4]))
    torch.cuda.synchronize()
    for i, x in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(x, want[i % 4])), i
