"""The paged cache (linattn_cache_write, _read, _attn) against the fp64 definition and against the same steps done by hand."""
import numpy as np
import pytest

from oracle import softmax_oracle as S

pytestmark = pytest.mark.gpu


def _cache(lengths, counts, n, H, d, page, e4m3, layout, seed, spare=2, width=None):
    """A cache whose pages lie in random order, the k and v of all tokens ([B][len, H, d], CPU bf16), and the chunk tensors."""
    import torch
    from paper_2510_08318_amd import torch_glue as G
    gen = torch.Generator().manual_seed(seed)
    B = len(lengths)
    width = width or max(1, -(-max(lengths) // page))
    pages = B * width + spare
    c = G.PagedCache.empty(pages, page, H, d, B, width, quantised=e4m3)
    order = torch.randperm(pages, generator=gen)[: B * width].view(B, width)
    used = torch.arange(width)[None] * page < torch.tensor(lengths)[:, None]
    c.table.copy_(torch.where(used, order, -1).int())
    c.lengths.copy_(torch.tensor(lengths, dtype=torch.int32))
    for t in (c.k, c.v):
        t.view(torch.uint8).fill_(0x7f)                                  # NaN (e4m3), 3.4e38 (bf16): rows that nothing may read
    kv = [[torch.randn((x, H, d), generator=gen).to(torch.bfloat16) for x in lengths] for _ in range(2)]

    def chunk(rows, counts, n, offset):
        x = torch.full((B, n, H, d), float("nan"), dtype=torch.bfloat16)
        for b in range(B):
            lo = lengths[b] - offset[b]
            x[b, : counts[b]] = rows[b][lo: lo + counts[b]]
        return (x.transpose(1, 2) if layout == "bhnd" else x).contiguous().cuda()
    return c, kv, chunk


def _filled(lengths, H, d, page, e4m3, layout, seed, **kw):
    import torch
    n = max(max(lengths), 1)
    c, kv, chunk = _cache(lengths, lengths, n, H, d, page, e4m3, layout, seed, **kw)
    counts = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    c.write(chunk(kv[0], lengths, n, lengths), chunk(kv[1], lengths, n, lengths), counts=counts, layout=layout)
    return c, kv


def _held(x, e4m3):
    """What the cache holds of rows [len, H, d]."""
    a = x.double().numpy()
    if not e4m3:
        return a
    return np.stack([[S.quantise(r)[0] for r in t] for t in a]) if a.size else a


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("layout", ["bhnd", "bnhd"])
@pytest.mark.parametrize("page,d", [(1, 64), (16, 128), (24, 64), (64, 128)])
def test_write_and_read_back(e4m3, layout, page, d):
    from paper_2510_08318_amd import torch_glue as G
    lengths = [0, 1, 37, 64]
    c, kv = _filled(lengths, 3, d, page, e4m3, layout, 5)
    for got, rows in zip(c.read(70, layout=layout), kv):
        got = G.to_host_f64(got)
        got = np.swapaxes(got, 1, 2) if layout == "bhnd" else got
        for b, length in enumerate(lengths):
            assert np.array_equal(got[b, :length], _held(rows[b], e4m3)), b
            assert (got[b, length:] == 0).all()


@pytest.mark.parametrize("e4m3", [False, True])
def test_a_chunk_changes_only_its_own_rows(e4m3):
    """Chunks of 0, 1, 5 and (more than the sequence has) 9 tokens after earlier ones."""
    import torch
    lengths, counts, page = [20, 21, 30, 4], [0, 1, 5, 9], 8
    c, kv, chunk = _cache(lengths, counts, 9, 2, 64, page, e4m3, "bnhd", 7)
    before = [t.clone() for t in (c.k.view(torch.uint8), c.v.view(torch.uint8))]
    x = [torch.randn((4, 9, 2, 64), device="cuda").to(torch.bfloat16) for _ in range(2)]
    c.write(*x, counts=torch.tensor(counts, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    table = c.table.cpu()
    written = torch.zeros((c.pages, c.page), dtype=torch.bool)
    got = c.read(30)
    for b in range(4):
        for t in range(counts[b]):
            j = lengths[b] - counts[b] + t
            if j < 0:
                continue
            written[table[b, j // page], j % page] = True
            for name in range(2):
                want = _held(x[name][b, t: t + 1].cpu(), e4m3)[0]
                assert np.array_equal(got[name][b, j].double().cpu().numpy(), want)
    assert written.sum() == 0 + 1 + 5 + 4
    for old, new in zip(before, (c.k.view(torch.uint8), c.v.view(torch.uint8))):
        same = (old.view(c.pages, 2, page, -1) == new.view(c.pages, 2, page, -1)).all(-1).all(1).cpu()
        assert same[~written].all()


def test_quantised_rows_of_every_magnitude():
    """Every finite bf16 exponent, ties, infinities and NaN, rows of zeros."""
    import torch
    from paper_2510_08318_amd import torch_glue as G
    n, d = 300, 64
    gen = torch.Generator().manual_seed(1)
    x = torch.randn((1, n, 1, d), generator=gen)
    x = (x * torch.exp2(torch.linspace(-140, 126, n))[None, :, None, None]).to(torch.bfloat16)
    x[0, 3] = 0.0
    x[0, 4, 0, 5], x[0, 5, 0, 6], x[0, 6] = float("inf"), float("nan"), float("-inf")
    x[0, 7, 0] = torch.arange(64) / 4 + 448 - 16                          # ties at every other one
    x[0, 8, 0] = 0.0
    x[0, 8, 0, 0] = 3.3895e38
    c = G.PagedCache.empty(n, 1, 1, d, 1, n, quantised=True)
    c.table.copy_(torch.arange(n, dtype=torch.int32)[None])
    c.lengths.fill_(n)
    c.write(x.cuda(), x.cuda())
    k, v = c.read(n)
    want = [S.quantise(r) for r in x[0, :, 0].double().numpy()]
    assert torch.equal(k.view(torch.int16), v.view(torch.int16))
    got = G.to_host_f64(k)[0, :, 0]
    assert np.array_equal(np.stack([w[0] for w in want]), got, equal_nan=True)
    assert [w[1] + 127 for w in want] == c.k_exp[:, 0, 0].tolist() == c.v_exp[:, 0, 0].tolist()


def _attend(lengths, counts, n, H, HK, d, page, e4m3, left, right, sinks, layout, seed=3, holes=()):
    """holes: (b, table entry) that name no page: those keys are not there."""
    import torch
    from paper_2510_08318_amd import torch_glue as G
    c, kv = _filled(lengths, HK, d, page, e4m3, layout, seed)
    for b, i in holes:
        c.table[b, i] = (c.pages, -7)[i % 2]
    gen = torch.Generator().manual_seed(seed + 100)
    B = len(lengths)
    q = torch.randn((B, n, H, d), generator=gen).to(torch.bfloat16)
    real = [min(n, counts[b]) for b in range(B)] if counts is not None else [n] * B
    for b in range(B):
        q[b, real[b]:] = float("nan")
    qd = (q.transpose(1, 2) if layout == "bhnd" else q).contiguous().cuda()
    cd = None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda")
    out, lse = c.attend(qd, counts=cd, left=left, right=right, sinks=sinks, layout=layout)
    torch.cuda.synchronize()
    out, lse = G.to_host_f64(out), G.to_host_f64(lse)
    out = out if layout == "bhnd" else np.swapaxes(out, 1, 2)
    for b in range(B):
        pos = lengths[b] - real[b] + np.arange(n)
        ok = S.seen(pos, range(lengths[b]), lengths[b], left, right, sinks) if lengths[b] else np.zeros((n, 1), bool)
        ok[(np.arange(n) >= real[b]) | (pos < 0)] = False
        for hb, i in holes:
            if hb == b:
                ok[:, i * page: (i + 1) * page] = False
        k, v = [_held(rows[b], e4m3) if lengths[b] else np.zeros((1, HK, d)) for rows in kv]
        for h in range(H):
            g = h // (H // HK)
            x = np.where(((np.arange(n) < real[b]) & (pos >= 0))[:, None], q[b, :, h].double().numpy(), 0.0)
            args = (x, k[:, g], v[:, g], ok, d ** -0.5)
            o, l, _ = S.forward(*args)
            bo, bl = S.forward_bounds(*args, 2.0 ** -8)
            over = np.abs(out[b, h] - o) - bo - 2.0 ** -8 * np.abs(o)
            assert (over <= 0).all(), (b, h, over.max())
            assert np.array_equal(np.isneginf(lse[b, h]), np.isneginf(l)), (b, h)
            some = np.isfinite(l)
            assert (np.abs(lse[b, h][some] - l[some]) <= bl[some]).all()


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("layout", ["bhnd", "bnhd"])
@pytest.mark.parametrize("d,page", [(64, 16), (128, 24), (128, 64)])
@pytest.mark.parametrize("left,right,sinks", [(-1, 0, 0), (40, 0, 3)])
def test_one_token(e4m3, layout, d, page, left, right, sinks):
    _attend([1, 100, 333, 64, 0], [1, 1, 1, 1, 1], 1, 4, 2, d, page, e4m3, left, right, sinks, layout)


@pytest.mark.parametrize("H,HK", [(1, 1), (8, 1), (12, 12), (40, 1)])
@pytest.mark.parametrize("n", [1, 3])
def test_few_rows_and_shared_key_heads(H, HK, n):
    _attend([700, 129], None, n, H, HK, 64, 32, True, -1, 0, 0, "bnhd")


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("n,left,right,sinks", [(40, -1, 0, 0), (40, -1, -1, 0), (100, 30, 0, 5), (150, 64, 20, 70), (17, 0, 0, 0)])
def test_chunks(e4m3, n, left, right, sinks):
    _attend([200, 150, 301], [n, n - 9, 1], n, 4, 2, 128, 16, e4m3, left, right, sinks, "bnhd")


@pytest.mark.parametrize("n", [200, 260])
def test_a_whole_prompt_at_once(n):
    _attend([n, n], None, n, 2, 2, 64, 64, False, -1, 0, 0, "bhnd")


@pytest.mark.parametrize("n,counts", [(1, [1, 1]), (90, [90, 50])])
def test_long_sequences_and_pages_of_odd_size(n, counts):
    _attend([2000, 1601], counts, n, 2, 1, 128, 100, True, -1, 0, 0, "bnhd")


def test_counts_beyond_the_chunk_and_the_sequence():
    """counts is brought into [0, n]; tokens at negative positions are padding."""
    _attend([30, 5, 12], [50, 8, 0], 8, 2, 2, 64, 8, False, -1, 0, 0, "bnhd")


@pytest.mark.parametrize("n", [8, 100])
def test_chunks_longer_than_their_sequences(n):
    """Without counts every sequence has n new tokens; those before its start are padding."""
    _attend([3, 120, 8], None, n, 4, 2, 64, 16, True, 20, 0, 2, "bhnd")


def test_pools_past_32_bits():
    """Pages behind 4 GB of a pool, written, read back and attended to."""
    import torch
    from paper_2510_08318_amd import torch_glue as G
    H, d, page = 8, 128, 128
    pages = 45_000                                                        # 5.9 GB of codes, 46 million exponents
    for quantised in (True, False):
        c = G.PagedCache.empty(pages if quantised else pages // 2, page, H, d, 1, 3, quantised=quantised)
        small = G.PagedCache.empty(3, page, H, d, 1, 3, quantised=quantised)
        c.table.copy_(torch.tensor([[c.pages - 1, c.pages - 7, c.pages - 2]], dtype=torch.int32))
        small.table.copy_(torch.tensor([[2, 0, 1]], dtype=torch.int32))
        gen = torch.Generator(device="cuda").manual_seed(4)
        k, v, q = [torch.randn((1, 300, H, d), device="cuda", generator=gen).to(torch.bfloat16) for _ in range(3)]
        res = []
        for cache in (c, small):
            cache.lengths.fill_(300)
            cache.write(k, v)
            res.append([*cache.read(300), *cache.attend(q, left=100), *cache.attend(q[:, -1:].contiguous())])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(*res))
        del c


def test_the_glue_refuses_what_the_library_cannot_see():
    import torch
    from paper_2510_08318_amd import binding as L, torch_glue as G
    c, _ = _filled([20, 20], 2, 64, 16, True, "bnhd", 3)
    q = torch.zeros((2, 3, 4, 64), dtype=torch.bfloat16, device="cuda")
    k = torch.zeros((2, 3, 2, 64), dtype=torch.bfloat16, device="cuda")
    for bad in (q.float(), q[:1], q[..., :32].contiguous(), q.transpose(1, 2), q[:, :, :3].contiguous()):
        with pytest.raises((ValueError, L.LinattnError)):
            c.attend(bad)
    for bad in (k.float(), k[:1], k[:, :, :1].contiguous(), q):
        with pytest.raises(ValueError):
            c.write(bad, k)
        with pytest.raises(ValueError):
            c.write(k, bad)
    for counts in (torch.zeros(2, dtype=torch.int64, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32)):
        with pytest.raises(ValueError):
            c.write(k, k, counts=counts)
    with pytest.raises(L.LinattnError):
        c.read(0)
    with pytest.raises(ValueError):
        c.read(5, layout="hbnd")
    for change in (dict(table=c.table.long()), dict(lengths=c.lengths[:1]), dict(k_exp=None), dict(v=c.v[:2]), dict(k=c.k.float())):
        with pytest.raises(ValueError):
            G.PagedCache(**{**dict(k=c.k, v=c.v, table=c.table, lengths=c.lengths, k_exp=c.k_exp, v_exp=c.v_exp), **change})


@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("e4m3", [False, True])
def test_table_entries_that_name_no_page(n, e4m3):
    _attend([100, 90], None, n, 2, 1, 64, 16, e4m3, -1, 0, 0, "bnhd", holes=[(0, 0), (0, 3), (1, 1), (1, 2)])


def test_lengths_beyond_the_table_are_brought_into_range():
    import torch
    c, _ = _filled([64, 64], 1, 64, 16, False, "bnhd", 3)
    q = torch.randn((2, 1, 1, 64), device="cuda").to(torch.bfloat16)
    want, _ = c.attend(q)
    k, _ = c.read(64)
    c.lengths.fill_(1000)
    got, _ = c.attend(q)
    k2, _ = c.read(80)
    torch.cuda.synchronize()
    assert torch.equal(want, got) and torch.equal(k, k2[:, :64]) and (k2[:, 64:] == 0).all()
    c.lengths.fill_(-3)
    got, lse = c.attend(q)
    torch.cuda.synchronize()
    assert (got == 0).all() and (lse == -float("inf")).all()


@pytest.mark.parametrize("n", [1, 50])
def test_keys_out_of_sight_do_not_matter(n):
    """A window of 30: NaN in keys and values before it, and behind the causal end, inside the tiles that are read."""
    import torch
    c, _ = _filled([300], 2, 64, 16, False, "bnhd", 3)
    q = torch.randn((1, n, 2, 64), device="cuda").to(torch.bfloat16)
    want, wl = c.attend(q, left=30, right=0)
    at = 300 - n - 31
    for t in (c.k, c.v):
        t[c.table[0, at // 16].item(), :, at % 16] = float("nan")
    got, gl = c.attend(q, left=30, right=0)
    torch.cuda.synchronize()
    assert torch.isfinite(got).all() and (want.float() - got.float()).abs().max() <= 2e-2 * want.float().abs().max()
    assert (wl - gl).abs().max() <= 1e-5
    # the last key is seen by the last query only
    at = 299
    for t in (c.k, c.v):
        t[c.table[0, at // 16].item(), :, at % 16] = float("nan")
    got, _ = c.attend(q, left=30, right=0)
    torch.cuda.synchronize()
    assert torch.isfinite(got[:, :-1]).all() and not torch.isfinite(got[:, -1]).all(-1).any()


@pytest.mark.parametrize("e4m3", [False, True])
def test_generation_chunk_by_chunk_is_one_pass_over_the_sequence(e4m3):
    """Writes and attends chunk after chunk, the last ones single tokens, equal the window operator on the values that the cache holds."""
    import torch
    from paper_2510_08318_amd import torch_glue as G
    total, H, HK, d = 150, 4, 2, 64
    gen = torch.Generator().manual_seed(2)
    q, k, v = [torch.randn((1, total, h, d), generator=gen).to(torch.bfloat16).cuda() for h in (H, HK, HK)]
    c = G.PagedCache.empty(20, 16, HK, d, 1, 10, quantised=e4m3)
    c.table.copy_(torch.randperm(20, generator=gen)[:10].int()[None])
    out, done = torch.empty_like(q), 0
    for n in (70, 40, 30, *[1] * 10):
        sl = slice(done, done + n)
        c.lengths.add_(n)
        c.write(k[:, sl].contiguous(), v[:, sl].contiguous())
        out[:, sl] = c.attend(q[:, sl].contiguous(), left=48, sinks=4)[0]
        done += n
    hk, hv = c.read(total)
    want, _ = G.window_attention(q, hk, hv, left=48, right=0, sinks=4, layout="bnhd")
    torch.cuda.synchronize()
    assert (out.float() - want.float()).abs().max() <= 4 * 2.0 ** -8 * hv.float().abs().max()


def test_captured_steps_replay():
    """A captured step (write, attend) replayed while lengths move on, against eager steps."""
    import torch
    from paper_2510_08318_amd import torch_glue as G
    H, d, B = 2, 64, 3
    caches = []
    for _ in range(2):
        c = G.PagedCache.empty(30, 16, H, d, B, 10, quantised=True)
        c.table.copy_(torch.arange(30, dtype=torch.int32).view(B, 10))
        caches.append(c)
    q, k, v = [torch.randn((B, 1, H, d), device="cuda").to(torch.bfloat16) for _ in range(3)]

    def step(c):
        c.lengths.add_(1)
        c.write(k, v)
        return c.attend(q)
    step(caches[0])
    step(caches[1])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out, lse = step(caches[0])
    for i in range(5):
        for t in (q, k, v):
            t.copy_(torch.roll(t, 1, 1 + i % 3))
        want, wl = step(caches[1])
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(caches[0].lengths, caches[1].lengths)
        assert torch.equal(out, want) and torch.equal(lse, wl), i


@pytest.mark.parametrize("e4m3,d,left,sinks", [(False, 64, -1, 0), (True, 128, -1, 0), (False, 128, 20400, 2)])
def test_long_parts_of_unlike_sequences(e4m3, d, left, sinks):
    """Blocks of rows that fill the chip, over sequences whose keys go in three parts, in two, in one, and an empty one; with a window also a key that is NaN, which a
    hundred of the rows do not see."""
    import torch
    from paper_2510_08318_amd import torch_glue as G
    lengths, n, H, page, width = [24000, 12288, 3000, 0], 1000, 12, 64, 384
    torch.manual_seed(11)
    c = G.PagedCache.empty(4 * width, page, H, d, 4, width, quantised=e4m3)
    c.table.copy_(torch.randperm(4 * width, device="cuda").view(4, width).int())
    c.lengths.copy_(torch.tensor(lengths, dtype=torch.int32))
    counts = c.lengths.clone()
    kv = [torch.randn((4, 24000, H, d), device="cuda").to(torch.bfloat16) for _ in range(2)]
    if left >= 0:
        kv[0][0, 3500, 11] = kv[1][0, 3500, 11] = float("nan")
    c.write(*kv, counts=counts)
    held = c.read(24000)
    q = torch.randn((4, n, H, d), device="cuda").to(torch.bfloat16)
    desc = c._describe("bnhd", None)
    assert G.B_.linattn_cache_workspace_bytes(desc, H, n) == 3 * 4 * H * n * (d + 2) * 4
    out, lse = c.attend(q, left=left, sinks=sinks)
    again, _ = c.attend(q, left=left, sinks=sinks)
    torch.cuda.synchronize()
    assert torch.equal(out.view(torch.int16), again.view(torch.int16))
    rows = np.arange(0, n, 9)
    for b, length in enumerate(lengths):
        if length == 0:
            assert (out[b] == 0).all() and torch.isneginf(lse[b]).all()
            continue
        pos = length - n + rows
        ok = S.seen(pos, range(length), length, left, 0, sinks)
        for h in (0, 11):
            x = q[b, rows, h].double().cpu().numpy()
            k, v = [t[b, :length, h].double().cpu().numpy() for t in held]
            got, gl = out[b, rows, h].double().cpu().numpy(), lse[b, h, rows].double().cpu().numpy()
            sound = np.ones(len(rows), bool)
            if left >= 0 and b == 0 and h == 11:
                sound = ~ok[:, 3500]
                assert 5 < sound.sum() < 20 and np.isnan(got[~sound]).all() and np.isfinite(got[sound]).all()
            args = (x[sound], k, v, ok[sound], d ** -0.5)
            o, l, _ = S.forward(*args)
            bo, bl = S.forward_bounds(*args, 2.0 ** -8)
            over = np.abs(got[sound] - o) - bo - 2.0 ** -8 * np.abs(o)
            assert (over <= 0).all(), (b, h, over.max())
            assert (np.abs(gl[sound] - l) <= bl).all(), (b, h)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("layout", ["bhnd", "bnhd"])
def test_writes_past_the_table_are_dropped(e4m3, layout):
    """Chunks of five whose tokens lie past the table's 64 places in part or all: places go by lengths as they are, and no earlier row changes."""
    import torch
    page, H, d, n = 16, 2, 64, 5
    c, _ = _filled([64] * 5, H, d, page, e4m3, layout, 3)
    gen = torch.Generator().manual_seed(8)
    x = [torch.randn((5, n, H, d), generator=gen).to(torch.bfloat16) for _ in range(2)]
    lengths, counts = [65, 67, 69, 1000, 2 ** 31 - 1], [1, 5, 5, 5, 3]
    before = [t.clone() for t in c.read(64)]
    c.lengths.copy_(torch.tensor(lengths, dtype=torch.int32))
    c.write(*[(t.transpose(1, 2) if layout == "bhnd" else t).contiguous().cuda() for t in x], counts=torch.tensor(counts, dtype=torch.int32, device="cuda"),
            layout=layout)
    after = c.read(64)
    torch.cuda.synchronize()
    for name in range(2):
        want = before[name].double().cpu().numpy()
        want[1, 62:] = _held(x[name][1, :2], e4m3)             # positions 62 .. 66 of the second sequence: two have a place
        assert np.array_equal(after[name].double().cpu().numpy(), want)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("n", [1, 12, 100])
@pytest.mark.parametrize("left,right,sinks", [(-1, 0, 0), (20, 0, 3), (20, 40, 0), (7, -1, 0)])
def test_attention_past_the_table_goes_by_position(e4m3, n, left, right, sinks):
    """Queries at positions past the 64 places of the table, some, most or all of a chunk: they see those of the 64 keys that their window still reaches."""
    import torch
    H, d, cap = 2, 64, 64
    lengths = [70, 64 + 20 + 5, 64 + n, 500, 2 ** 30]
    c, kv = _filled([cap] * 5, H, d, 16, e4m3, "bnhd", 3)
    c.lengths.copy_(torch.tensor(lengths, dtype=torch.int32))
    q = torch.randn((5, n, H, d), generator=torch.Generator().manual_seed(9)).to(torch.bfloat16)
    out, lse = c.attend(q.cuda(), left=left, right=right, sinks=sinks)
    torch.cuda.synchronize()
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    held = [[_held(x, e4m3) for x in rows] for rows in kv]
    for b in range(5):
        pos = lengths[b] - n + np.arange(n)
        ok = S.seen(pos, range(cap), cap, left, right, sinks)
        ok[pos < 0] = False
        for h in range(H):
            x = np.where((pos >= 0)[:, None], q[b, :, h].double().numpy(), 0.0)
            args = (x, held[0][b][:, h], held[1][b][:, h], ok, d ** -0.5)
            o, l, _ = S.forward(*args)
            bo, bl = S.forward_bounds(*args, 2.0 ** -8)
            assert (np.abs(out[b, :, h] - o) <= bo + 2.0 ** -8 * np.abs(o)).all(), (b, h)
            assert np.array_equal(np.isneginf(lse[b, h]), np.isneginf(l)), (b, h)
            some = np.isfinite(l)
            assert (np.abs(lse[b, h][some] - l[some]) <= bl[some]).all(), (b, h)


@pytest.mark.parametrize("e4m3", [False, True])
def test_assigned_tensors_are_the_ones_that_calls_use(e4m3):
    """lengths, tables and pools that are replaced, not written in place; the old tensors stay alive here, so that nothing reads freed memory."""
    import torch
    c, _ = _filled([40, 64], 2, 64, 16, e4m3, "bnhd", 3)
    q = torch.randn((2, 3, 2, 64), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    old = [c.lengths, c.table, c.k, c.v, c.k_exp, c.v_exp]

    def results():
        res = [*c.read(64), *c.attend(q)]
        torch.cuda.synchronize()
        return res

    def same(a, b):
        return all(torch.equal(x, y) for x, y in zip(a, b))
    first = results()
    c.lengths = c.lengths - 5
    got = results()
    old[0].sub_(5)
    c.lengths = old[0]
    assert same(got, results()) and not same(got, first)
    c.table = c.table.flip(0).contiguous()                     # sequences change places; the table of the second is full
    c.lengths = c.lengths.flip(0).contiguous()
    swapped = results()
    assert torch.equal(swapped[0][0], got[0][1]) and torch.equal(swapped[1][1], got[1][0])
    zeros = torch.zeros_like(c.v.view(torch.uint8)).view(c.v.dtype)
    c.v = zeros
    assert (results()[1] == 0).all() and torch.equal(results()[0], swapped[0])
    c.v = old[3]
    wide = torch.cat((c.table, torch.full_like(c.table, -1)), 1)
    c.table = wide
    assert c.width == 8 and same(swapped, results())


def test_assigned_tensors_are_checked():
    import torch
    c, _ = _filled([40, 64], 2, 64, 16, True, "bnhd", 3)
    bad = dict(lengths=[c.lengths.long(), c.lengths[:1], c.lengths.cpu(), None], table=[c.table.long(), c.table[:1], c.table[0], c.table.t(), None],
               k=[c.k[:2], c.k.view(torch.uint8), None], v=[c.v[:, :, :8], c.v.to(torch.bfloat16)], k_exp=[None, c.k_exp.int()], v_exp=[c.v_exp[:1]])
    for name, values in bad.items():
        for value in values:
            kept = getattr(c, name)
            with pytest.raises((ValueError, AttributeError, TypeError)):
                setattr(c, name, value)
            assert getattr(c, name) is kept
    assert torch.isfinite(c.read(40)[0]).all()


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("layout", ["bhnd", "bnhd"])
@pytest.mark.parametrize("n,left,right,sinks", [(100, 30, 0, 5), (70, 64, 20, 70), (150, -1, -1, 0), (90, 0, 0, 0)])
def test_chunks_of_width_64(e4m3, layout, n, left, right, sinks):
    _attend([200, 150, 301], [n, n - 9, 1], n, 4, 2, 64, 24, e4m3, left, right, sinks, layout)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 20, 90])
def test_sharp_scores_over_the_cache(e4m3, d, n):
    """Scores up to a few hundred: most weights vanish, the running maximum moves a lot, and parts of a row differ in it by more than fp32's exponents hold."""
    import torch
    lengths, H, HK = [700, 300], 4, 2
    c, kv = _filled(lengths, HK, d, 32, e4m3, "bnhd", 3)
    q = (8 * torch.randn((2, n, H, d), generator=torch.Generator().manual_seed(4))).to(torch.bfloat16)
    out, lse = c.attend(q.cuda(), left=600, sinks=2, scale=0.5)
    torch.cuda.synchronize()
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    for b, length in enumerate(lengths):
        ok = S.seen(length - n + np.arange(n), range(length), length, 600, 0, 2)
        k, v = [_held(rows[b], e4m3) for rows in kv]
        for h in range(H):
            g = h // (H // HK)
            args = (q[b, :, h].double().numpy(), k[:, g], v[:, g], ok, 0.5)
            o, l, _ = S.forward(*args)
            bo, bl = S.forward_bounds(*args, 2.0 ** -8)
            assert (np.abs(out[b, :, h] - o) <= bo + 2.0 ** -8 * np.abs(o)).all(), (b, h)
            assert (np.abs(lse[b, h] - l) <= bl).all(), (b, h)


@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("e4m3", [False, True])
def test_pages_that_no_table_names_do_not_matter(e4m3, d, n):
    """A window whose earlier pages have been given back, and a table with a tile's worth of holes: bit for bit the same whatever the first page of the pool,
    which belongs to no sequence, holds."""
    import torch
    from paper_2510_08318_amd import torch_glue as G
    H, page, width, length = 2, 16, 12, 180
    gen = torch.Generator().manual_seed(5)
    c = G.PagedCache.empty(2 * width + 1, page, H, d, 2, width, quantised=e4m3)
    c.table.copy_(1 + torch.randperm(2 * width, generator=gen).view(2, width).int())
    c.lengths.fill_(length)
    k, v, q = [torch.randn((2, m, H, d), generator=gen).to(torch.bfloat16).cuda() for m in (length, length, n)]
    c.write(k, v)
    c.table[0, : (length - n - 30) // page] = -1               # what no query's window of 30 reaches
    c.table[1, 4:8] = c.pages                                  # keys 64 .. 127
    res = []
    for byte in (0, 0xff):
        for t in (c.k, c.v, c.k_exp, c.v_exp):
            if t is not None:
                t[0].view(torch.uint8).fill_(byte)
        res.append([*c.attend(q, left=30), *c.attend(q)])
    torch.cuda.synchronize()
    for i in (0, 1):                                           # (of the sequence without its first pages only the window)
        assert torch.isfinite(res[0][i]).all()
    for a, b in zip(*res):
        assert torch.equal(a, b)
