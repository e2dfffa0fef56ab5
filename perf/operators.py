"""The softmax branch and its cache as timed and compared cases.

A case is one pass through an operator: `window` (softmax attention in which a token sees a window of tokens around it and
the first tokens, forward), `window_train` (the same and its backward), `write` (the keys and values of new tokens into a
paged cache), `roundtrip` (a chunk quantised into the cache and the cache read back), `read` (the cache read back) and
`attend` (a chunk of new tokens, or one, over the paged cache).

Token counts are those of the converted video models (30 x 52 = 1560 tokens to a latent frame at 832x480, 21 frames; 12 heads of
width 128; 30 heads of width 64), of the small fp32 configuration, and of short tests; the serving batches are generic.
Keys and queries are normalised before attention, so their entries are N(0, 1) times a scale per head from U(0.5, 1.5).
"""
import math

import numpy as np
import torch

own = False        # true: run() makes the library's calls; false: the plain form

FRAME = 30 * 52


def _window(name, *, train=False, mode="bf16", B=1, H=1, HK=0, n=1, d=128, left=-1, right=-1, sinks=0, layout="bhnd", ragged=False):
    case = dict(op="window_train" if train else "window", mode=mode, B=B, H=H, HK=HK or H, n=n, d=d, left=left, right=right, sinks=sinks,
                layout=layout, ragged=ragged)
    return dict(name=name, **case) if name else case


def _cache(name, *, op, e4m3=False, B=1, H=0, HK=1, n=1, d=128, tokens=0, page=64, left=-1, right=0, sinks=0, layout="bnhd", ragged=False):
    """tokens: of the longest sequence in the cache, the n new ones included."""
    case = dict(op=op, e4m3=e4m3, B=B, H=H or HK, HK=HK, n=n, d=d, tokens=max(tokens, n), page=page, left=left, right=right, sinks=sinks,
                layout=layout, ragged=ragged)
    return dict(name=name, **case) if name else case


def listed():
    return [
        # a short clip or a test input: a call whose time is launches and latency
        _window("window_small", H=4, n=1000, d=64, left=128, right=128, sinks=4),
        # the softmax branch of a layer at 832x480, two frames to either side and the first frame, heads interleaved as the projections leave them
        _window("window_480p", H=12, n=21 * FRAME, left=2 * FRAME, right=2 * FRAME, sinks=FRAME, layout="bnhd"),
        # a training step of that branch, one frame to either side
        _window("window_train_480p", train=True, H=12, n=21 * FRAME, left=FRAME, right=FRAME, sinks=FRAME),
        # a padded batch of causal sequences with shared key heads
        _window("window_train_ragged", train=True, B=2, H=12, HK=4, n=4133, d=64, left=1024, right=0, sinks=16, layout="bnhd", ragged=True),
        # the small fp32 configuration, a reference step
        _window("window_train_f32", train=True, mode="f32", H=2, n=1024, d=64, left=256, right=256, sinks=16),
        # serving: one new token of each of 64 sequences goes into the cache
        _cache("write_tokens", op="write", B=64, HK=8, n=1, tokens=128, ragged=True),
        # streaming generation: a chunk of three latent frames is quantised into the cache and read back
        _cache("roundtrip_chunk_e4m3", op="roundtrip", e4m3=True, HK=12, n=3 * FRAME, tokens=3 * FRAME, page=FRAME),
        # the whole quantised cache of a batch read back, as before a rewrite of its first frames
        _cache("read_480p_e4m3", op="read", e4m3=True, B=4, HK=12, tokens=21 * FRAME, ragged=True),
        # streaming generation: a chunk of three frames attends to itself and everything before, quantised cache
        _cache("attend_chunk_480p_e4m3", op="attend", e4m3=True, HK=12, n=3 * FRAME, tokens=21 * FRAME, page=FRAME, right=-1),
        # serving: chunks of prompts over a cache with a window, first tokens, shared key heads
        _cache("attend_prompt_bf16", op="attend", B=4, H=32, HK=8, n=512, tokens=8192, left=4096, sinks=16, ragged=True),
        # serving: one token of each of 32 long sequences, every key read once
        _cache("attend_tokens_bf16", op="attend", B=32, H=32, HK=8, n=1, tokens=16384, ragged=True),
        # serving: one token of one sequence, where latency counts
        _cache("attend_token_small_e4m3", op="attend", e4m3=True, H=8, HK=2, n=1, d=64, tokens=2000, page=16),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("window", "window_train", "write", "roundtrip", "read", "attend", "attend"))
    d, layout, ragged = rng.choice((64, 128)), rng.choice(("bhnd", "bnhd")), rng.random() < 0.5
    HK = _log_int(rng, 1, 12)
    H = HK * rng.choice((1, 1, 2, 4))
    B = rng.choice((1, 1, 2, 3))
    sinks = rng.choice((0, 1, 4, 64, _log_int(rng, 1, FRAME)))
    if op.startswith("window"):
        mode = rng.choices(("bf16", "f32", "f32math"), (0.7, 0.15, 0.15))[0]
        pairs = (6e8 if op == "window" else 2.5e8) * (1.0 if mode == "bf16" else 0.2)      # below the largest listed case
        n = _log_int(rng, 32, 21 * FRAME)
        reach = min(n, max(1, int(pairs / (B * H * n)) - sinks))
        left = min(n, _log_int(rng, 1, max(1, reach)))
        right = rng.choice((0, min(n, max(0, reach - left))))
        if B * H * n * n < pairs and rng.random() < 0.4:
            left = -1
            right = rng.choice((-1, 0))
        return _window(None, train=op == "window_train", mode=mode, B=B, H=H, HK=HK, n=n, d=d, left=left, right=right,
                       sinks=min(sinks, n), layout=layout, ragged=ragged)
    page = rng.choice((16, 64, 128, _log_int(rng, 7, FRAME)))
    e4m3 = op == "roundtrip" or rng.random() < 0.5
    B = _log_int(rng, 1, 32)
    most = 12_000_000 // (B * HK * d)      # token rows: the largest listed reads 4 x 12 x 32760 x 128
    if op == "write":
        n = rng.choice((1, _log_int(rng, 1, 4096)))
        n = max(1, min(n, most))
        return _cache(None, op=op, e4m3=False, B=B, HK=HK, n=n, d=d, tokens=n + _log_int(rng, 1, 300), page=page, layout=layout, ragged=ragged)
    tokens = min(_log_int(rng, 64, 21 * FRAME), max(64, most))
    if op in ("roundtrip", "read"):
        n = tokens if op == "roundtrip" else 1
        return _cache(None, op=op, e4m3=e4m3, B=B, HK=HK, n=n, d=d, tokens=tokens, page=page, layout=layout, ragged=ragged)
    n = rng.choice((1, 1, _log_int(rng, 1, 64), _log_int(rng, 1, 4096)))
    n = max(1, min(n, tokens, int(1.2e9 / (B * H * tokens))))
    left, right = rng.choice(((-1, 0), (-1, -1), (_log_int(rng, 1, tokens), 0), (_log_int(rng, 1, tokens), 0)))
    return _cache(None, op=op, e4m3=e4m3, B=B, H=H, HK=HK, n=n, d=d, tokens=tokens, page=page, left=left, right=right, sinks=sinks,
                  layout=layout, ragged=ragged)


def _lengths(case):
    """Tokens of each sequence: all of them, or a spread of lengths down to a third."""
    most, B = case["n"] if case["op"].startswith("window") else case["tokens"], case["B"]
    if not case["ragged"]:
        return [most] * B
    return [max(1, most - (most * ((5 * b) % 8)) // 12) for b in range(B)]


def _counts(case):
    """New tokens of each sequence: the chunk, or less where the sequence is shorter or the batch ragged."""
    return [max(1, min(case["n"], length) - ((3 * b) % 4 * case["n"] // 8 if case["ragged"] else 0)) for b, length in enumerate(_lengths(case))]


def _dtype(case):
    return torch.float32 if case.get("mode") == "f32" else torch.bfloat16


def _quantise(x):
    """x [..., d] -> e4m3 codes and the exponent byte of each row."""
    x = x.float()
    amax = torch.where(x.isfinite(), x.abs(), 0.0).amax(-1)
    m, e = torch.frexp(amax)                                   # amax = m 2^e, m in [1/2, 1); 448 = 7/8 2^9
    e = torch.where(amax > 0, e - 9 + (m > 0.875), -117).clamp(min=-117)
    return torch.ldexp(x, -e[..., None]).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _values(codes, exps):
    return torch.ldexp(codes.float(), exps.int()[..., None] - 127)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    B, H, HK, n, d, dt = case["B"], case["H"], case["HK"], case["n"], case["d"], _dtype(case)

    def tokens(heads, n, scaled):
        """[B, heads, n, d] or [B, n, heads, d]"""
        shape = (B, n, heads, d) if case["layout"] == "bnhd" else (B, heads, n, d)
        x = torch.randn(shape, generator=gen, device="cuda")
        if scaled:
            scale = torch.rand((B, heads), generator=gen, device="cuda") + 0.5
            x *= scale[:, None, :, None] if case["layout"] == "bnhd" else scale[:, :, None, None]
        return x.to(dt)

    s = {"case": case, "lengths": torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")}
    if case["op"].startswith("window"):
        s["lengths"] = s["lengths"] if case["ragged"] else None
        s["q"], s["k"], s["v"] = tokens(H, n, True), tokens(HK, n, True), tokens(HK, n, False)
        if case["op"] == "window_train":
            s["dout"] = tokens(H, n, False) * 0.1
        return s
    page, width = case["page"], -(-case["tokens"] // case["page"])
    s["counts"] = torch.tensor(_counts(case), dtype=torch.int32, device="cuda")
    pages = B * width + 3
    used = torch.arange(width, device="cuda")[None] * page < s["lengths"][:, None]
    s["table"] = torch.where(used, torch.randperm(pages, generator=gen, device="cuda")[: B * width].view(B, width), -1).int()
    for name in ("k", "v"):
        pool = torch.randn((pages, HK, page, d), generator=gen, device="cuda")
        if name == "k":
            pool *= torch.rand((HK, 1, 1), generator=gen, device="cuda") + 0.5
        if case["e4m3"]:
            s[name + "_pool"], s[name + "_exp"] = _quantise(pool)
        else:
            s[name + "_pool"] = pool.to(dt)
    if case["op"] in ("write", "roundtrip"):
        s["k"], s["v"] = tokens(HK, n, True), tokens(HK, n, False)
    if case["op"] == "attend":
        s["q"] = tokens(H, n, True)
    return s


# ---- the library's calls ----------------------------------------------------------------------------------------------


def _own_window(s):
    from paper_2510_08318_amd import torch_glue as G
    c = s["case"]
    sees = dict(left=c["left"], right=c["right"], sinks=c["sinks"], layout=c["layout"], lengths=s["lengths"], f32_math=c["mode"] == "f32math")
    out, lse = G.window_attention(s["q"], s["k"], s["v"], **sees)
    res = {"out": out, "lse": lse}
    if c["op"] == "window_train":
        res["dq"], res["dk"], res["dv"] = G.window_attention_backward(s["q"], s["k"], s["v"], out, lse, s["dout"], **sees)
    return res


def _own_cache(s):
    from paper_2510_08318_amd import torch_glue as G
    c, layout = s["case"], s["case"]["layout"]
    if "cache" not in s:
        s["cache"] = G.PagedCache(s["k_pool"], s["v_pool"], s["table"], s["lengths"], s.get("k_exp"), s.get("v_exp"))
    cache = s["cache"]
    if c["op"] == "attend":
        out, lse = cache.attend(s["q"], counts=s["counts"], left=c["left"], right=c["right"], sinks=c["sinks"], layout=layout)
        return {"out": out, "lse": lse}
    if c["op"] != "read":
        cache.write(s["k"], s["v"], counts=s["counts"], layout=layout)
        if c["op"] == "write":
            return {"k_pool": cache.k, "v_pool": cache.v}
    k, v = cache.read(c["tokens"], layout=layout)
    res = {"k": k, "v": v}
    if c["op"] == "roundtrip":
        res["k_exp"], res["v_exp"] = cache.k_exp, cache.v_exp
    return res


# ---- the plain form ---------------------------------------------------------------------------------------------------


def _seen(p, j, length, left, right, sinks):
    """Whether the query at position p sees key j of `length`."""
    ok = j < length
    if right >= 0:
        ok = ok & (j <= p + right)
    if left >= 0:
        ok = ok & ((j >= p - left) | (j < sinks))
    return ok


def _softmax(s, ok):
    """Scores and visibility -> probabilities and the logarithm of their sum; a row that sees nothing has zeros and -inf."""
    s = s.masked_fill_(~ok, -math.inf)
    top = s.amax(-1, keepdim=True)
    p = (s - top.masked_fill(top == -math.inf, 0.0)).exp_()
    total = p.sum(-1, keepdim=True)
    return p.div_(total.clamp(min=1e-30)), (top + total.log()).squeeze(-1)


def _heads_first(x, layout):
    return x.transpose(1, 2) if layout == "bnhd" else x


def _plain_window(s):
    c, layout = s["case"], s["case"]["layout"]
    B, H, HK, n, d = c["B"], c["H"], c["HK"], c["n"], c["d"]
    G, left, right, scale, dev = H // HK, c["left"], c["right"], 1.0 / math.sqrt(d), s["q"].device
    lengths = s["lengths"].long() if s["lengths"] is not None else torch.full((B,), n, device=dev)
    live = torch.arange(n, device=dev)[None] < lengths[:, None]                         # [B, n]
    q, k, v = [_heads_first(s[t], layout).float() * live[:, None, :, None] for t in ("q", "k", "v")]
    # Blocks of queries against the band of keys that they reach and the first tokens; one block against all keys where that is no fewer.
    block, first = 520, min(c["sinks"], n)
    banded = left >= 0 and right >= 0 and first + block + left + right < n
    if not banded:
        block, first = n, 0
    blocks = -(-n // block)
    start = torch.arange(blocks, device=dev) * block
    pos = start[:, None] + torch.arange(block, device=dev)                              # [blocks, block]
    if banded:
        band = start[:, None] - left + torch.arange(block + left + right, device=dev)
        keys = torch.cat((torch.arange(first, device=dev).expand(blocks, first), band), 1)
        once = torch.cat((torch.ones(blocks, first, dtype=torch.bool, device=dev), band >= first), 1)
    else:
        keys, once = torch.arange(n, device=dev)[None], torch.ones(1, n, dtype=torch.bool, device=dev)
    there = once & (keys >= 0) & (keys < n)
    length = lengths[:, None, None, None]
    ok = _seen(pos[:, :, None], keys[:, None, :], length, left, right, c["sinks"]) & there[:, None, :] & (pos[:, :, None] < length)
    ok = ok[:, None, None]                                                              # [B, 1, 1, blocks, block, keys]
    at = keys.clamp(0, n - 1).reshape(-1)

    def queries(x):
        return torch.nn.functional.pad(x, (0, 0, 0, blocks * block - n)).view(B, HK, G, blocks, block, -1)

    def gathered(x):
        return x[:, :, at].view(B, HK, 1, blocks, -1, d)

    def rows(x):
        return x.reshape(B, H, blocks * block, -1)[:, :, :n]

    qb, kb, vb = queries(q), gathered(k), gathered(v)
    p, lse = _softmax((qb @ kb.transpose(-1, -2)).mul_(scale), ok)
    ob = p @ vb
    res = {"out": rows(ob), "lse": rows(lse[..., None])[..., 0].contiguous()}
    if c["op"] == "window_train":
        do = queries(_heads_first(s["dout"], layout).float() * live[:, None, :, None])
        ds = (do @ vb.transpose(-1, -2)).sub_((do * ob).sum(-1, keepdim=True)).mul_(p)
        res["dq"] = rows((ds @ kb).mul_(scale))

        def scattered(x):                                                               # [B, HK, G, blocks, keys, d] -> [B, HK, n, d]
            return torch.zeros((B, HK, n, d), device=dev).index_add_(2, at, x.sum(2).view(B, HK, -1, d))

        res["dv"] = scattered(p.transpose(-1, -2) @ do)
        res["dk"] = scattered((ds.transpose(-1, -2) @ qb).mul_(scale))
    return {name: x if name == "lse" else _heads_first(x, layout).to(s["q"].dtype).contiguous() for name, x in res.items()}


def _slots(s, pos):
    """Rows of the pool, as (page, row), of positions [B, n]."""
    page, width = s["case"]["page"], s["table"].shape[1]
    return s["table"].long().gather(1, (pos // page).clamp(0, width - 1)).clamp(min=0), pos % page


def _plain_write(s):
    c = s["case"]
    n, lengths, counts = c["n"], s["lengths"].long(), s["counts"].long()
    t = torch.arange(n, device=lengths.device)
    pos = (lengths - counts)[:, None] + t
    page, row = _slots(s, pos.clamp(min=0))
    b, t = ((t[None] < counts[:, None]) & (pos >= 0)).nonzero(as_tuple=True)
    page, row = page[b, t], row[b, t]
    for name in ("k", "v"):
        x = s[name] if c["layout"] == "bnhd" else s[name].transpose(1, 2)               # [B, n, HK, d]
        x = x[b, t]
        if c["e4m3"]:
            codes, exps = _quantise(x)
            s[name + "_pool"].view(torch.uint8)[page, :, row] = codes.view(torch.uint8)
            s[name + "_exp"][page, :, row] = exps
        else:
            s[name + "_pool"][page, :, row] = x


def _gathered(s, name):
    """The cache's values in 32 bits, [B, HK, tokens, d], zeros behind a sequence."""
    c, dev = s["case"], s["lengths"].device
    pos = torch.arange(c["tokens"], device=dev).expand(c["B"], -1)
    page, row = _slots(s, pos)
    if c["e4m3"]:
        codes = s[name + "_pool"].view(torch.uint8)[page, :, row].view(torch.float8_e4m3fn)
        x = _values(codes, s[name + "_exp"][page, :, row])                               # [B, tokens, HK, d]
    else:
        x = s[name + "_pool"][page, :, row].float()
    return x.masked_fill_((pos >= s["lengths"][:, None])[:, :, None, None], 0.0).transpose(1, 2)


def _plain_cache(s):
    c, layout = s["case"], s["case"]["layout"]
    if c["op"] in ("write", "roundtrip"):
        _plain_write(s)
        if c["op"] == "write":
            return {"k_pool": s["k_pool"], "v_pool": s["v_pool"]}
    if c["op"] != "attend":
        res = {name: _heads_first(_gathered(s, name), layout).to(torch.bfloat16).contiguous() for name in ("k", "v")}
        if c["op"] == "roundtrip":
            res["k_exp"], res["v_exp"] = s["k_exp"], s["v_exp"]
        return res
    B, H, HK, n, d, dev = c["B"], c["H"], c["HK"], c["n"], c["d"], s["lengths"].device
    lengths, counts = s["lengths"].long()[:, None, None], s["counts"].long()[:, None, None]
    t = torch.arange(n, device=dev)[None, :, None]
    pos = lengths - counts + t
    ok = _seen(pos, torch.arange(c["tokens"], device=dev)[None, None], lengths, c["left"], c["right"], c["sinks"]) & (t < counts) & (pos >= 0)
    k, v = _gathered(s, "k"), _gathered(s, "v")
    q = _heads_first(s["q"], layout).float().reshape(B, HK, H // HK * n, d)
    scores = (q @ k.transpose(-1, -2)).mul_(1.0 / math.sqrt(d)).view(B, HK, H // HK, n, -1)
    p, lse = _softmax(scores, ok[:, None, None])
    out = (p.view(B, HK, -1, c["tokens"]) @ v).view(B, H, n, d)
    return {"out": _heads_first(out, layout).to(torch.bfloat16).contiguous(), "lse": lse.reshape(B, H, n)}


def run(state):
    window = state["case"]["op"].startswith("window")
    if own:
        return _own_window(state) if window else _own_cache(state)
    return _plain_window(state) if window else _plain_cache(state)


# ---- work and the definition in 64 bits -------------------------------------------------------------------------------


def _sight(case):
    """Of each sequence: pairs of a query and a key that it sees, and keys that any query sees."""
    left, right, sinks, res = case["left"], case["right"], case["sinks"], []
    counts = _lengths(case) if case["op"].startswith("window") else _counts(case)
    for length, count in zip(_lengths(case), counts):
        p = np.arange(length - count, length)
        hi = np.minimum(length, p + right + 1) if right >= 0 else np.full(count, length)
        lo = np.maximum(0, p - left) if left >= 0 else np.zeros(count, dtype=np.int64)
        res.append((int((hi - lo + np.minimum(sinks, lo)).sum()), int(hi.max() - lo.min() + min(sinks, lo.min()))))
    return res


def work(case):
    """Bytes: every tensor row that the operator needs read or written once.  flops: two contractions of a forward pair, five of a backward one."""
    H, HK, n, d = case["H"], case["HK"], case["n"], case["d"]
    esz = 4 if case.get("mode") == "f32" else 2
    if case["op"].startswith("window"):
        rows, train, pairs = sum(_lengths(case)), case["op"] == "window_train", sum(p for p, _ in _sight(case))
        values = rows * d * (2 * H + 2 * HK) + (rows * d * (3 * H + 4 * HK) if train else 0)
        return {"bytes": values * esz + (2 if train else 1) * rows * H * 4, "flops": pairs * H * d * (14 if train else 4)}
    row = HK * (d + 1 if case["e4m3"] else 2 * d)              # of the cache, k or v
    new, held = sum(_counts(case)), sum(_lengths(case))
    if case["op"] == "attend":
        sight = _sight(case)
        return {"bytes": 2 * sum(k for _, k in sight) * row + new * H * (2 * d * 2 + 4), "flops": sum(p for p, _ in sight) * H * d * 4}
    write, read = 2 * new * (HK * d * 2 + row), 2 * held * (HK * d * 2 + row)
    return {"bytes": {"write": write, "read": read, "roundtrip": write + read}[case["op"]], "flops": 0}


def _attention64(q, k, v, ok, scale):
    """One head: q [m, d], k, v [keys, d], ok [m, keys]."""
    s = torch.where(ok, scale * (q @ k.t()), -math.inf)
    lse = torch.logsumexp(s, -1)
    return torch.exp(s - torch.where(lse.isinf(), 0.0, lse)[:, None]) @ v, lse


def _exact_window(case, s):
    B, H, HK, n, d, layout = case["B"], case["H"], case["HK"], case["n"], case["d"], case["layout"]
    left, right, sinks, train = case["left"], case["right"], case["sinks"], case["op"] == "window_train"

    def head(name, b, h, length):
        return (s[name][b, :length, h] if layout == "bnhd" else s[name][b, h, :length]).double()

    def put(name, b, h, i0, i1, x):
        (res[name][b, i0:i1, h] if layout == "bnhd" else res[name][b, h, i0:i1]).add_(x)

    res = {"out": torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda"),
           "lse": torch.full((B, H, n), -math.inf, dtype=torch.float64, device="cuda")}
    if train:
        res.update({g: torch.zeros(s[t].shape, dtype=torch.float64, device="cuda") for g, t in (("dq", "q"), ("dk", "k"), ("dv", "v"))})
    for b, length in enumerate(_lengths(case)):
        for h in range(H):
            q, k, v = head("q", b, h, length), head("k", b, h // (H // HK), length), head("v", b, h // (H // HK), length)
            do = head("dout", b, h, length) if train else None
            for i0 in range(0, length, 2048):
                i1 = min(length, i0 + 2048)
                lo = max(0, i0 - left) if left >= 0 else 0
                hi = min(length, i1 + right) if right >= 0 else length
                first = min(sinks, lo)
                j = torch.cat((torch.arange(first, device="cuda"), torch.arange(lo, hi, device="cuda")))
                i = torch.arange(i0, i1, device="cuda")[:, None]
                ok = torch.ones((i1 - i0, j.numel()), dtype=torch.bool, device="cuda")
                if right >= 0:
                    ok &= j <= i + right
                if left >= 0:
                    ok &= (i - j <= left) | (j < sinks)
                parts = [x.detach().requires_grad_(train) for x in (q[i0:i1], k[j], v[j])]
                out, lse = _attention64(*parts, ok, d ** -0.5)
                put("out", b, h, i0, i1, out.detach())
                res["lse"][b, h, i0:i1] = lse.detach()
                if train:
                    gq, gk, gv = torch.autograd.grad(out, parts, do[i0:i1])
                    put("dq", b, h, i0, i1, gq)
                    for name, g in (("dk", gk), ("dv", gv)):
                        put(name, b, h // (H // HK), 0, first, g[:first])
                        put(name, b, h // (H // HK), lo, hi, g[first:])
    return res


def _e4m3_grid():
    """The non-negative numbers of e4m3 in order, so that a number's place is its code."""
    small = [m * 2.0 ** -9 for m in range(8)]
    return torch.tensor(small + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)][:-1], dtype=torch.float64, device="cuda")


def _rounded64(x):
    """Rows of x rounded as the quantised cache holds them, in 64 bits."""
    grid, x = _e4m3_grid(), x.double()
    amax = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(torch.where(amax > 0, amax, 1e-300) / 448.0)).clamp(min=-117)
    e = torch.where(amax > 448.0 * torch.exp2(e), e + 1, torch.where(amax <= 448.0 * torch.exp2(e - 1), (e - 1).clamp(min=-117), e))
    y = x.abs() * torch.exp2(-e)
    at = torch.searchsorted(grid, y).clamp(1, grid.numel() - 1)
    below, above = grid[at - 1], grid[at]
    up = (y - below > above - y) | ((y - below == above - y) & (at % 2 == 0))
    return torch.copysign(torch.where(up, above, below) * torch.exp2(e), x)


def _sequence64(case, s, name, b, length):
    """The cache's values of one sequence, [length, HK, d], page by page."""
    got = []
    for i in range(-(-length // case["page"])):
        at = int(s["table"][b, i])
        x = s[name + "_pool"][at].double()
        got.append(x * torch.exp2(s[name + "_exp"][at].double() - 127.0)[..., None] if case["e4m3"] else x)
    return torch.cat(got, 1)[:, :length].transpose(0, 1)


def _exact_cache(case, s):
    B, H, HK, n, d, layout, op = case["B"], case["H"], case["HK"], case["n"], case["d"], case["layout"], case["op"]
    counts, lengths = _counts(case), _lengths(case)

    def new(name, b, count):
        return s[name][b, :count] if layout == "bnhd" else s[name][b, :, :count].transpose(0, 1)      # [count, heads, d]

    if op == "write":
        res = {}
        for name in ("k", "v"):
            res[name + "_pool"] = pool = s[name + "_pool"].double()
            for b in range(B):
                x, at = new(name, b, counts[b]).double(), lengths[b] - counts[b]
                while at < lengths[b]:                                          # up to the end of the page
                    end = min(lengths[b], (at // case["page"] + 1) * case["page"])
                    t = at - lengths[b] + counts[b]
                    pool[int(s["table"][b, at // case["page"]]), :, at % case["page"]: at % case["page"] + end - at] = x[t: t + end - at].transpose(0, 1)
                    at = end
        return res
    if op in ("read", "roundtrip"):
        res = {}
        for name in ("k", "v"):
            x = torch.zeros((B, case["tokens"], HK, d), dtype=torch.float64, device="cuda")
            for b in range(B):
                x[b, : lengths[b]] = _sequence64(case, s, name, b, lengths[b])
                if op == "roundtrip":
                    x[b, lengths[b] - counts[b]: lengths[b]] = _rounded64(new(name, b, counts[b]))
            res[name] = x if layout == "bnhd" else x.transpose(1, 2).contiguous()
        return {**res, **({"k_exp": None, "v_exp": None} if op == "roundtrip" else {})}
    out = torch.zeros((B, n, H, d), dtype=torch.float64, device="cuda")
    lse = torch.full((B, H, n), -math.inf, dtype=torch.float64, device="cuda")
    for b, (length, count) in enumerate(zip(lengths, counts)):
        k, v, q = _sequence64(case, s, "k", b, length), _sequence64(case, s, "v", b, length), new("q", b, count).double()
        i, j = torch.arange(length - count, length, device="cuda")[:, None], torch.arange(length, device="cuda")
        ok = torch.ones((count, length), dtype=torch.bool, device="cuda")
        if case["right"] >= 0:
            ok &= j - i <= case["right"]
        if case["left"] >= 0:
            ok &= (i - j <= case["left"]) | (j < case["sinks"])
        for h in range(H):
            g = h // (H // HK)
            out[b, :count, h], lse[b, h, :count] = _attention64(q[:, h], k[:, g].contiguous(), v[:, g].contiguous(), ok, d ** -0.5)
    return {"out": out if layout == "bnhd" else out.transpose(1, 2).contiguous(), "lse": lse}


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_window(case, s) if case["op"].startswith("window") else _exact_cache(case, s)
