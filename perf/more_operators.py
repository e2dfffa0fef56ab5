"""Rotary positions and linear attention with a decay as timed and compared cases.

A case is one pass through an operator: `rotary` (q and k turned by their positions along one to three axes; inverse: their gradients turned
back), `decay` (causal linear attention with a decay for each head, over whole sequences or chunks that continue a state, forward), `decay_train`
(the same and its backward) and `step` (one new token, or a few, of each sequence of a batch, whose states lie in a pool and are updated in place).

Token counts are those of the converted video models (30 x 52 = 1560 tokens to a latent frame at 832x480, 45 x 80 at 1280x720, 21 frames; 12 or 40
heads of width 128), of the small fp32 configuration, and of short tests; the serving batches are generic.  Keys and queries are normalised
before attention, so their entries are N(0, 1) times a scale per head from U(0.5, 1.5).  Decays go from a memory of a few tokens to one of some hundreds.
"""
import math

import torch

own = False        # true: run() makes the library's calls; false: the plain form

FRAMES, ROWS, COLUMNS = 21, 30, 52
FRAME = ROWS * COLUMNS


def _rotary(name, *, mode="bf16", B=1, H=1, HK=0, n=1, d=128, dims=(128,), grid=(), first=(), explicit=False, far=1, pairs="adjacent", inverse=False,
            layout="bhnd", ragged=False):
    """dims: channels of each axis.  Positions: `grid` from `first` on, or explicit ones below `far`.  Tuples are kept as text: "44 42 42"."""
    case = dict(op="rotary", mode=mode, B=B, H=H, HK=HK or H, n=n, d=d, dims=" ".join(map(str, dims)), grid=" ".join(map(str, grid or (1,) * len(dims))),
                first=" ".join(map(str, first or (0,) * len(dims))), explicit=explicit, far=far, pairs=pairs, inverse=inverse, layout=layout, ragged=ragged)
    return dict(name=name, **case) if name else case


def _decay(name, *, op="decay", mode="bf16", B=1, H=1, HK=0, n=1, d=128, state=False, layout="bhnd", ragged=False):
    """state: the sequences continue a state and hand theirs on (training: with its gradient); step always does."""
    case = dict(op=op, mode=mode, B=B, H=H, HK=HK or H, n=n, d=d, state=state or op == "step", layout=layout, ragged=ragged)
    return dict(name=name, **case) if name else case


def listed():
    return [
        # serving: the new token of each of 64 sequences, positions as far as its sequence has come
        _rotary("rotary_tokens", B=64, H=32, HK=8, n=1, explicit=True, far=100_000, pairs="halves", layout="bnhd"),
        # q and k of a layer at 832x480 by frame, row and column, heads interleaved as the projections leave them
        _rotary("rotary_480p", H=12, n=FRAMES * FRAME, dims=(44, 42, 42), grid=(FRAMES, ROWS, COLUMNS), layout="bnhd"),
        # gradients of fp32 tensors turned back, a padded batch with shared key heads, frames that continue a clip
        _rotary("rotary_back_f32", mode="f32", B=2, H=12, HK=4, n=4133, d=64, dims=(32, 16, 16), grid=(1, 24, 40), first=(7, 0, 0), pairs="halves", inverse=True,
                ragged=True),
        # a layer at 832x480 with a causal linear branch
        _decay("decay_480p", H=12, n=FRAMES * FRAME, layout="bnhd"),
        # the large model's layer at 1280x720
        _decay("decay_720p", H=40, n=FRAMES * 45 * 80),
        # streaming generation: three latent frames continue the state of all before, and hand theirs on
        _decay("decay_chunk_480p", H=12, n=3 * FRAME, state=True, layout="bnhd"),
        # serving: prompts of a batch, shared key heads
        _decay("decay_prompts", B=4, H=32, HK=8, n=2048, state=True, layout="bnhd", ragged=True),
        # a training step at 832x480
        _decay("decay_train_480p", op="decay_train", H=12, n=FRAMES * FRAME),
        # a padded batch, shared key heads, gradients through the states
        _decay("decay_train_ragged", op="decay_train", B=2, H=12, HK=4, n=4133, d=64, state=True, layout="bnhd", ragged=True),
        # the small fp32 configuration, a reference step
        _decay("decay_train_f32", op="decay_train", mode="f32", H=2, n=1024, d=64),
        # serving: one token of each of 64 sequences, states updated in place
        _decay("step_tokens", op="step", B=64, H=32, HK=8, n=1, layout="bnhd"),
        # one token of one sequence, where latency counts
        _decay("step_token_small", op="step", H=12, n=1, d=64, layout="bnhd"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("rotary", "rotary", "decay", "decay", "decay_train", "decay_train", "step"))
    d, layout, ragged = rng.choice((64, 128)), rng.choice(("bhnd", "bnhd")), rng.random() < 0.5
    HK = _log_int(rng, 1, 12)
    H = HK * rng.choice((1, 1, 2, 4))
    B = rng.choice((1, 1, 2, 3, 5))
    mode = rng.choices(("bf16", "f32", "f32math"), (0.7, 0.2, 0.1))[0]
    if op == "step":
        B = _log_int(rng, 1, 64)
        return _decay(None, op=op, mode=mode, B=B, H=H, HK=HK, n=rng.choice((1, 1, 1, _log_int(rng, 2, 16))), d=d, layout=layout, ragged=ragged)
    most = 400_000 if op == "decay" else 200_000 if op == "rotary" else 130_000         # rows of H heads, below the largest listed cases
    most = int(most * (128 / d) * (1.0 if mode == "bf16" else 0.3))
    n = max(1, min(_log_int(rng, 1, FRAMES * FRAME), most // (B * H)))
    if op != "rotary":
        return _decay(None, op=op, mode=mode, B=B, H=H, HK=HK, n=n, d=d, state=rng.random() < 0.5, layout=layout, ragged=ragged)
    halves = rng.random() < 0.5
    dims = rng.choice({64: ((64,), (32,), (32, 32), (32, 16, 16), (24, 20, 20), (16, 12, 10)),
                       128: ((128,), (64,), (64, 64), (32, 48, 48), (44, 42, 42), (16, 56, 56))}[d])
    rows, columns = _log_int(rng, 3, 45), _log_int(rng, 3, 80)
    grid = {1: (n,), 2: (-(-n // columns), columns), 3: (-(-n // (rows * columns)), rows, columns)}[len(dims)]
    first = tuple(rng.choice((0, 0, _log_int(rng, 1, 1000))) for _ in dims)
    explicit = rng.random() < 0.4
    return _rotary(None, mode="f32" if mode == "f32" else "bf16", B=B, H=H, HK=HK, n=n, d=d, dims=dims, grid=grid, first=first, explicit=explicit,
                   far=_log_int(rng, 100, 1_000_000) if explicit else 1, pairs="halves" if halves else "adjacent", inverse=rng.random() < 0.4, layout=layout,
                   ragged=ragged)


def _tuple(text):
    return tuple(int(x) for x in text.split())


def _lengths(case):
    """Tokens of each sequence: all of them, or a spread of lengths down to a third."""
    most, B = case["n"], case["B"]
    if not case["ragged"]:
        return [most] * B
    return [max(1, most - (most * ((5 * b + 2) % 8)) // 12) for b in range(B)]


def _dtype(case):
    return torch.float32 if case["mode"] == "f32" else torch.bfloat16


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    B, H, HK, n, d, dt = case["B"], case["H"], case["HK"], case["n"], case["d"], _dtype(case)

    def tokens(heads, scaled):
        """[B, heads, n, d] or [B, n, heads, d]"""
        shape = (B, n, heads, d) if case["layout"] == "bnhd" else (B, heads, n, d)
        x = torch.randn(shape, generator=gen, device="cuda")
        if scaled:
            scale = torch.rand((B, heads), generator=gen, device="cuda") + 0.5
            x *= scale[:, None, :, None] if case["layout"] == "bnhd" else scale[:, :, None, None]
        return x.to(dt)

    s = {"case": case, "q": tokens(H, True), "k": tokens(HK, True),
         "lengths": torch.tensor(_lengths(case), dtype=torch.int32, device="cuda") if case["ragged"] else None}
    if case["op"] == "rotary":
        s["positions"] = None
        if case["explicit"]:
            s["positions"] = torch.randint(0, case["far"], (B, n, len(_tuple(case["dims"]))), generator=gen, device="cuda", dtype=torch.int32)
        return s
    s["v"] = tokens(HK, False)
    slope = -torch.exp2(-8.0 * torch.arange(1, H + 1, device="cuda") / H)                # memories of about 1 to 256 tokens
    s["log_decay"] = slope * (torch.rand((H,), generator=gen, device="cuda") * 0.2 + 0.9)
    s["state"] = s["slots"] = None
    if case["state"]:
        rows = B + 3 if case["op"] == "step" else B
        s["state"] = torch.randn((rows, H, d, d), generator=gen, device="cuda") * (0.5 / -s["log_decay"])[:, None, None].sqrt()
        if case["op"] == "step":
            s["slots"] = torch.randperm(rows, generator=gen, device="cuda")[:B].int()
    if case["op"] == "decay_train":
        s["dout"] = tokens(H, False) * 0.1
        if case["state"]:
            s["dstate"] = torch.randn((B, H, d, d), generator=gen, device="cuda") * 0.1
    return s


# ---- the library's calls ----------------------------------------------------------------------------------------------


def _own_rotary(s):
    from paper_2510_08318_amd import torch_glue as G
    c = s["case"]
    q, k = G.rotary(s["q"], s["k"], dims=_tuple(c["dims"]), grid=_tuple(c["grid"]), first=_tuple(c["first"]), positions=s["positions"], pairs=c["pairs"],
                    inverse=c["inverse"], layout=c["layout"], lengths=s["lengths"])
    return {"q": q, "k": k}


def _own_decay(s):
    from paper_2510_08318_amd import torch_glue as G
    c = s["case"]
    kw = dict(state=s["state"], layout=c["layout"], lengths=s["lengths"], f32_math=c["mode"] == "f32math")
    if c["op"] == "step":
        out, _ = G.decay_attention(s["q"], s["k"], s["v"], s["log_decay"], slots=s["slots"], state_out=s["state"], **kw)
        return {"out": out, "state": s["state"]}
    out, state = G.decay_attention(s["q"], s["k"], s["v"], s["log_decay"], state_out=None if c["state"] else False, **kw)
    res = {"out": out}
    if c["state"]:
        res["state"] = state
    if c["op"] == "decay_train":
        res["dq"], res["dk"], res["dv"], dstate = G.decay_attention_backward(s["q"], s["k"], s["v"], s["log_decay"], s["dout"], dstate=s.get("dstate"), **kw)
        if c["state"]:
            res["dstate"] = dstate
    return res


# ---- the plain form ---------------------------------------------------------------------------------------------------


def _heads_first(x, layout):
    return x.transpose(1, 2) if layout == "bnhd" else x


def _live(s):
    c = s["case"]
    t = torch.arange(c["n"], device=s["q"].device)
    lengths = s["lengths"].long() if s["lengths"] is not None else torch.full((c["B"],), c["n"], device=t.device)
    return t[None] < lengths[:, None], lengths                                          # [B, n], [B]


def _positions(s):
    """[B, n, axes] in 64 bits."""
    c = s["case"]
    if s["positions"] is not None:
        return s["positions"].double()
    at, axes = torch.arange(c["n"], device=s["q"].device), []
    for size, first in reversed(list(zip(_tuple(c["grid"])[1:], _tuple(c["first"])[1:]))):
        axes.append(at % size + first)
        at = at // size
    axes.append(at + _tuple(c["first"])[0])
    return torch.stack(axes[::-1], -1)[None].double()


def _plain_rotary(s):
    c = s["case"]
    pos, live, d = _positions(s), _live(s)[0], c["d"]
    one, two, angles, off = [], [], [], 0
    for a, size in enumerate(_tuple(c["dims"])):
        m = torch.arange(size // 2, device=pos.device)
        one.append(off + 2 * m if c["pairs"] == "adjacent" else off + m)
        two.append(one[-1] + (1 if c["pairs"] == "adjacent" else size // 2))
        angles.append(pos[..., a, None] * torch.pow(10000.0, -2.0 * m.double() / size))
        off += size
    one, two, angles = torch.cat(one), torch.cat(two), torch.cat(angles, -1)
    cos, sin = angles.cos().float(), (-angles if c["inverse"] else angles).sin().float()
    over_heads = 2 if c["layout"] == "bnhd" else 1
    cos, sin, rows = cos.unsqueeze(over_heads), sin.unsqueeze(over_heads), live.unsqueeze(over_heads).unsqueeze(-1)
    res = {}
    for name in ("q", "k"):
        x = s[name].float()
        y = x.clone()
        x1, x2 = x[..., one], x[..., two]
        y[..., one], y[..., two] = x1 * cos - x2 * sin, x1 * sin + x2 * cos
        res[name] = (y * rows).to(s[name].dtype)
    return res


def _weights(g, r):
    """exp(g r) of heads and distances, worked out in 64 bits."""
    return torch.exp(g.double().view(-1, *[1] * r.dim()) * r).float()


def _pass(a, b, c, g, extra=None, chunk=128):
    """o_i = sum_{j <= i} exp(g (i - j)) (a_i . b_j) c_j of [B, H, n, d]."""
    B, H, n, d = a.shape
    parts = -(-n // chunk)
    a, b, c = [torch.nn.functional.pad(x, (0, 0, 0, parts * chunk - n)).view(B, H, parts, chunk, d) for x in (a, b, c)]
    t = torch.arange(chunk, device=a.device)
    gap = (t[:, None] - t[None]).double()
    inside = _weights(g, gap.clamp(min=0)) * (gap >= 0)
    out = ((a @ b.transpose(-1, -2)) * inside[None, :, None]) @ c
    if parts > 1:
        sums = (b * _weights(g, chunk - 1 - t.double())[None, :, None, :, None]).transpose(-1, -2) @ c
        whole = _weights(g, torch.tensor(float(chunk), dtype=torch.float64, device=a.device))[None, :, None, None]
        for i in range(1, parts):
            sums[:, :, i].add_(sums[:, :, i - 1] * whole)
        out[:, :, 1:] += (a[:, :, 1:] @ sums[:, :, :-1]) * _weights(g, t.double() + 1)[None, :, None, :, None]
    return out.reshape(B, H, parts * chunk, d)[:, :, :n]


def _plain_decay(s):
    c, layout = s["case"], s["case"]["layout"]
    H, HK, n, d, dt = c["H"], c["HK"], c["n"], c["d"], s["q"].dtype
    scale, g, (live, lengths) = 1.0 / math.sqrt(d), s["log_decay"], _live(s)
    t = torch.arange(n, device=g.device)

    def rows(name):
        return _heads_first(s[name], layout).float() * live[:, None, :, None]

    q, k, v = rows("q"), rows("k").repeat_interleave(H // HK, 1), rows("v").repeat_interleave(H // HK, 1)
    before = _weights(g, t.double() + 1)[None, :, :, None]                               # of the state before the first token
    to_end = torch.exp(g.double()[None, :, None] * (lengths[:, None, None] - 1 - t).clamp(min=0)).float()[..., None]
    whole = torch.exp(g.double()[None, :, None, None] * lengths[:, None, None, None]).float()
    state = s["state"]
    if state is not None and s["slots"] is not None:
        state = state[s["slots"].long()]
    out = _pass(q, k, v, g)
    if state is not None:
        out += (q @ state) * before
    res = {"out": out * scale}
    if state is not None:
        after = (k * to_end).transpose(-1, -2) @ v + state * whole
        if s["slots"] is not None:
            s["state"][s["slots"].long()] = after
            after = s["state"]
        res["state"] = after
    if c["op"] == "decay_train":
        do = rows("dout")
        dq = _pass(do, v, k, g)
        if state is not None:
            dq += (do @ state.transpose(-1, -2)) * before
        dk, dv = [_pass(*[x.flip(2) for x in abc], g).flip(2) * scale for abc in ((v, do, q), (k, q, do))]
        if state is not None:
            dk += (v @ s["dstate"].transpose(-1, -2)) * to_end * live[:, None, :, None]
            dv += (k @ s["dstate"]) * to_end * live[:, None, :, None]
            res["dstate"] = (q * _weights(g, t.double() + 1)[None, ..., None]).transpose(-1, -2) @ do * scale + s["dstate"] * whole
        res["dq"] = dq * scale
        for name, x in (("dk", dk), ("dv", dv)):
            res[name] = x.view(c["B"], HK, H // HK, n, d).sum(2)
    return {name: x if "state" in name else _heads_first(x * live[:, None, :, None], layout).to(dt).contiguous() for name, x in res.items()}


def run(state):
    rotary = state["case"]["op"] == "rotary"
    if own:
        return _own_rotary(state) if rotary else _own_decay(state)
    return _plain_rotary(state) if rotary else _plain_decay(state)


# ---- work and the definition in 64 bits -------------------------------------------------------------------------------


def work(case):
    """Bytes: every tensor row that the operator needs read or written once, states as well.  flops: what the recurrence does, a state's update and its
    read for each token of a head; the backward has three reads and two updates."""
    H, HK, d, rows = case["H"], case["HK"], case["d"], sum(_lengths(case))
    esz = 4 if case["mode"] == "f32" else 2
    if case["op"] == "rotary":
        turned = sum(_tuple(case["dims"]))
        return {"bytes": 2 * rows * (H + HK) * d * esz, "flops": 3 * rows * (H + HK) * turned}
    train = case["op"] == "decay_train"
    states = case["B"] * H * d * d * 4 * (4 if train else 2) if case["state"] else 0
    values = rows * d * (2 * H + 2 * HK) + (rows * d * (3 * H + 4 * HK) if train else 0)
    return {"bytes": values * esz + states, "flops": rows * H * d * d * (4 + (10 if train else 0))}


def _exact_rotary(case, s):
    pos, lengths, d = _positions(s), _lengths(case), case["d"]
    res = {}
    for name in ("q", "k"):
        x = _heads_first(s[name], case["layout"]).double()                              # [B, heads, n, d]
        y, off = x.clone(), 0
        for a, size in enumerate(_tuple(case["dims"])):
            part = x[..., off: off + size]
            z = torch.view_as_complex(part.unflatten(-1, (size // 2, 2)).contiguous()) if case["pairs"] == "adjacent" else torch.complex(
                part[..., : size // 2].contiguous(), part[..., size // 2:].contiguous())
            turn = pos[:, None, :, None, a] / 10000.0 ** (torch.arange(0, size, 2, dtype=torch.float64, device="cuda") / size)
            z = z * torch.polar(torch.ones_like(turn), -turn if case["inverse"] else turn)
            y[..., off: off + size] = torch.view_as_real(z).flatten(-2) if case["pairs"] == "adjacent" else torch.cat((z.real, z.imag), -1)
            off += size
        for b, length in enumerate(lengths):
            y[b, :, length:] = 0.0
        res[name] = _heads_first(y, case["layout"]).contiguous()
    return res


def _exact_decay(case, s):
    B, H, HK, n, d, layout, train = case["B"], case["H"], case["HK"], case["n"], case["d"], case["layout"], case["op"] == "decay_train"
    scale = d ** -0.5

    def head(name, b, h, length):
        return (s[name][b, :length, h] if layout == "bnhd" else s[name][b, h, :length]).double()

    def add(name, b, h, x):
        (res[name][b, : x.shape[0], h] if layout == "bnhd" else res[name][b, h, : x.shape[0]]).add_(x)

    def zeros(like):
        return torch.zeros(s[like].shape, dtype=torch.float64, device="cuda")

    res = {"out": zeros("q")}
    if case["state"]:
        res["state"] = s["state"].double() if case["op"] == "step" else zeros("state")
    if train:
        res.update(dq=zeros("q"), dk=zeros("k"), dv=zeros("v"))
        if case["state"]:
            res["dstate"] = zeros("dstate")
    for b, length in enumerate(_lengths(case)):
        at = int(s["slots"][b]) if s["slots"] is not None else b
        i = torch.arange(length, dtype=torch.float64, device="cuda")
        for h in range(H):
            g = float(s["log_decay"][h].double())
            q, k, v = head("q", b, h, length), head("k", b, h // (H // HK), length), head("v", b, h // (H // HK), length)
            do = head("dout", b, h, length) if train else None
            decay = torch.exp(g * i)                                                    # of distances
            out, dq = torch.empty_like(q), torch.empty_like(q)
            dk, dv = torch.zeros_like(k), torch.zeros_like(v)
            for i0 in range(0, length, 1024):                                           # rows i0 .. i1 - 1 against the tokens up to them
                i1 = min(length, i0 + 1024)
                gap = (i[i0:i1, None] - i[None, :i1]).long()
                w = torch.where(gap >= 0, decay[gap.clamp(min=0)], 0.0)
                p = (q[i0:i1] @ k[:i1].T) * w
                out[i0:i1] = p @ v[:i1]
                if train:
                    dp = (do[i0:i1] @ v[:i1].T) * w
                    dq[i0:i1] = dp @ k[:i1]
                    dk[:i1] += dp.T @ q[i0:i1]
                    dv[:i1] += p.T @ do[i0:i1]
            if case["state"]:
                start = s["state"][at, h].double()
                w = torch.exp(g * (i + 1.0))[:, None]
                out += w * (q @ start)
                res["state"][at, h] = math.exp(g * length) * start + (k * torch.exp(g * (length - 1.0 - i))[:, None]).T @ v
            add("out", b, h, scale * out)
            if not train:
                continue
            dk, dv, dq = scale * dk, scale * dv, scale * dq
            if case["state"]:
                end, back = s["dstate"][b, h].double(), torch.exp(g * (length - 1.0 - i))[:, None]
                dq += scale * w * (do @ start.T)
                dk += back * (v @ end.T)
                dv += back * (k @ end)
                res["dstate"][b, h] = scale * (w * q).T @ do + math.exp(g * length) * end
            add("dq", b, h, dq)
            add("dk", b, h // (H // HK), dk)
            add("dv", b, h // (H // HK), dv)
    return res


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_rotary(case, s) if case["op"] == "rotary" else _exact_decay(case, s)
