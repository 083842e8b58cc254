"""The 4-bit paged cache's operators as they are measured: the append that quantises, the reading back of cached
tokens (from pages of any type), and the attention over 4-bit pages.  `run` computes a case in its plain form
(elementary torch operations in 32 bits) or, where `own` is true, through the library's entry points; `exact` is
the definition in 64 bits."""
import math

import numpy as np
import torch

own = False

FIX = 44  # a turn of the rotary angle as 2**FIX, so that a long position times a frequency loses nothing
BASE = 10000.0
PAGES_SPARE = 3
GROUP = 16  # channels that share a scale


# ------------------------------------------------------------------------------------------------ cases
def listed():
    """Sizes: the two backbone shapes of synthetic/workloads.py (30x52 tokens a frame with 12 heads of 128, 44x80
    with 24 heads of 128), and the token-by-token serving of a sequence model with shared KV heads."""
    return [
        # one token each for a few sessions, with the step's queries rotated on the way: the smallest append; what was
        # written is read back
        dict(name="append tokens f4", op="append", batch=8, new=1, ragged=False, kv=3000, heads=16, kv_heads=4, dim=128, rot=128,
             layout="half", page=16, mix=3),
        # prompts of several sessions at once, odd lengths that end and begin inside a page, part of the head rotated
        dict(name="append prompts f4", op="append", batch=6, new=701, ragged=True, kv=5000, heads=12, kv_heads=3, dim=64, rot=32,
             layout="interleaved", page=32, mix=5),
        # four latent frames of the large backbone at once, and back as the blocks that the routing takes
        dict(name="append frames f4", op="append", batch=1, new=14080, ragged=False, kv=30001, heads=24, kv_heads=24, dim=128, rot=128,
             layout="half", page=64, mix=7),
        # the small backbone's whole history (16 frames) as bf16 blocks
        dict(name="read history f4", op="read", batch=1, new=24960, ragged=False, kv=24960, kv_heads=12, dim=128, page=64, cache="f4",
             out="bf16", mix=41),
        # the last tokens of several sessions from 8-bit pages, odd lengths
        dict(name="read sessions f8", op="read", batch=9, new=777, ragged=True, kv=6001, kv_heads=5, dim=64, page=32, cache="f8",
             out="f32", mix=43),
        # the smallest attention: one new token of one young session
        dict(name="decode one f4", op="attend", batch=1, new=1, ragged=False, kv=301, heads=8, kv_heads=2, dim=64, page=16,
             causal=True, window=0, sinks=0, lse=False, mix=11),
        # many sessions with a bounded memory: a window and the first tokens
        dict(name="decode window f4", op="attend", batch=48, new=1, ragged=True, kv=20000, heads=32, kv_heads=8, dim=128, page=16,
             causal=True, window=4096, sinks=128, lse=False, mix=13),
        # many sessions that see everything: what the cache's size bounds
        dict(name="decode full f4", op="attend", batch=24, new=1, ragged=True, kv=32768, heads=32, kv_heads=8, dim=128, page=64,
             causal=True, window=0, sinks=0, lse=True, mix=17),
        # a few drafted tokens of each session checked at once
        dict(name="decode drafts f4", op="attend", batch=4, new=7, ragged=False, kv=60011, heads=20, kv_heads=4, dim=128, page=32,
             causal=True, window=0, sinks=0, lse=False, mix=19),
        # prompts of odd lengths, three query heads to a KV head, a short window
        dict(name="prompts window f4", op="attend", batch=6, new=1201, ragged=True, kv=2500, heads=6, kv_heads=2, dim=64, page=16,
             causal=True, window=500, sinks=4, lse=True, mix=23),
        # a latent frame of the small backbone: all of the frame, a window of frames, the first frame as sinks
        dict(name="frame window f4", op="attend", batch=1, new=1560, ragged=False, kv=24960, heads=12, kv_heads=12, dim=128, page=64,
             causal=False, window=9360, sinks=1560, lse=False, mix=29),
        # a latent frame of the large backbone over eight frames
        dict(name="frame full f4", op="attend", batch=1, new=3520, ragged=False, kv=28160, heads=24, kv_heads=24, dim=128, page=64,
             causal=False, window=0, sinks=0, lse=False, mix=31),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "read", "attend", "attend"])
    dim = rng.choice([64, 128])
    kv_heads = rng.randint(1, 12)
    group = rng.choice([1, 1, 2, 3, 4, 5, 8])
    page = rng.choice([16, 32, 64, 128])
    mix = rng.randint(1, 1 << 20)
    if op == "append":
        batch = _log(rng, 1, 32)
        new = min(rng.choice([1, _log(rng, 1, 6000), _log(rng, 1, 6000)]), max(1, 12_000_000 // (batch * kv_heads * dim)))
        return dict(op=op, batch=batch, new=new, ragged=rng.random() < 0.5, kv=_log(rng, 1, 8000), heads=rng.choice([0, kv_heads * group]),
                    kv_heads=kv_heads, dim=dim, rot=rng.choice([dim, dim // 2]), layout=rng.choice(["half", "interleaved"]), page=page,
                    mix=mix)
    if op == "read":
        batch = _log(rng, 1, 32)
        new = min(_log(rng, 1, 20000), max(1, 30_000_000 // (batch * kv_heads * dim)))
        return dict(op=op, batch=batch, new=new, ragged=rng.random() < 0.5, kv=new + _log(rng, 1, 8000), kv_heads=kv_heads, dim=dim, page=page,
                    cache=rng.choice(["f4", "f4", "f8", "bf16"]), out=rng.choice(["bf16", "bf16", "f32"]), mix=mix)
    kind = rng.choice(["token", "few", "chunk"])
    if kind == "chunk":
        batch = _log(rng, 1, 6)
        new = _log(rng, 33, 2000)
        kv = new + _log(rng, 1, 20000)
        kv = max(new, min(kv, 2_200_000_000 // (batch * new * kv_heads * group * dim // 64)))
    else:
        batch = _log(rng, 1, 64)
        new = 1 if kind == "token" else rng.randint(2, 16)
        kv = new + min(_log(rng, 1, 60000), 400_000_000 // (batch * kv_heads * dim))
    window = rng.choice([0, 0, _log(rng, 1, 8000)])
    return dict(op=op, batch=batch, new=new, ragged=rng.random() < 0.5, kv=kv, heads=kv_heads * group, kv_heads=kv_heads, dim=dim, page=page,
                causal=rng.random() < 0.7, window=window, sinks=rng.choice([0, 4, 100, 1000]) if window else 0,
                lse=rng.random() < 0.3, mix=mix)


def _lengths(case):
    """(new tokens, tokens in the cache with them) of each sequence: they go by the case alone."""
    r = np.random.RandomState(case["mix"] % (1 << 31))
    B, new, kv = case["batch"], case["new"], case["kv"]
    q = np.full(B, new, dtype=np.int64)
    n = np.full(B, max(kv, new), dtype=np.int64)
    if case["ragged"]:
        q = np.where(np.arange(B) == 0, new, r.randint(1, new + 1, B))
        n = np.maximum(q, np.where(np.arange(B) == 0, kv, r.randint(kv // 4, kv + 1, B)))
    return q, n


def _visible(case):
    """Of each sequence: keys that any row sees, and (row, key) pairs that are seen."""
    keys, pairs = 0, 0
    for q, n in zip(*_lengths(case)):
        p = np.arange(n - q, n)
        hi = p + 1 if case["causal"] else np.full(q, n)
        lo = np.maximum(p - case["window"] + 1, 0) if case["window"] else np.zeros(q, dtype=np.int64)
        sink = np.minimum(case["sinks"], lo) if case["window"] else np.zeros(q, dtype=np.int64)
        keys += int(n - lo[0] + min(case["sinks"], lo[0]))
        pairs += int(np.sum(hi - lo + sink))
    return keys, pairs


def work(case):
    d, Hk = case["dim"], case["kv_heads"]
    held = {"f4": 0.5 + 1 / GROUP, "f8": 1, "bf16": 2}[case.get("cache", "f4")]  # bytes of a channel in the cache
    q, _ = _lengths(case)
    T = int(q.sum())
    if case["op"] == "append":  # the new rows come in, lie in the cache, and go out again
        return dict(bytes=int(T * Hk * d * 2 * (2 + 2 * held + 2) + T * case["heads"] * d * 4), flops=3 * T * (Hk + case["heads"]) * case["rot"])
    if case["op"] == "read":
        return dict(bytes=int(T * Hk * d * 2 * (held + (2 if case["out"] == "bf16" else 4))), flops=T * Hk * d * 2)
    keys, pairs = _visible(case)
    Hq = case["heads"]
    return dict(bytes=int(keys * Hk * d * 2 * held) + T * Hq * d * 4 + (4 * T * Hq if case["lse"] else 0), flops=4 * d * pairs * Hq)


# ------------------------------------------------------------------------------------------------ 4 bits
# Channels 2i and 2i + 1 are the low and the high half of a byte: a sign and a magnitude 0, 1/2, 1, 3/2, 2, 3, 4, 6.
# 16 channels share a scale of 8 bits (5 exponent, 3 mantissa bits; the upper half of an f16 number without its sign):
# their largest magnitude over 6, rounded to nearest even.
MAGNITUDES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
TOP_SCALE = 10240.0


def _quantised(x):
    """x [..., d] in 32 bits as (codes [..., d/2], scales [..., d/16]), both uint8."""
    g = x.unflatten(-1, (-1, GROUP))
    a = g.abs().amax(-1).double()
    a = a / torch.full_like(a, 6)  # (a number as divisor becomes a product with its rounded inverse)
    step = torch.exp2((torch.frexp(a)[1] - 1).clamp(min=-14).double() - 3)
    s = (torch.round(a / step) * step).clamp(max=TOP_SCALE).float()
    y = torch.where(s[..., None] > 0, g / torch.where(s > 0, s, 1.0)[..., None], 0.0)
    m = y.abs()
    step = torch.where(m < 2, 0.5, torch.where(m < 4, 1.0, 2.0))
    m = (torch.round(m / step) * step).clamp(max=6)
    code = torch.where(m < 2, 2 * m, torch.where(m < 4, m + 2, m / 2 + 4)) + torch.where(y < 0, 8.0, 0.0)
    code = code.flatten(-2).to(torch.uint8)
    return code[..., 0::2] | code[..., 1::2] << 4, (s.half().view(torch.int16) >> 7).to(torch.uint8)


def _values(codes, scales):
    """The values that codes [..., d/2] with scales [..., d/16] stand for, in 32 bits."""
    one = torch.tensor(MAGNITUDES + [-m for m in MAGNITUDES], device=codes.device)
    two = torch.stack([one.repeat(16), one.repeat_interleave(16)], 1)  # of a byte
    x = two[codes.int()].flatten(-2).unflatten(-1, (-1, GROUP))
    return (x * (scales.short() << 7).view(torch.float16).float()[..., None]).flatten(-2)


# ------------------------------------------------------------------------------------------------ inputs
def _turns(case):
    """Radians a position of every pair (64 bits)."""
    n = case["rot"] // 2
    return [BASE ** (-k / n) for k in range(n)]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dev = "cuda"
    d, Hk, ps = case["dim"], case["kv_heads"], case["page"]
    s = dict(case=case)

    def randn(*shape):
        return torch.randn(shape, generator=g, device=dev)

    q, n = _lengths(case)
    T, B = int(q.sum()), len(q)
    per = int(-(-n.max() // ps))
    pages = int((-(-n // ps)).sum()) + PAGES_SPARE
    order = torch.randperm(pages, generator=g, device=dev).to(torch.int32)
    table, at = torch.zeros((B, per), dtype=torch.int32, device=dev), 0
    for b in range(B):  # pages as an allocator hands them out: in no order
        c = int(-(-n[b] // ps))
        table[b, :c] = order[at:at + c]
        at += c
    s["table"], s["rows"], s["max_new"] = table, T, int(q.max())
    s["len"] = torch.tensor(n, dtype=torch.int32, device=dev)
    s["cu"] = torch.tensor(np.concatenate([[0], np.cumsum(q)]), dtype=torch.int32, device=dev) if case["ragged"] else None
    kind = case.get("cache", "f4")
    for name in ("k", "v"):
        if kind == "f4":
            s["cache_" + name] = torch.empty((pages, Hk, ps, d // 2), dtype=torch.uint8, device=dev)
            s["scale_" + name] = torch.empty((pages, Hk, ps, d // GROUP), dtype=torch.uint8, device=dev)
            some = max(1, 60_000_000 // (Hk * ps * d))
            for i in range(0, pages, some):
                x = randn(min(some, pages - i), Hk, ps, d)
                s["cache_" + name][i:i + some], s["scale_" + name][i:i + some] = _quantised(x)
        elif kind == "f8":
            s["cache_" + name] = (randn(pages, ps, Hk, d) * 90).clamp_(-448, 448).to(torch.float8_e4m3fn)
            s["scale_" + name] = torch.exp2(torch.randint(-8, -5, (pages, Hk), generator=g, device=dev).float())
        else:
            s["cache_" + name] = randn(pages, ps, Hk, d).to(torch.bfloat16)
    if case["op"] == "append":
        s["turns"] = torch.tensor([round(w / (2 * math.pi) * 2.0 ** FIX) for w in _turns(case)], device=dev)
        s["k"], s["v"] = randn(T, Hk, d).to(torch.bfloat16), randn(T, Hk, d).to(torch.bfloat16)
    if case.get("heads"):
        s["q"] = (1.5 * randn(T, case["heads"], d)).to(torch.bfloat16)
    return s


# ------------------------------------------------------------------------------------------------ the library's calls
def _handles(s):
    """What a user's program makes once: the rotary table and the cache's handle."""
    if "handles" not in s:
        from paper_2609_34144_gb300 import native as cast
        case, h = s["case"], dict(cast=cast)
        if "turns" in s:
            h["table"] = cast.rotary_table(case["rot"], layout=case["layout"], base=BASE)
        h["cache"] = cast.kv_cache(s["cache_k"], s["cache_v"], s.get("scale_k"), s.get("scale_v"))
        s["handles"] = h
    return s["handles"]


def _own(s):
    case, h = s["case"], _handles(s)
    cast, batch = h["cast"], dict(cu_new=s["cu"], max_new=s["max_new"])
    if case["op"] == "append":
        q = cast.cast_cache_append(s["k"], s["v"], h["cache"], s["table"], s["len"], rotary=h["table"], q=s.get("q"), **batch)
        k, v = cast.cast_cache_read(h["cache"], s["table"], s["len"], s["rows"], **batch)
        return dict(k=k, v=v, **({} if q is None else {"q": q}))
    if case["op"] == "read":
        k, v = cast.cast_cache_read(h["cache"], s["table"], s["len"], s["rows"], dtype=_out(case), **batch)
        return dict(k=k, v=v)
    return cast.cast_cache_attention(s["q"], h["cache"], s["table"], s["len"], causal=case["causal"], window=case["window"],
                                     sinks=case["sinks"], want_lse=case["lse"], **batch)


def _out(case):
    return torch.float32 if case.get("out") == "f32" else torch.bfloat16


# ------------------------------------------------------------------------------------------------ plain forms
def _turn(x, positions, s):
    """x [T, H, d] rotated by the positions [T], in 32 bits."""
    case = s["case"]
    r, n = case["rot"], case["rot"] // 2
    turns = (positions[:, None] * s["turns"]) & ((1 << FIX) - 1)
    angle = turns.float() * (2 * math.pi / 2.0 ** FIX)
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]
    y = x.float().clone()
    i = (slice(0, n), slice(n, r)) if case["layout"] == "half" else (slice(0, r, 2), slice(1, r, 2))
    a, b = x[..., i[0]].float(), x[..., i[1]].float()
    y[..., i[0]], y[..., i[1]] = a * cos - b * sin, b * cos + a * sin
    return y


def _rows(s):
    """Of each new token: its sequence and its position in it."""
    n, T = s["len"].long(), s["rows"]
    B = n.numel()
    cu = s["cu"].long() if s["cu"] is not None else torch.arange(B + 1, device=n.device) * (T // B)
    t = torch.arange(T, device=n.device)
    b = torch.searchsorted(cu, t, right=True) - 1
    return b, n[b] - (cu[b + 1] - t), cu


def _read(s, name, b, p):
    """The rows at positions p of sequences b, [T, Hk, d] in 32 bits."""
    ps = s["case"]["page"]
    page, row, c = s["table"].long()[b, p // ps], p % ps, s["cache_" + name]
    if "scale_" + name not in s:
        return c[page, row].float()
    if c.dtype is torch.uint8:
        return _values(c[page, :, row], s["scale_" + name][page, :, row])
    return c.view(torch.uint8)[page, row].view(torch.float8_e4m3fn).float() * s["scale_" + name][page][:, :, None]


def _store(s, name, x, b, p):
    """The new rows x [T, Hk, d] (32 bits) into the 4-bit cache."""
    ps = s["case"]["page"]
    page, row = s["table"].long()[b, p // ps], p % ps
    s["cache_" + name][page, :, row], s["scale_" + name][page, :, row] = _quantised(x)


def _gathered(s, name):
    """Every sequence's rows in order, [B, Hk, L, d] in 32 bits."""
    t = s["table"].long()
    return _values(s["cache_" + name][t], s["scale_" + name][t]).transpose(1, 2).flatten(2, 3)


def _attend(s):
    case, q = s["case"], s["q"]
    b, p, cu = _rows(s)
    B, Hk, d, G = len(cu) - 1, case["kv_heads"], case["dim"], case["heads"] // case["kv_heads"]
    k, v = _gathered(s, "k"), _gathered(s, "v")
    L, Q, n = k.shape[2], s["max_new"], s["len"].long()
    i = torch.arange(q.shape[0], device=q.device) - cu[b]
    pad = torch.zeros((B, Q, Hk, G, d), device=q.device)
    pad[b, i] = q.float().view(-1, Hk, G, d)
    at = torch.full((B, Q), -1, device=q.device)
    at[b, i] = p
    j = torch.arange(L, device=q.device)
    see = (j < n[:, None, None]) & (at >= 0)[:, :, None]
    if case["causal"]:
        see = see & (j <= at[:, :, None])
    if case["window"]:
        see = see & ((j > at[:, :, None] - case["window"]) | (j < case["sinks"]))
    x = pad.permute(0, 2, 3, 1, 4).reshape(B, Hk, G * Q, d) @ k.transpose(2, 3)
    x = (x.view(B, Hk, G, Q, L) / math.sqrt(d)).masked_fill_(~see[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    x = x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    v = torch.where((j < n[:, None])[:, None, :, None], v, 0.0)
    o = x.view(B, Hk, G * Q, L) @ v
    o = o.view(B, Hk, G, Q, d) / torch.where(total > 0, total, 1.0)
    o = o.permute(0, 3, 1, 2, 4)[b, i].reshape(-1, Hk * G * d).to(torch.bfloat16)
    if not case["lse"]:
        return o
    return o, (top + total.log())[..., 0].permute(0, 3, 1, 2)[b, i].reshape(-1, Hk * G)


def run(state):
    if own:
        return _own(state)
    case = state["case"]
    if case["op"] == "attend":
        return _attend(state)
    b, p, _ = _rows(state)
    out = {}
    if case["op"] == "append":
        _store(state, "k", _turn(state["k"], p, state), b, p)
        _store(state, "v", state["v"].float(), b, p)
        if "q" in state:
            out["q"] = _turn(state["q"], p, state).to(torch.bfloat16)
    return dict(k=_read(state, "k", b, p).to(_out(case)), v=_read(state, "v", b, p).to(_out(case)), **out)


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def _exact_turn(x, positions, case):
    x = x.double()
    n = case["rot"] // 2
    out = x.clone()
    for i, f in enumerate(_turns(case)):
        lo, hi = (i, i + n) if case["layout"] == "half" else (2 * i, 2 * i + 1)
        w = positions.double() * f
        z = torch.polar(torch.ones_like(w), w)[:, None] * torch.complex(x[..., lo], x[..., hi])
        out[..., lo], out[..., hi] = z.real, z.imag
    return out


def _exact_rounded(x):
    """What 4 bits keep of x [T, H, d]: of each channel the nearest of the 15 values times its group's scale."""
    for c in range(0, x.shape[2], GROUP):
        g = x[:, :, c:c + GROUP]
        a = g.abs().amax(2) / torch.full_like(g[:, :, 0], 6)
        unit = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** -14))) - 3)
        s = (torch.round(a / unit) * unit).clamp(max=TOP_SCALE)[:, :, None]
        best, err = torch.zeros_like(g), g.abs()
        # in the order of even codes first, so that of two values equally near the even code stays
        for m in (1.0, 2.0, 4.0, 0.5, 1.5, 3.0, 6.0):
            off = (g.abs() - m * s).abs()
            near = off < err
            best, err = torch.where(near, m * s * g.sign(), best), torch.where(near, off, err)
        x[:, :, c:c + GROUP] = best
    return x


def _exact_page(s, name, page):
    """The pages' values, [..., Hk, ps, d] in 64 bits."""
    c = s["cache_" + name][page]
    if "scale_" + name not in s:
        return c.double().transpose(-2, -3)
    scale = s["scale_" + name][page]
    if c.dtype is not torch.uint8:
        return c.double().transpose(-2, -3) * scale.double()[..., None, None]
    codes = torch.stack([c % 16, c // 16], -1).flatten(-2).long()
    low = codes % 8
    value = torch.where(low < 2, 0.5 * low, (1 + 0.5 * (low % 2)) * torch.exp2((low // 2 - 1).double()))
    e, m = (scale // 8).double(), (scale % 8).double()
    times = torch.where(e > 0, (8 + m) * torch.exp2(e - 18), m * 2.0 ** -17)
    return value * (1 - 2 * (codes // 8)) * times.repeat_interleave(GROUP, -1)


def exact(case, seed):
    s = prepare(case, seed)
    q, n = _lengths(case)
    ps, at = case["page"], 0
    T, Hk, d = int(q.sum()), case["kv_heads"], case["dim"]
    if case["op"] == "append":
        positions = torch.cat([torch.arange(m - c, m, device="cuda") for c, m in zip(q.tolist(), n.tolist())])
        out = dict(k=_exact_rounded(_exact_turn(s["k"], positions, case)), v=_exact_rounded(s["v"].double()))
        if "q" in s:
            out["q"] = _exact_turn(s["q"], positions, case)
        return out
    if case["op"] == "read":
        out = {x: torch.empty((T, Hk, d), dtype=torch.float64, device="cuda") for x in ("k", "v")}
        for b, (c, m) in enumerate(zip(q.tolist(), n.tolist())):
            first = (m - c) // ps
            page = s["table"][b, first:-(-m // ps)].long()
            for x in ("k", "v"):
                rows = _exact_page(s, x, page).transpose(1, 2).reshape(-1, Hk, d)
                out[x][at:at + c] = rows[m - c - first * ps:m - first * ps]
            at += c
        return out
    G = case["heads"] // Hk
    o = torch.zeros((T, Hk * G, d), dtype=torch.float64, device="cuda")
    lse = torch.full((T, Hk * G), -math.inf, dtype=torch.float64, device="cuda")
    for b, (c, m) in enumerate(zip(q.tolist(), n.tolist())):
        page = s["table"][b, :-(-m // ps)].long()
        key, row = torch.arange(m, device="cuda"), torch.arange(m - c, m, device="cuda")[:, None]
        hidden = (key > row) if case["causal"] else torch.zeros((c, m), dtype=torch.bool, device="cuda")
        if case["window"]:
            hidden = hidden | ((key <= row - case["window"]) & (key >= case["sinks"]))
        k, v = (_exact_page(s, x, page).transpose(0, 1).reshape(Hk, -1, d)[:, :m] for x in ("k", "v"))
        for h in range(Hk):
            for a in range(h * G, h * G + G):
                z = (s["q"][at:at + c, a].double() @ k[h].T * d ** -0.5).masked_fill_(hidden, -math.inf)
                lse[at:at + c, a] = torch.logsumexp(z, 1)
                o[at:at + c, a] = torch.nan_to_num(torch.softmax(z, 1)) @ v[h]
        at += c
    o = o.view(T, -1)
    return (o, lse) if case["lse"] else o
