"""The paged KV cache's operators as they are measured: rotary positions, the append to the cache, and the
attention over it.  `run` computes a case in its plain form (elementary torch operations in 32 bits) or, where
`own` is true, through the library's entry points; `exact` is the definition in 64 bits."""
import math

import numpy as np
import torch

own = False

FIX = 44  # a turn of the rotary angle as 2**FIX, so that a long position times a frequency loses nothing
PAGES_SPARE = 3


# ------------------------------------------------------------------------------------------------ cases
def listed():
    """Sizes: the two backbone shapes of synthetic/workloads.py (30x52 tokens a frame with 12 heads of 128, 44x80
    with 24 heads of 128), and the token-by-token serving of a sequence model with shared KV heads."""
    return [
        # one latent frame's queries before attention: (frame, row, column) positions
        dict(name="rotary frame bf16", op="rotary", tokens=1560, heads=12, dim=128, rot=128, layout="half", axes=3, dtype="bf16",
             inverse=False, scaling="none", factor=1.0, reach=4096),
        # the gradient through the rotation of a long ragged prompt, part of the head, stretched context
        dict(name="rotary gradient f32", op="rotary", tokens=9973, heads=7, dim=64, rot=48, layout="interleaved", axes=1, dtype="f32",
             inverse=True, scaling="parts", factor=8.0, reach=200000),
        # one token each for a few sessions: the smallest append, with the step's queries rotated on the way
        dict(name="append tokens bf16", op="append", batch=8, new=1, ragged=False, kv=3000, heads=16, kv_heads=4, dim=128, rot=128,
             layout="half", page=16, cache="bf16", mix=3),
        # prompts of several sessions at once, odd lengths, 8-bit pages that end and begin inside a page
        dict(name="append prompts f8", op="append", batch=6, new=701, ragged=True, kv=5000, heads=12, kv_heads=3, dim=64, rot=32,
             layout="interleaved", page=32, cache="f8", mix=5),
        # four latent frames of the large backbone at once into 8-bit pages
        dict(name="append frames f8", op="append", batch=1, new=14080, ragged=False, kv=30001, heads=24, kv_heads=24, dim=128, rot=128,
             layout="half", page=64, cache="f8", mix=7),
        # the smallest attention: one new token of one young session
        dict(name="decode one bf16", op="attend", batch=1, new=1, ragged=False, kv=301, heads=8, kv_heads=2, dim=64, page=16,
             cache="bf16", causal=True, window=0, sinks=0, lse=False, mix=11),
        # many sessions with a bounded memory: a window and the first tokens
        dict(name="decode window bf16", op="attend", batch=48, new=1, ragged=True, kv=20000, heads=32, kv_heads=8, dim=128, page=16,
             cache="bf16", causal=True, window=4096, sinks=128, lse=False, mix=13),
        # many sessions that see everything, in 8 bits: what the cache's size bounds
        dict(name="decode full f8", op="attend", batch=24, new=1, ragged=True, kv=32768, heads=32, kv_heads=8, dim=128, page=64,
             cache="f8", causal=True, window=0, sinks=0, lse=True, mix=17),
        # a few drafted tokens of each session checked at once
        dict(name="decode drafts f8", op="attend", batch=4, new=7, ragged=False, kv=60011, heads=20, kv_heads=4, dim=128, page=32,
             cache="f8", causal=True, window=0, sinks=0, lse=False, mix=19),
        # prompts of odd lengths, three query heads to a KV head, a short window
        dict(name="prompts window bf16", op="attend", batch=6, new=1201, ragged=True, kv=2500, heads=6, kv_heads=2, dim=64, page=16,
             cache="bf16", causal=True, window=500, sinks=4, lse=True, mix=23),
        # a latent frame of the small backbone: all of the frame, a window of frames, the first frame as sinks
        dict(name="frame window bf16", op="attend", batch=1, new=1560, ragged=False, kv=24960, heads=12, kv_heads=12, dim=128, page=64,
             cache="bf16", causal=False, window=9360, sinks=1560, lse=False, mix=29),
        # a latent frame of the large backbone over eight frames held in 8 bits
        dict(name="frame full f8", op="attend", batch=1, new=3520, ragged=False, kv=28160, heads=24, kv_heads=24, dim=128, page=64,
             cache="f8", causal=False, window=0, sinks=0, lse=False, mix=31),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotary", "append", "attend", "attend"])
    dim = rng.choice([64, 128])
    if op == "rotary":
        heads = rng.randint(1, 24)
        rot = rng.choice([dim, dim, dim // 2, 48])
        tokens = min(_log(rng, 1, 15000), 40_000_000 // (heads * dim))
        axes = rng.choice([1, 1, 3])
        return dict(op=op, tokens=tokens, heads=heads, dim=dim, rot=rot, layout=rng.choice(["half", "interleaved"]), axes=axes,
                    dtype=rng.choice(["bf16", "f32"]), inverse=rng.random() < 0.4,
                    scaling=rng.choice(["none", "linear", "parts", "stretch"]), factor=float(rng.choice([2, 4, 8])),
                    reach=_log(rng, 4096, 250000))
    kv_heads = rng.randint(1, 12)
    group = rng.choice([1, 1, 2, 3, 4, 5, 8])
    page, cache = rng.choice([16, 32, 64, 128]), rng.choice(["bf16", "f8"])
    mix = rng.randint(1, 1 << 20)
    if op == "append":
        batch = _log(rng, 1, 32)
        new = min(rng.choice([1, _log(rng, 1, 6000), _log(rng, 1, 6000)]), max(1, 12_000_000 // (batch * kv_heads * dim)))
        return dict(op=op, batch=batch, new=new, ragged=rng.random() < 0.5, kv=_log(rng, 1, 8000), heads=rng.choice([0, kv_heads * group]),
                    kv_heads=kv_heads, dim=dim, rot=rng.choice([dim, dim // 2]), layout=rng.choice(["half", "interleaved"]), page=page,
                    cache=cache, mix=mix)
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
                cache=cache, causal=rng.random() < 0.7, window=window, sinks=rng.choice([0, 4, 100, 1000]) if window else 0,
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
    d = case["dim"]
    if case["op"] == "rotary":
        elt = 2 if case["dtype"] == "bf16" else 4
        n = case["tokens"] * case["heads"]
        return dict(bytes=2 * n * d * elt + 4 * case["tokens"] * case["axes"], flops=3 * n * case["rot"])
    q, n = _lengths(case)
    T, Hk, Hq = int(q.sum()), case["kv_heads"], case["heads"]
    elt = 1 if case["cache"] == "f8" else 2
    if case["op"] == "append":
        return dict(bytes=T * Hk * d * 2 * (2 + elt) + T * Hq * d * 4, flops=3 * T * (Hk + Hq) * case["rot"])
    keys, pairs = _visible(case)
    scales = 8 * keys * Hk / case["page"] if case["cache"] == "f8" else 0
    return dict(bytes=keys * Hk * d * 2 * elt + scales + T * Hq * d * 4 + (4 * T * Hq if case["lse"] else 0), flops=4 * d * pairs * Hq)


# ------------------------------------------------------------------------------------------------ inputs
BASE, ORIGINAL = 10000.0, 4096


def _sections(case):
    """Pairs of each position axis: a quarter for the frame and the rest in halves, or all of them for one axis."""
    n = case["rot"] // 2
    if case.get("axes", 1) == 1:
        return [n]
    t = n - 2 * (3 * n // 8)
    return [t, 3 * n // 8, 3 * n // 8]


def _frequencies(case):
    """Radians a position of every pair (64 bits), the axis of each, and the amplitude."""
    s, kind, amp = case.get("factor", 1.0), case.get("scaling", "none"), 1.0
    f, axis = [], []
    for a, n in enumerate(_sections(case)):
        for k in range(n):
            base = BASE * s ** (n / (n - 1)) if kind == "stretch" else BASE
            w = base ** (-k / n)
            if kind == "linear":
                w /= s
            if kind == "parts":
                g = min(1.0, max(0.0, (ORIGINAL * w / (2 * math.pi) - 1) / (32 - 1)))
                w *= g + (1 - g) / s
            f.append(w)
            axis.append(a)
    if kind == "parts":
        amp = 0.1 * math.log(s) + 1
    return f, axis, amp


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dev = "cuda"
    d = case["dim"]
    s = dict(case=case)

    def randn(*shape):
        return torch.randn(shape, generator=g, device=dev)

    def rotation():
        f, axis, amp = _frequencies(case)
        s["turns"] = torch.tensor([round(w / (2 * math.pi) * 2.0 ** FIX) for w in f], device=dev)
        s["axis"], s["amp"] = torch.tensor(axis, device=dev), amp

    if case["op"] == "rotary":
        rotation()
        s["x"] = randn(case["tokens"], case["heads"], d).to(torch.bfloat16 if case["dtype"] == "bf16" else torch.float32)
        s["positions"] = torch.randint(0, case["reach"], (case["tokens"], case["axes"]), generator=g, device=dev, dtype=torch.int32)
        return s
    q, n = _lengths(case)
    T, B, Hk, Hq, ps = int(q.sum()), len(q), case["kv_heads"], case["heads"], case["page"]
    per = int(-(-n.max() // ps))
    pages = int((-(-n // ps)).sum()) + PAGES_SPARE
    order = torch.randperm(pages, generator=g, device=dev).to(torch.int32)
    table, at = torch.zeros((B, per), dtype=torch.int32, device=dev), 0
    for b in range(B):  # pages as an allocator hands them out: in no order
        c = int(-(-n[b] // ps))
        table[b, :c] = order[at:at + c]
        at += c
    s["table"], s["max_new"] = table, int(q.max())
    s["len"] = torch.tensor(n, dtype=torch.int32, device=dev)
    s["cu"] = torch.tensor(np.concatenate([[0], np.cumsum(q)]), dtype=torch.int32, device=dev) if case["ragged"] else None
    shape = (pages, ps, Hk, d)
    for name in ("k", "v"):
        if case["cache"] == "f8":
            s["cache_" + name] = (randn(*shape) * 90).clamp_(-448, 448).to(torch.float8_e4m3fn)
            s["scale_" + name] = torch.exp2(torch.randint(-8, -5, (pages, Hk), generator=g, device=dev).float())
        else:
            s["cache_" + name] = randn(*shape).to(torch.bfloat16)
    if case["op"] == "append":
        rotation()
        s["k"], s["v"] = randn(T, Hk, d).to(torch.bfloat16), randn(T, Hk, d).to(torch.bfloat16)
    if Hq:
        s["q"] = (1.5 * randn(T, Hq, d)).to(torch.bfloat16)
    return s


# ------------------------------------------------------------------------------------------------ the library's calls
def _handles(s):
    """What a user's program makes once: the rotary table and the cache's handle."""
    if "handles" not in s:
        from paper_2609_34144_gb300 import native as cast
        case, h = s["case"], dict(cast=cast)
        if "turns" in s:
            scaling = {"none": None}.get(case.get("scaling", "none"), (case.get("scaling"), case.get("factor"), ORIGINAL))
            h["table"] = cast.rotary_table(case["rot"], layout=case["layout"], base=BASE, sections=_sections(case), scaling=scaling)
        if "cache_k" in s:
            h["cache"] = cast.kv_cache(s["cache_k"], s["cache_v"], s.get("scale_k"), s.get("scale_v"))
        s["handles"] = h
    return s["handles"]


def _own(s):
    case, h = s["case"], _handles(s)
    cast = h["cast"]
    if case["op"] == "rotary":
        return cast.cast_rotary(s["x"], s["positions"], h["table"], inverse=case["inverse"])
    if case["op"] == "append":
        q = cast.cast_cache_append(s["k"], s["v"], h["cache"], s["table"], s["len"], cu_new=s["cu"], max_new=s["max_new"], rotary=h["table"],
                                   q=s.get("q"))
        return _appended(s, q)
    return cast.cast_cache_attention(s["q"], h["cache"], s["table"], s["len"], cu_new=s["cu"], max_new=s["max_new"], causal=case["causal"],
                                     window=case["window"], sinks=case["sinks"], want_lse=case["lse"])


def _appended(s, q):
    return dict({k: s[k] for k in ("cache_k", "cache_v", "scale_k", "scale_v") if k in s}, **({} if q is None else {"q": q}))


# ------------------------------------------------------------------------------------------------ plain forms
def _turn(x, positions, s, inverse=False):
    """x [T, H, d] rotated by the positions [T, axes], in 32 bits."""
    case = s["case"]
    r, n = case["rot"], case["rot"] // 2
    turns = (positions[:, s["axis"]].long() * s["turns"]) & ((1 << FIX) - 1)
    angle = turns.float() * (2 * math.pi / 2.0 ** FIX)
    cos, sin = (angle.cos() * s["amp"])[:, None], (angle.sin() * (-s["amp"] if inverse else s["amp"]))[:, None]
    y = x.float().clone()
    i = (slice(0, n), slice(n, r)) if case["layout"] == "half" else (slice(0, r, 2), slice(1, r, 2))
    a, b = x[..., i[0]].float(), x[..., i[1]].float()
    y[..., i[0]], y[..., i[1]] = a * cos - b * sin, b * cos + a * sin
    return y


def _rows(s):
    """Of each new token: its sequence and its position in it."""
    n, T = s["len"].long(), (s["k"] if "k" in s else s["q"]).shape[0]
    B = n.numel()
    cu = s["cu"].long() if s["cu"] is not None else torch.arange(B + 1, device=n.device) * (T // B)
    t = torch.arange(T, device=n.device)
    b = torch.searchsorted(cu, t, right=True) - 1
    return b, n[b] - (cu[b + 1] - t), cu


def _store(s, name, x, b, p, cu):
    """The new rows x [T, Hk, d] (32 bits) into the cache."""
    c, ps = s["cache_" + name], s["case"]["page"]
    page, row = s["table"].long()[b, p // ps], p % ps
    if "scale_" + name not in s:
        c[page, row] = x.to(c.dtype)
        return
    scale, Hk = s["scale_" + name], x.shape[1]
    amax = torch.full_like(scale, -1).index_reduce_(0, page, x.abs().amax(2), "amax")
    m, e = torch.frexp(amax)
    e = torch.where(amax > 0, e - 9 + (m > 0.875), -120).clamp(-120, 120)
    first = p[cu[:-1]]  # a sequence's first new token: a page that it only continues keeps what is in it
    head = s["table"].long()[torch.arange(len(first), device=c.device), first // ps]
    head, kept = head[first % ps > 0], (first % ps)[first % ps > 0]
    new = torch.where(amax >= 0, torch.ldexp(torch.ones_like(scale), e), scale)
    new[head] = torch.maximum(new[head], scale[head])
    old = (c[head].float() * (scale[head] / new[head])[:, None, :, None]).to(c.dtype)
    keep = torch.arange(ps, device=c.device)[None, :] < kept[:, None]
    c[head] = torch.where(keep[:, :, None, None], old.float(), c[head].float()).to(c.dtype)
    scale.copy_(new)
    c.view(torch.uint8)[page, row] = (x / new[page][:, :, None]).to(c.dtype).view(torch.uint8)


def _gathered(s, name):
    """Every sequence's rows in order, [B, L, Hk, d] in 32 bits."""
    t = s["table"].long()
    c = s["cache_" + name].view(torch.uint8)[t].view(torch.float8_e4m3fn) if "scale_" + name in s else s["cache_" + name][t]
    c = c.float()
    if "scale_" + name in s:
        c = c * s["scale_" + name][t][:, :, None, :, None]
    return c.flatten(1, 2)


def _attend(s):
    case, q = s["case"], s["q"]
    b, p, cu = _rows(s)
    B, Hk, d, G = len(cu) - 1, case["kv_heads"], case["dim"], case["heads"] // case["kv_heads"]
    k, v = _gathered(s, "k"), _gathered(s, "v")
    L, Q, n = k.shape[1], s["max_new"], s["len"].long()
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
    x = pad.permute(0, 2, 3, 1, 4).reshape(B, Hk, G * Q, d) @ k.permute(0, 2, 3, 1)
    x = (x.view(B, Hk, G, Q, L) / math.sqrt(d)).masked_fill_(~see[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    x = x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    v = torch.where((j < n[:, None])[:, :, None, None], v, 0.0)
    o = x.view(B, Hk, G * Q, L) @ v.permute(0, 2, 1, 3)
    o = o.view(B, Hk, G, Q, d) / torch.where(total > 0, total, 1.0)
    o = o.permute(0, 3, 1, 2, 4)[b, i].reshape(-1, Hk * G * d).to(torch.bfloat16)
    if not case["lse"]:
        return o
    return o, (top + total.log())[..., 0].permute(0, 3, 1, 2)[b, i].reshape(-1, Hk * G)


def run(state):
    if own:
        return _own(state)
    case = state["case"]
    if case["op"] == "rotary":
        return _turn(state["x"], state["positions"], state, case["inverse"]).to(state["x"].dtype)
    if case["op"] == "append":
        b, p, cu = _rows(state)
        _store(state, "k", _turn(state["k"], p[:, None], state), b, p, cu)
        _store(state, "v", state["v"].float(), b, p, cu)
        return _appended(state, _turn(state["q"], p[:, None], state).to(torch.bfloat16) if "q" in state else None)
    return _attend(state)


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def _exact_turn(x, positions, case, inverse=False):
    f, axis, amp = _frequencies(case)
    x = x.double()
    n = case["rot"] // 2
    out = x.clone()
    for i in range(n):
        lo, hi = (i, i + n) if case["layout"] == "half" else (2 * i, 2 * i + 1)
        w = positions[:, axis[i]].double() * f[i]
        z = torch.polar(torch.full_like(w, amp), -w if inverse else w)[:, None] * torch.complex(x[..., lo], x[..., hi])
        out[..., lo], out[..., hi] = z.real, z.imag
    return out


def _exact_e4m3(x):
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rotary":
        return _exact_turn(s["x"], s["positions"], case, case["inverse"])
    q, n = _lengths(case)
    ps, at = case["page"], 0
    f8 = case["cache"] == "f8"
    if case["op"] == "append":
        out = {x: s[x].double() for x in ("cache_k", "cache_v", "scale_k", "scale_v") if x in s}
        positions = torch.cat([torch.arange(m - c, m, device="cuda") for c, m in zip(q.tolist(), n.tolist())])
        if "q" in s:
            out["q"] = _exact_turn(s["q"], positions[:, None], case)
        rows = dict(k=_exact_turn(s["k"], positions[:, None], case), v=s["v"].double())
        for b, (c, m) in enumerate(zip(q.tolist(), n.tolist())):
            for g in range((m - c) // ps, (m - 1) // ps + 1):
                page, lo, hi = int(s["table"][b, g]), max(g * ps, m - c), min(g * ps + ps, m)
                for x in ("k", "v"):
                    new, cache = rows[x][at + lo - (m - c):at + hi - (m - c)], out["cache_" + x]
                    if f8:
                        scale, old = out["scale_" + x], out["scale_" + x][page].clone()
                        top = new.abs().amax((0, 2))
                        e = torch.where(top > 0, torch.ceil(torch.log2((top / 448).clamp(min=2.0 ** -300))), -120.0).clamp(-120, 120)
                        scale[page] = torch.exp2(e) if lo == g * ps else torch.maximum(old, torch.exp2(e))
                        cache[page, :lo % ps] = _exact_e4m3(cache[page, :lo % ps] * (old / scale[page])[:, None])
                        new = _exact_e4m3(new / scale[page][:, None])
                    cache[page, lo - g * ps:hi - g * ps] = new
            at += c
        return out
    Hk, G, d = case["kv_heads"], case["heads"] // case["kv_heads"], case["dim"]
    T = int(q.sum())
    o = torch.zeros((T, Hk * G, d), dtype=torch.float64, device="cuda")
    lse = torch.full((T, Hk * G), -math.inf, dtype=torch.float64, device="cuda")
    for b, (c, m) in enumerate(zip(q.tolist(), n.tolist())):
        page = s["table"][b, :-(-m // ps)].long()
        key, row = torch.arange(m, device="cuda"), torch.arange(m - c, m, device="cuda")[:, None]
        hidden = (key > row) if case["causal"] else torch.zeros((c, m), dtype=torch.bool, device="cuda")
        if case["window"]:
            hidden = hidden | ((key <= row - case["window"]) & (key >= case["sinks"]))
        for h in range(Hk):
            kv = []
            for x in ("k", "v"):
                r = s["cache_" + x][:, :, h].double()[page]
                kv.append((r * s["scale_" + x][page, h].double()[:, None, None] if f8 else r).reshape(-1, d)[:m])
            for a in range(h * G, h * G + G):
                z = (s["q"][at:at + c, a].double() @ kv[0].T * d ** -0.5).masked_fill_(hidden, -math.inf)
                lse[at:at + c, a] = torch.logsumexp(z, 1)
                o[at:at + c, a] = torch.nan_to_num(torch.softmax(z, 1)) @ kv[1]
        at += c
    o = o.view(T, -1)
    return (o, lse) if case["lse"] else o
