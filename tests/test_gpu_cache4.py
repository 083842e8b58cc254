"""4-bit pages on the GPU against 64 bits: the append, the reading back (of pages of every type), the attention."""
import numpy as np
import pytest
import torch

from tests import cache4_ref as R4
from tests import cache_ref as R

pytestmark = pytest.mark.gpu


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def i32(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Pages4:
    """A 4-bit cache of B sequences, pages in no order, NaN scales wherever nothing was stored."""

    def __init__(self, lib, lens, H, d, page, seed=0, spare=2, apart=False):
        g = gen(seed)
        self.lib, self.lens, self.H, self.d, self.page = lib, list(lens), H, d, page
        per = [-(-n // page) for n in lens]
        n = sum(per) + spare
        pool = torch.randint(0, 256, (n, 2, H, page, d // 2), generator=g, device="cuda", dtype=torch.uint8)
        # K and V of a page side by side in one pool, or tensors of their own
        self.k, self.v = (pool[:, 0], pool[:, 1]) if apart else (pool[:, 0].contiguous(), pool[:, 1].contiguous())
        self.ks, self.vs = (torch.full((n, H, page, d // 16), 0xff, dtype=torch.uint8, device="cuda") for _ in range(2))
        order = torch.randperm(n, generator=torch.Generator().manual_seed(seed))
        self.table = torch.full((len(lens), max(max(per), 1)), -7, dtype=torch.int32)
        at = 0
        for b, c in enumerate(per):
            self.table[b, :c] = order[at:at + c].int()
            at += c
        self.table = self.table.cuda()
        self.kv_len = i32(*lens)
        self.cache = lib.kv_cache(self.k, self.v, self.ks, self.vs)

    def fill(self, seed=1, scale=1.0):
        """Everything stored: codes of normal numbers, in place."""
        g = gen(seed)
        out = []
        for b, n in enumerate(self.lens):
            k, v = (randn(g, n, self.H, self.d) * scale for _ in range(2))
            kq, ks = R4.quantise(f64(k))
            vq, vs = R4.quantise(f64(v))
            for page_t, scale_t, q, s in ((self.k, self.ks, kq, ks), (self.v, self.vs, vq, vs)):
                codes = encode(q, s)
                for i in range(0, n, self.page):
                    p, m = int(self.table[b, i // self.page]), min(self.page, n - i)
                    page_t[p, :, :m] = torch.from_numpy(codes[i:i + m]).cuda().transpose(0, 1)
                    scale_t[p, :, :m] = torch.from_numpy(s[i:i + m]).cuda().transpose(0, 1)
            out.append((kq, vq))
        return out

    def held(self, name, b):
        """Values [len, H, d] and scale bytes of sequence b as they lie."""
        t, s = (self.k, self.ks) if name == "k" else (self.v, self.vs)
        n, p = self.lens[b], self.table[b, :-(-self.lens[b] // self.page)].long()
        codes = t[p].transpose(1, 2).reshape(-1, self.H, self.d // 2)[:n].cpu().numpy()
        scales = s[p].transpose(1, 2).reshape(-1, self.H, self.d // 16)[:n].cpu().numpy()
        return R4.decode(codes, scales), scales


def encode(values, scales):
    s = np.repeat(R4.scale_value(scales), 16, -1)
    with np.errstate(all="ignore"):
        m = np.where((s > 0) & np.isfinite(s), np.abs(values) / np.where(s > 0, s, 1), 0)
    c = np.searchsorted(R4.VALUES, m).astype(np.uint8) | np.where(values < 0, 8, 0).astype(np.uint8)
    return (c[..., 0::2] | c[..., 1::2] << 4).astype(np.uint8)


# ------------------------------------------------------------------------------------ append
APPEND = [
    # lens, new, H, H_q, d, page, rot, layout, sections
    ([301], [1], 2, 8, 128, 16, 128, "half", None),
    ([5, 17, 64, 33], [1, 1, 1, 1], 3, 3, 64, 16, 64, "half", None),
    ([100, 7, 40], [64, 7, 1], 5, 10, 128, 32, 64, "interleaved", None),
    ([200, 131], [131, 90], 1, 4, 64, 64, 48, "half", None),          # a scale's channels in two units
    ([300], [290], 13, 13, 128, 128, 96, "half", [16, 16, 16]),
    ([40, 50], [40, 50], 2, 0, 64, 16, 0, "half", None),              # keys as they are
    ([129], [129], 4, 0, 128, 64, 16, "interleaved", None),
]


@pytest.mark.parametrize("lens,new,H,H_q,d,page,rot,layout,sections", APPEND)
@pytest.mark.parametrize("apart", [False, True])
def test_append(lib, lens, new, H, H_q, d, page, rot, layout, sections, apart):
    c = Pages4(lib, lens, H, d, page, seed=len(lens) + d, apart=apart)
    before = c.fill(seed=5)
    g = gen(7)
    T = sum(new)
    k, v = randn(g, T, H, d).to(torch.bfloat16), (3 * randn(g, T, H, d)).to(torch.bfloat16)
    q = randn(g, T, H_q, d).to(torch.bfloat16) if H_q else None
    table = lib.rotary_table(rot, layout, sections=sections) if rot else None
    axes = len(sections or [0])
    pos = torch.randint(0, 5000, (T, axes), generator=g, device="cuda", dtype=torch.int32) if axes > 1 else None
    cu = i32(*np.concatenate([[0], np.cumsum(new)]))
    untouched = torch.ones(c.k.shape[0], dtype=torch.bool, device="cuda")
    for b in range(len(lens)):
        untouched[c.table[b, :-(-lens[b] // page)].long()] = False
    spare = [t[untouched].clone() for t in (c.k, c.v, c.ks, c.vs)]
    out = lib.cast_cache_append(k, v, c.cache, c.table, c.kv_len, cu_new=cu, rotary=table, positions=pos, q=q)
    lib.cast_check_device()
    for was, t in zip(spare, (c.k, c.v, c.ks, c.vs)):
        assert torch.equal(was, t[untouched])
    at = 0
    for b, (n, m) in enumerate(zip(lens, new)):
        rows = slice(at, at + m)
        p = pos[rows].cpu().numpy() if pos is not None else np.arange(n - m, n)[:, None]
        x, err = f64(k[rows]), np.zeros((m, H, d))
        if rot:
            x, err = R.rotate(x, p, rot, layout, sections=sections)
        held, scales = c.held("k", b)
        assert np.array_equal(held[:n - m], before[b][0][:n - m])
        R4.check_quantised(held[n - m:], scales[n - m:], x, err)
        held, scales = c.held("v", b)
        assert np.array_equal(held[:n - m], before[b][1][:n - m])
        want, code = R4.quantise(f64(v[rows]))       # bf16 values: no rounding before, so to the bit
        assert np.array_equal(held[n - m:], want) and np.array_equal(scales[n - m:], code)
        if H_q:
            x, err = R.rotate(f64(q[rows]), p, rot, layout, sections=sections)
            assert (np.abs(f64(out[rows]) - x) <= err + R.UBF * (np.abs(x) + err)).all()
        at += m


def test_append_every_scale_and_every_tie(lib):
    """Values at and around the halfway points of codes, at every scale that a group's largest channel gives; ties of
    the scale itself; the ends of the range; zeros."""
    rows = []
    for e in range(-22, 18):
        for m in range(128, 256):
            top = m * 2.0 ** (e - 7)
            s = float(R4.scale_value(R4.scale_code(np.array([top / 6])))[0])
            t = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 1.0, 6.0]) * s
            rows.append(np.concatenate([[top], t * (1 - 2 * (np.arange(9) % 2)), [0, -0.0, -top, top / 2, top / 3, 2.0 ** -19]])[:16])
    x = torch.tensor(np.array(rows), dtype=torch.float32, device="cuda").to(torch.bfloat16)
    T = x.shape[0] // 4
    x = x.reshape(T, 1, 64)
    c = Pages4(lib, [T], 1, 64, 128)
    lib.cast_cache_append(x, x, c.cache, c.table, c.kv_len)
    want, code = R4.quantise(f64(x))
    for name in "kv":
        held, scales = c.held(name, 0)
        assert np.array_equal(scales, code) and np.array_equal(held, want)


def test_append_what_is_not_finite_or_too_large(lib):
    x = torch.ones((4, 1, 64), dtype=torch.bfloat16, device="cuda")
    x[0, 0, 3], x[1, 0, 20], x[2, 0, 63], x[3, 0, 5] = float("nan"), float("inf"), float("-inf"), 3e38
    c = Pages4(lib, [4], 1, 64, 16)
    lib.cast_cache_append(x, x, c.cache, c.table, c.kv_len)
    held, scales = c.held("k", 0)
    assert (scales[[0, 1, 2], 0, [0, 1, 3]] == R4.NAN_SCALE).all() and scales[3, 0, 0] == 0xe2
    want = np.ones((4, 64)) * 1.0
    one = R4.quantise(np.ones((1, 16)))[0][0, 0]
    want[:] = one
    want[0, :16], want[1, 16:32], want[2, 48:] = np.nan, np.nan, np.nan
    want[3, :16] = 0
    want[3, 5] = 61440
    assert np.array_equal(held[:, 0], want, equal_nan=True)


# ------------------------------------------------------------------------------------ reading back
READ = [
    # lens, rows, H, d, page
    ([301], [301], 2, 128, 16),
    ([5, 17, 64, 33], [1, 17, 3, 30], 3, 64, 16),
    ([700, 7, 411], [650, 0, 333], 5, 128, 32),
    ([2000, 131], [1999, 90], 1, 64, 64),
    ([300, 1], [290, 1], 13, 128, 128),
]


@pytest.mark.parametrize("lens,new,H,d,page", READ)
@pytest.mark.parametrize("kind", ["f4", "f8", "bf16"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_read(lib, lens, new, H, d, page, kind, dtype):
    g = gen(len(lens) * 3 + d)
    c = Pages4(lib, lens, H, d, page, seed=3, apart=True)
    cache = c.cache
    if kind == "f4":
        want = c.fill(seed=9)
    else:
        n = c.k.shape[0]
        k, v = randn(g, n, page, H, d), randn(g, n, page, H, d)
        ks = vs = None
        if kind == "f8":
            k, v = (100 * k).to(torch.float8_e4m3fn), (100 * v).to(torch.float8_e4m3fn)
            ks, vs = (torch.exp2(torch.randint(-20, 8, (n, H), generator=g, device="cuda").float()) for _ in range(2))
        else:
            k, v = k.to(torch.bfloat16), v.to(torch.bfloat16)
        cache = lib.kv_cache(k, v, ks, vs)
        want = []
        for b, m in enumerate(lens):
            p = c.table[b, :-(-m // page)].long()
            one = lambda x, s: ((x.view(torch.uint8)[p].view(x.dtype) if s is not None else x[p]).double() *
                                (s[p].double()[:, None, :, None] if s is not None else 1)).reshape(-1, H, d)[:m].cpu().numpy()
            want.append((one(k, ks), one(v, vs)))
    cu = i32(*np.concatenate([[0], np.cumsum(new)]))
    T = sum(new)
    room = torch.full((T + 3, 2, H, d), 7.0, dtype=dtype, device="cuda")
    ko, vo = lib.cast_cache_read(cache, c.table, c.kv_len, T + 3, cu_new=cu, dtype=dtype, v_out=room[:, 1])
    lib.cast_check_device()
    assert vo.data_ptr() == room[:, 1].data_ptr() and (room[:, 0] == 7).all() and (room[T:] == 7).all()
    at = 0
    for b, m in enumerate(new):
        for got, ref in ((ko, want[b][0]), (vo, want[b][1])):
            assert np.array_equal(f64(got[at:at + m]), ref[lens[b] - m:], equal_nan=True)   # (a code may be NaN)
        at += m
    only, none = lib.cast_cache_read(cache, c.table, c.kv_len, T, cu_new=cu, dtype=dtype, values=False)
    assert none is None and torch.equal(only.nan_to_num(3.0), ko[:T].nan_to_num(3.0))
    none, only = lib.cast_cache_read(cache, c.table, c.kv_len, T, cu_new=cu, dtype=dtype, keys=False)
    assert none is None and torch.equal(only.nan_to_num(3.0), vo[:T].nan_to_num(3.0))


def test_read_what_is_not_there(lib):
    """Positions below 0 and pages out of range read as zeros; rows past max_new are left as they were."""
    c = Pages4(lib, [40], 2, 64, 16)
    c.fill()
    k, v = lib.cast_cache_read(c.cache, c.table, i32(5), 9)
    lib.cast_check_device()
    assert (k[:4] == 0).all() and (v[:4] == 0).all() and (k[4:] != 0).any()
    table = c.table.clone()
    table[0, 1] = 99
    k, v = lib.cast_cache_read(c.cache, table, c.kv_len, 40)
    with pytest.raises(lib.CastError):
        lib.cast_check_device()
    assert (k[16:32] == 0).all() and (v[16:32] == 0).all() and (k[32:] != 0).any()
    k, _ = lib.cast_cache_read(c.cache, c.table[:, :1], c.kv_len, 40)
    with pytest.raises(lib.CastError):
        lib.cast_check_device()
    assert (k[16:] == 0).all() and (k[:16] != 0).any()
    out = torch.full((40, 2, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    lib.cast_cache_read(c.cache, c.table, c.kv_len, 40, cu_new=i32(0, 40), max_new=7, k_out=out, values=False)
    with pytest.raises(lib.CastError):
        lib.cast_check_device()
    assert (out[7:] == 5).all()
    assert lib.cast_cache_read(c.cache, c.table, c.kv_len, 0)[0].shape == (0, 2, 64)


def test_read_shows_nan_groups(lib):
    c = Pages4(lib, [3], 1, 64, 16)
    c.fill()
    page = int(c.table[0, 0])
    c.vs[page, 0, 1, 2] = R4.NAN_SCALE
    k, v = lib.cast_cache_read(c.cache, c.table, c.kv_len, 3, dtype=torch.float32)
    bad = torch.isnan(v)
    assert not torch.isnan(k).any() and bad[1, 0, 32:48].all() and int(bad.sum()) == 16


def test_read_gives_blocks_that_route(lib):
    """The pages of a 4-bit history as the blocks that the routing takes: the same choice as from the values."""
    M, Bv, H, d = 6, 64, 2, 64
    c = Pages4(lib, [M * Bv], H, d, 16)
    (kq, vq), = c.fill(seed=21)
    k, v = lib.cast_cache_read(c.cache, c.table, c.kv_len, M * Bv)
    q = randn(gen(2), 2, 64, H, d).to(torch.bfloat16)
    want = [torch.from_numpy(x).cuda().to(torch.bfloat16).view(M, Bv, H, d) for x in (kq, vq)]
    a = lib.cast_route_topk(q, [0, 1], k.view(M, Bv, H, d), v.view(M, Bv, H, d), 3)
    b = lib.cast_route_topk(q, [0, 1], *want, 3)
    first = lambda x: x[0] if isinstance(x, tuple) else x
    assert torch.equal(first(a), first(b))


# ------------------------------------------------------------------------------------ attention
def check_attention(lib, c, held, q, new, out, lse, only=None, **kw):
    at = 0
    for b, m in enumerate(new):
        if m == 0:
            continue
        rows = slice(at, at + m)
        o, want, eo, el = R4.attention(f64(q[rows]), *held[b], c.lens[b], **kw)
        got = f64(out[rows]).reshape(o.shape)
        tol = eo + (R.UBF * (np.abs(o) + eo) if out.dtype == torch.bfloat16 else R.U32 * np.abs(o))
        bad = ~(np.abs(got - o) <= tol)
        assert not bad.any(), f"sequence {b}: {bad.sum()} of {bad.size} outside, worst {np.nanmax(np.abs(got - o) / np.maximum(tol, 1e-300)):.3g} x"
        if lse is not None:
            x = lse[rows].cpu().numpy().astype(np.float64)
            assert np.array_equal(np.isinf(x), np.isinf(want))
            f = np.isfinite(want)
            assert (np.abs(x - want)[f] <= el[f]).all()
        at += m


ROWS = [
    # lens, new, H, H_q, d, page, causal, window, sinks
    ([1], [1], 1, 1, 64, 16, True, 0, 0),
    ([301], [1], 2, 8, 64, 16, True, 0, 0),
    ([301, 17, 1, 1500], [1, 1, 1, 1], 3, 12, 128, 16, True, 0, 0),
    ([3000, 2500, 777], [1, 1, 1], 8, 32, 128, 64, True, 0, 0),           # shares cut anywhere
    ([3000, 2500, 777], [1, 1, 1], 2, 30, 64, 128, True, 0, 0),           # 15 rows
    ([2050, 90], [4, 3], 5, 10, 128, 32, True, 0, 0),                     # drafts: 8 rows
    ([2050, 90], [7, 1], 5, 10, 128, 32, False, 0, 0),                    # 14 rows, ragged
    ([4000, 1500, 2], [1, 1, 1], 4, 16, 128, 16, True, 1024, 40),
    ([4000, 1500, 31], [2, 1, 2], 3, 15, 64, 16, True, 333, 5),
    ([900, 1000], [5, 5], 40, 120, 64, 32, True, 0, 0),                   # 15 rows
    ([700] * 33, [1] * 33, 2, 2, 64, 16, False, 100, 0),
    ([500, 400], [8, 8], 33, 99, 64, 16, True, 0, 0),                     # 24 rows, 66 units
    ([1300, 400], [8, 3], 33, 132, 64, 64, True, 200, 17),                # 32 rows
    ([3000, 950, 41], [10, 7, 10], 2, 8, 128, 16, True, 0, 0),            # 40 rows
    ([1100, 950, 41], [5, 1, 5], 3, 15, 128, 64, True, 300, 20),          # 25 rows
    ([2500, 64], [33, 33], 3, 3, 128, 32, False, 0, 0),                   # 33 rows
    ([2500, 77, 8], [8, 8, 8], 2, 16, 64, 16, True, 0, 0),                # 64 rows
    ([800, 50], [13, 50], 2, 2, 64, 128, False, 70, 3),                   # 50 rows
]


@pytest.mark.parametrize("lens,new,H,H_q,d,page,causal,window,sinks", ROWS)
def test_attention_few_rows(lib, lens, new, H, H_q, d, page, causal, window, sinks):
    c = Pages4(lib, lens, H, d, page, seed=H, apart=d == 128)
    held = c.fill(seed=H + d)
    q = (1.5 * randn(gen(d), sum(new), H_q, d)).to(torch.bfloat16)
    cu = i32(*np.concatenate([[0], np.cumsum(new)])) if len(set(new)) > 1 else None
    kw = dict(causal=causal, window=window, sinks=sinks)
    o, lse = lib.cast_cache_attention(q, c.cache, c.table, c.kv_len, cu_new=cu, max_new=max(new), want_lse=True, **kw)
    lib.cast_check_device()
    check_attention(lib, c, held, q, new, o, lse, **kw)
    o32 = lib.cast_cache_attention(q, c.cache, c.table, c.kv_len, cu_new=cu, max_new=max(new), out_dtype=torch.float32, **kw)
    check_attention(lib, c, held, q, new, o32, None, **kw)


TILES = [
    # lens, new, H, H_q, d, page, causal, window, sinks
    ([41], [41], 1, 1, 128, 16, True, 0, 0),
    ([301], [40], 2, 8, 64, 16, True, 0, 0),
    ([200, 500], [129, 77], 1, 3, 64, 16, True, 0, 0),
    ([300, 17, 1000], [130, 5, 64], 3, 3, 128, 32, True, 0, 0),
    ([2000], [300], 2, 2, 128, 64, False, 0, 0),                    # parts joined over CTAs
    ([3000, 1500, 100], [9, 9, 9], 2, 10, 128, 128, True, 0, 0),    # one tile of few rows
    ([2600, 700], [200, 130], 2, 6, 64, 64, True, 500, 4),
    ([2600, 700], [260, 130], 1, 2, 128, 16, False, 700, 130),
    ([1500] * 3, [128] * 3, 5, 5, 128, 64, False, 0, 0),
    ([900, 1], [300, 1], 1, 128, 64, 32, True, 0, 0),
]


@pytest.mark.parametrize("lens,new,H,H_q,d,page,causal,window,sinks", TILES)
def test_attention_many_rows(lib, lens, new, H, H_q, d, page, causal, window, sinks):
    test_attention_few_rows(lib, lens, new, H, H_q, d, page, causal, window, sinks)


HIDDEN = [
    # lens, new, H, H_q, d, page, causal, window, sinks
    ([333], [1], 2, 4, 128, 16, True, 100, 5),
    ([333], [3], 1, 4, 64, 32, True, 0, 0),
    ([333, 200], [40, 12], 2, 4, 128, 16, True, 0, 0),
    ([700], [300], 1, 2, 64, 64, True, 130, 9),
]


@pytest.mark.parametrize("lens,new,H,H_q,d,page,causal,window,sinks", HIDDEN)
def test_attention_never_reads_what_is_hidden(lib, lens, new, H, H_q, d, page, causal, window, sinks):
    """NaN and infinite scales: at positions that no row sees they change nothing; at a position that some rows see,
    those rows alone."""
    kw = dict(causal=causal, window=window, sinks=sinks)
    c = Pages4(lib, lens, H, d, page, seed=2)
    held = c.fill(seed=3)
    T = sum(new)
    q = randn(gen(4), T, H_q, d).to(torch.bfloat16)
    cu = i32(*np.concatenate([[0], np.cumsum(new)]))
    call = lambda: lib.cast_cache_attention(q, c.cache, c.table, c.kv_len, cu_new=cu, max_new=max(new), out_dtype=torch.float32, **kw)
    clean = call()
    at = 0
    for b, (n, m) in enumerate(zip(lens, new)):
        p, j = n - m + np.arange(m)[:, None], np.arange(n)[None, :]
        see = np.ones((m, n), bool)
        if causal:
            see &= j <= p
        if window:
            see &= (j > p - window) | (j < sinks)
        ref, _, eo, _ = R4.attention(f64(q[at:at + m]), *held[b], n, **kw)
        ref, eo = ref.reshape(m, -1), (eo + R.U32 * np.abs(ref)).reshape(m, -1)

        def unchanged(got, rows):
            """Of rows that do not see the token: to the bit where nobody sees it, else within the bound (the tokens of
            its block are added one by one, in another order and by other roundings)."""
            if not rows.any():
                assert torch.equal(got, clean), (b, key)
            assert (np.abs(f64(got[mine]) - ref) <= eo)[~rows.cpu().numpy()].all(), (b, key)

        for bad in (0xff, 0xf8):
            for key in sorted({0, n - 1, n - m, max(0, n - m - window), n // 3}):
                page_of, row = int(c.table[b, key // page]), key % page
                keep = c.vs[page_of, :, row].clone()
                c.vs[page_of, :, row] = bad
                got = call()
                rows = torch.from_numpy(see[:, key]).cuda()
                mine = slice(at, at + m)
                unchanged(got, rows)
                # every channel: a value that is not finite, or infinity times a code of 0
                assert not torch.isfinite(got[mine][rows]).any(), (b, key)
                others = torch.ones(T, dtype=torch.bool, device="cuda")
                others[mine] = False
                assert torch.equal(got[others], clean[others])
                c.vs[page_of, :, row] = keep
                keep = c.ks[page_of, :, row].clone()
                c.ks[page_of, :, row] = bad
                got = call()
                unchanged(got, rows)
                if bad == 0xff:
                    assert torch.isnan(got[mine][rows]).all(), (b, key)
                c.ks[page_of, :, row] = keep
        at += m
    lib.cast_check_device()
    check_attention(lib, c, held, q, new, clean, None, **kw)


@pytest.mark.parametrize("new,d", [(1, 128), (8, 64), (40, 128), (300, 64)])
def test_attention_of_pages_and_rows_that_are_not_there(lib, new, d):
    """A page out of range reads as zeros; a sequence of no tokens gives zeros; rows behind the last are left."""
    c = Pages4(lib, [600, 0], 2, d, 16, seed=8)
    (k, v), _ = c.fill(seed=9)
    table = c.table.clone()
    table[0, 5], table[0, 30] = -1, 10 ** 6
    q = randn(gen(1), 2 * new, 4, d).to(torch.bfloat16)
    out = torch.full((2 * new + 2, 4 * d), 7.0, device="cuda")
    cu = i32(0, new, 2 * new)
    qq = torch.cat([q, q[:2]])
    lib.cast_cache_attention(qq, c.cache, table, c.kv_len, cu_new=cu, max_new=new, causal=False, out=out, out_dtype=torch.float32)
    with pytest.raises(lib.CastError):
        lib.cast_check_device()
    assert (out[2 * new:] == 7).all() and (out[new:2 * new] == 0).all()
    for x in (k, v):
        x[80:96] = 0
        x[480:496] = 0
    check_attention(lib, c, [(k, v), None], q[:new], [new], out[:new], None, causal=False)


@pytest.mark.parametrize("new,H_q,d", [(1, 4, 128), (1, 12, 64), (60, 4, 128), (200, 2, 64)])
def test_attention_of_large_and_small_values(lib, new, H_q, d):
    """Values at the ends of what 4 bits hold; queries at the ends of bf16, rows of zeros."""
    c = Pages4(lib, [700], 2, d, 32, seed=8)
    (k, v), = c.fill(seed=9, scale=9000.0)
    q = randn(gen(1), new, H_q, d).to(torch.bfloat16) * 1e-4
    q[new // 2] = 0
    o, lse = lib.cast_cache_attention(q, c.cache, c.table, c.kv_len, want_lse=True, out_dtype=torch.float32)
    check_attention(lib, c, [(k, v)], q, [new], o, lse)
    (k, v), = c.fill(seed=10, scale=2e-4)
    q = randn(gen(2), new, H_q, d).to(torch.bfloat16) * 2e4
    o, lse = lib.cast_cache_attention(q, c.cache, c.table, c.kv_len, want_lse=True, out_dtype=torch.float32)
    check_attention(lib, c, [(k, v)], q, [new], o, lse)


CUT = [
    # units cut anywhere by the shares: at their first blocks, between units and at their last
    ([20000, 131, 4100, 257], [2, 1, 2, 1], 2, 8, 64, 64, True, 0, 0),
    ([9000] * 7, [1] * 7, 3, 15, 128, 16, True, 4000, 100),
    ([0, 12000, 1], [0, 3, 1], 1, 4, 128, 128, True, 0, 0),
    ([20000, 131, 4100, 257], [9, 20, 40, 64], 2, 8, 64, 64, True, 0, 0),
    ([9000] * 7, [5] * 7, 3, 15, 128, 16, True, 4000, 100),
    ([6000, 6100, 6200], [300, 129, 17], 2, 4, 128, 32, False, 0, 0),
    ([0, 12000, 1], [6, 40, 6], 1, 24, 128, 128, True, 0, 0),
    ([1100 + 130 * i for i in range(9)], [70 - 7 * i for i in range(9)], 5, 5, 64, 16, True, 0, 0),
]


@pytest.mark.parametrize("lens,new,H,H_q,d,page,causal,window,sinks", CUT)
def test_units_cut_anywhere(lib, lens, new, H, H_q, d, page, causal, window, sinks):
    """... also with rows of a sequence shorter than its new tokens, which see nothing."""
    c = Pages4(lib, [max(n, 0) for n in lens], H, d, page, seed=8)
    held = c.fill(seed=9)
    q = (1.5 * randn(gen(3), sum(new), H_q, d)).to(torch.bfloat16)
    kw = dict(causal=causal, window=window, sinks=sinks)
    o, lse = lib.cast_cache_attention(q, c.cache, c.table, c.kv_len, cu_new=i32(*np.concatenate([[0], np.cumsum(new)])), max_new=max(new),
                                      want_lse=True, **kw)
    lib.cast_check_device()
    check_attention(lib, c, held, q, new, o, lse, **kw)


@pytest.mark.parametrize("new", [1, 3, 8, 30])
def test_many_sequences(lib, new):
    """More sequences than a warp has lanes, of very different lengths; enough units that CTAs take whole ones, too."""
    lens = [max(new, (37 * i * i) % 1700) for i in range(70)]
    c = Pages4(lib, lens, 1, 64, 16, seed=2)
    held = c.fill(seed=5)
    n = [min(new, 1 + i % new) for i in range(70)]
    q = randn(gen(1), sum(n), 4, 64).to(torch.bfloat16)
    o, lse = lib.cast_cache_attention(q, c.cache, c.table, c.kv_len, cu_new=i32(*np.concatenate([[0], np.cumsum(n)])), max_new=new, want_lse=True)
    lib.cast_check_device()
    check_attention(lib, c, held, q, n, o, lse)


@pytest.mark.parametrize("new", [2, 60])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_query_that_is_not_finite_stays_its_own(lib, new, bad):
    c = Pages4(lib, [500], 2, 128, 32)
    c.fill(seed=5)
    q = randn(gen(1), new, 4, 128).to(torch.bfloat16)
    want = lib.cast_cache_attention(q, c.cache, c.table, c.kv_len)
    q[1, 2, 77] = bad
    got = lib.cast_cache_attention(q, c.cache, c.table, c.kv_len)
    got, want = got.view(new, 4, 128), want.view(new, 4, 128)
    assert torch.isnan(got[1, 2]).all()
    got[1, 2] = want[1, 2]
    assert torch.equal(got, want)


@pytest.mark.parametrize("new", [1, 90])
def test_table_is_a_slice_shared_and_too_short(lib, new):
    c = Pages4(lib, [900, 333], 2, 64, 16, seed=4)
    held = c.fill(seed=5)
    wide = torch.full((2, 5000), -7, dtype=torch.int32, device="cuda")
    wide[:, 100:100 + c.table.shape[1]] = c.table
    q = randn(gen(1), 2 * new, 4, 64).to(torch.bfloat16)
    o = lib.cast_cache_attention(q, c.cache, wide[:, 100:4100], c.kv_len)
    k, _ = lib.cast_cache_read(c.cache, wide[:, 100:4100], c.kv_len, 600)
    lib.cast_check_device()
    check_attention(lib, c, held, q, [new, new], o, None)
    assert np.array_equal(f64(k[300:]), held[1][0][33:])
    # one table for several sequences, of different lengths
    one = c.table[:1].expand(2, -1)
    o = lib.cast_cache_attention(q, c.cache, one, i32(900, 411))
    lib.cast_check_device()
    two = Pages4.__new__(Pages4)
    two.lens = [900, 411]
    check_attention(lib, two, [held[0], tuple(x[:411] for x in held[0])], q, [new, new], o, None)
    lib.cast_cache_attention(q, c.cache, c.table[:, :30], c.kv_len, causal=False)   # room for 480 of 900
    with pytest.raises(lib.CastError):
        lib.cast_check_device()


@pytest.mark.parametrize("said", [2, 60])
def test_more_new_tokens_than_said_are_left_out(lib, said):
    c = Pages4(lib, [300, 300], 1, 64, 16)
    c.fill(seed=5)
    n = [said, said + 5]
    cu = i32(0, n[0], sum(n))
    q = randn(gen(2), sum(n), 2, 64).to(torch.bfloat16)
    out = torch.full((sum(n), 128), 5.0, dtype=torch.bfloat16, device="cuda")
    lib.cast_cache_attention(q, c.cache, c.table, c.kv_len, cu_new=cu, max_new=said, out=out)
    with pytest.raises(lib.CastError):
        lib.cast_check_device()
    assert (out[n[0] + said:] == 5).all() and not (out[:n[0] + said] == 5).all(1).any()


def test_append_leaves_out_what_is_out_of_range(lib):
    """Pages outside the pool, positions past the table and below 0, tokens past max_new: nothing else is touched."""
    x = randn(gen(1), 40, 2, 64).to(torch.bfloat16)
    c = Pages4(lib, [40], 2, 64, 16, seed=3)
    before = [t.clone() for t in (c.k, c.v, c.ks, c.vs)]
    for table, n, said, rows in ((i32(-1, 5000, -7)[None], i32(40), 40, 0), (c.table[:, :1], i32(40), 40, 16), (c.table, i32(40), 7, 7),
                                 (c.table, i32(9), 40, 9)):
        cu = i32(0, 40)
        lib.cast_cache_append(x, x, c.cache, table, n, cu_new=cu, max_new=said)
        if n.item() == 40:
            with pytest.raises(lib.CastError):
                lib.cast_check_device()
        else:
            lib.cast_check_device()
        p = c.table[0].long()
        changed = (c.ks[p] != before[2][p]).any(-1).any(1).flatten()
        assert int(changed.sum()) == rows and changed[:rows].all()
        for t, was in zip((c.k, c.v, c.ks, c.vs), before):
            t.copy_(was)


def test_append_strided_in_place_and_on_another_stream(lib):
    """Rows of a fused buffer, queries rotated where they lie, a stream of its own; as many heads as there are fetched
    ahead and more."""
    for H in (1, 3, 5, 13):
        g = gen(H)
        buf = randn(g, 50, 4 * H, 128).to(torch.bfloat16)
        q, k, v = buf[:, :2 * H], buf[:, 2 * H:3 * H], buf[:, 3 * H:]
        table = lib.rotary_table(128)
        a, b = (Pages4(lib, [50], H, 128, 32, seed=1) for _ in range(2))
        want = lib.cast_cache_append(k.contiguous(), v.contiguous(), a.cache, a.table, a.kv_len, rotary=table, q=q.contiguous())
        rest = buf[:, 2 * H:].clone()
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        lib.cast_cache_append(k, v, b.cache, b.table, b.kv_len, rotary=table, q=q, q_out=q, stream=s)
        read = lib.cast_cache_read(b.cache, b.table, b.kv_len, 50, stream=s)
        torch.cuda.current_stream().wait_stream(s)
        assert torch.equal(q, want) and torch.equal(buf[:, 2 * H:], rest)
        for x, y in zip(read, lib.cast_cache_read(a.cache, a.table, a.kv_len, 50)):
            assert torch.equal(x, y)


@pytest.mark.parametrize("new,H_q", [(1, 8), (30, 8), (300, 2)])
def test_attention_again_strided_and_on_another_stream(lib, new, H_q):
    c = Pages4(lib, [5000, 900], 2, 64, 16, seed=7)
    c.fill(seed=8)
    buf = randn(gen(2), 2 * new, 3 * H_q, 64).to(torch.bfloat16)
    q = buf[:, H_q:2 * H_q]
    want = lib.cast_cache_attention(q.contiguous(), c.cache, c.table, c.kv_len)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = [lib.cast_cache_attention(q, c.cache, c.table, c.kv_len, stream=s) for _ in range(3)]
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(x, want) for x in got)


def test_attention_with_a_workspace_of_earlier_calls(lib):
    """Calls of every kind one after the other in one workspace that held anything."""
    ws = torch.randint(0, 256, (1 << 28,), dtype=torch.uint8, device="cuda")
    for lens, new, H, H_q, d, page, causal, window, sinks in ROWS[3:6] + CUT + TILES[3:6]:
        c = Pages4(lib, lens, H, d, page, seed=1)
        c.fill(seed=2)
        q = randn(gen(d), sum(new), H_q, d).to(torch.bfloat16)
        kw = dict(cu_new=i32(*np.concatenate([[0], np.cumsum(new)])), max_new=max(new), causal=causal, window=window, sinks=sinks)
        want = lib.cast_cache_attention(q, c.cache, c.table, c.kv_len, **kw)
        assert torch.equal(lib.cast_cache_attention(q, c.cache, c.table, c.kv_len, workspace=ws, **kw), want)
        ws.random_(0, 256)


def test_offsets_beyond_32_bits(lib):
    """Pages far into a pool of more than 2^32 bytes."""
    H, d, page = 8, 128, 128
    n = (1 << 32) // (H * page * d // 2) * 5 // 4 + 3
    assert n * H * page * (d // 16) < 1 << 32 and n * H * page * d // 2 > 1 << 32
    k, v = (torch.empty((n, H, page, d // 2), dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.empty((n, H, page, d // 16), dtype=torch.uint8, device="cuda") for _ in range(2))
    big = lib.kv_cache(k, v, ks, vs)
    c = Pages4(lib, [300], H, d, page)
    c.fill(seed=4)
    far = torch.tensor([[n - 1, n - 3, n // 2 + 1]], dtype=torch.int32, device="cuda")
    for t, x in ((k, c.k), (v, c.v), (ks, c.ks), (vs, c.vs)):
        t[far[0].long()] = x[c.table[0].long()]
    for new in (1, 50):
        q = randn(gen(new), new, 16, d).to(torch.bfloat16)
        assert torch.equal(lib.cast_cache_attention(q, big, far, c.kv_len), lib.cast_cache_attention(q, c.cache, c.table, c.kv_len))
    x = randn(gen(9), 140, H, d).to(torch.bfloat16)
    for cache, table in ((big, far), (c.cache, c.table)):
        lib.cast_cache_append(x, x, cache, table, c.kv_len)
    for a, b in zip(lib.cast_cache_read(big, far, c.kv_len, 300), lib.cast_cache_read(c.cache, c.table, c.kv_len, 300)):
        assert torch.equal(a, b)
    lib.cast_check_device()


def test_a_session_in_a_graph(lib):
    """What serving does: prompts appended and attended to, then token by token the append, the attention and the reading
    of the last page in one captured graph, replayed as the lengths grow; against 64 bits and against eager calls."""
    B, H, H_q, d, page = 3, 2, 8, 128, 16
    c = Pages4(lib, [200] * B, H, d, page, seed=5)
    table = lib.rotary_table(d)
    g = gen(1)
    new = [100, 31, 64]
    c.lens, c.kv_len = new, i32(*new)
    cu = i32(*np.concatenate([[0], np.cumsum(new)]))
    qkv = randn(g, sum(new), H_q + 2 * H, d).to(torch.bfloat16)
    split = lambda x: (x[:, :H_q], x[:, H_q:H_q + H], x[:, H_q + H:])
    q, k, v = split(qkv)
    turned = lib.cast_cache_append(k, v, c.cache, c.table, c.kv_len, cu_new=cu, rotary=table, q=q)
    o, lse = lib.cast_cache_attention(turned, c.cache, c.table, c.kv_len, cu_new=cu, want_lse=True)
    held = [tuple(c.held(x, b)[0] for x in "kv") for b in range(B)]
    check_attention(lib, c, held, turned, new, o, lse)
    x = randn(g, B, H_q + 2 * H, d).to(torch.bfloat16)
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")

    def step():
        c.kv_len += 1
        q, k, v = split(x)
        turned = lib.cast_cache_append(k, v, c.cache, c.table, c.kv_len, rotary=table, q=q)
        return (turned, lib.cast_cache_attention(turned, c.cache, c.table, c.kv_len, window=150, sinks=4, workspace=ws),
                *lib.cast_cache_read(c.cache, c.table, c.kv_len, B * 7))

    step()   # not captured: loads what a first call loads
    x.copy_(randn(g, *x.shape))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(20):
        x.copy_(randn(g, *x.shape))
        graph.replay()
        if i % 6:
            continue
        c.lens = [n + 2 + i for n in new]
        assert c.kv_len.tolist() == c.lens
        held = [tuple(c.held(y, b)[0] for y in "kv") for b in range(B)]
        check_attention(lib, c, held, out[0], [1] * B, out[1], None, window=150, sinks=4)
        for b in range(B):
            for y, z in zip(out[2:], held[b]):
                assert np.array_equal(f64(y[7 * b:7 * b + 7]), z[-7:])
        again = [t.clone() for t in out]
        c.kv_len -= 1
        for a, b in zip(again, step()):
            assert torch.equal(a, b)
    lib.cast_check_device()


@pytest.mark.parametrize("bits", [4, 8])
def test_rollout_example(lib, bits):
    """The example's steps with 4-bit pages against 64 bits, and its chunk routed over pages that are read back."""
    from examples.cache_rollout import Rollout
    r = Rollout(H=2, H_q=4, d=64, grid=(8, 8), page=64, n_pages=16, bits=bits, window=150)
    for tokens, causal in ((64, False), (64, False), (1, True), (64, False), (64, False), (1, True)):
        (q, k, v, pos), turned, o = r.step(tokens, causal)
        kk, vv = lib.cast_cache_read(r.cache, r.table, r.kv_len, r.len, dtype=torch.float32)
        if bits == 4:
            ref, err = R.rotate(f64(k), pos.cpu().numpy(), 64, sections=[32 - 2 * 12, 12, 12])
            page = lambda t: t.transpose(1, 2).reshape(-1, 2, t.shape[-1])[r.len - tokens:r.len].cpu().numpy()
            R4.check_quantised(f64(kk[r.len - tokens:]), page(r.cache._keep[2]), ref, err)
            want, _, eo, _ = R4.attention(f64(turned), f64(kk), f64(vv), r.len, causal, 150, 64)
            assert (np.abs(f64(o).reshape(want.shape) - want) <= eo + R.UBF * (np.abs(want) + eo)).all()
    k, v = r.blocks()
    assert k.shape == (r.len // 64, 64, 2, 64) and torch.equal(k.reshape(-1, 2, 64).float(), kk[:r.len // 64 * 64])
    assert torch.isfinite(r.routed_chunk(n_frames=3, anchors=(0, 2), K=2).float()).all()
    lib.cast_check_device()


def test_pages_of_the_type_of_two_values(lib):
    if not hasattr(torch, "float4_e2m1fn_x2"):
        pytest.skip("no such type")
    c = Pages4(lib, [100], 2, 64, 16)
    c.fill()
    other = lib.kv_cache(c.k.view(torch.float4_e2m1fn_x2), c.v.view(torch.float4_e2m1fn_x2), c.ks, c.vs)
    for a, b in zip(lib.cast_cache_read(c.cache, c.table, c.kv_len, 100), lib.cast_cache_read(other, c.table, c.kv_len, 100)):
        assert torch.equal(a, b)


def test_binding_refuses_tensors_that_are_not_on_the_gpu(lib):
    c = Pages4(lib, [100], 2, 64, 16)
    host = lib.kv_cache(*(t.cpu() for t in (c.k, c.v, c.ks, c.vs)))
    some = lib.kv_cache(c.k, c.v, c.ks, c.vs.cpu())
    out = torch.empty((5, 2, 64), dtype=torch.bfloat16)
    for call in (lambda: lib.cast_cache_read(host, c.table, c.kv_len, 5), lambda: lib.cast_cache_read(some, c.table, c.kv_len, 5),
                 lambda: lib.cast_cache_read(c.cache, c.table.cpu(), c.kv_len, 5), lambda: lib.cast_cache_read(c.cache, c.table, c.kv_len.cpu(), 5),
                 lambda: lib.cast_cache_read(c.cache, c.table, c.kv_len, 5, cu_new=torch.tensor([0, 5], dtype=torch.int32)),
                 lambda: lib.cast_cache_read(c.cache, c.table, c.kv_len, 5, k_out=out), lambda: lib.cast_cache_read(c.cache, c.table, c.kv_len, 5, v_out=out)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new,H_q", [(1, 6), (2, 12), (3, 20), (50, 8)])
def test_every_page_size_and_form(lib, page, d, new, H_q):
    """Blocks and tiles of several pages and of parts of one, whole units and shares, sinks and windows that begin and end
    inside pages, with whole pages between them that no row sees, whose table entries are out of range."""
    H, lens, window, sinks = 2, [3001, 1400, 77], 333, 21
    c = Pages4(lib, lens, H, d, page, seed=page + d)
    held = c.fill(seed=page)
    q = (1.5 * randn(gen(new), 3 * new, H_q, d)).to(torch.bfloat16)
    for kw, table in ((dict(), c.table), (dict(window=window, sinks=sinks), c.table.clone())):
        if kw:
            for b, n in enumerate(lens):
                first, last = -(-sinks // page), max(0, n - new - window + 1) // page   # pages that no row sees
                if last > first:
                    table[b, first:last] = -5
        o, lse = lib.cast_cache_attention(q, c.cache, table, c.kv_len, want_lse=True, **kw)
        lib.cast_check_device()
        check_attention(lib, c, held, q, [new] * 3, o, lse, **kw)
    # a short table: at most 1024 tokens, so that every CTA has a whole unit
    short = [min(n, 1024) for n in lens]
    o, lse = lib.cast_cache_attention(q, c.cache, c.table[:, :1024 // page], i32(*short), want_lse=True)
    lib.cast_check_device()
    some = Pages4.__new__(Pages4)
    some.lens = short
    check_attention(lib, some, [tuple(x[:n] for x in h) for h, n in zip(held, short)], q, [new] * 3, o, lse)
