"""The paged KV cache on the GPU against 64 bits: rotary positions, the append, the attention."""
import numpy as np
import pytest
import torch

from tests import cache_ref as R

pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def within(got, ref, tol, what):
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} outside, worst {np.nanmax(np.abs(got - ref) / np.maximum(tol, 1e-300)):.3g} x"


# ------------------------------------------------------------------------------------ rotary
ROTARY = [
    # T, H, d, rot, layout, axes, dtype, scaling
    (1, 1, 64, 64, "half", None, torch.float32, None),
    (5, 3, 128, 128, "half", None, torch.bfloat16, ("linear", 4.0)),
    (513, 12, 128, 128, "interleaved", [16, 24, 24], torch.bfloat16, None),
    (77, 5, 96, 48, "half", None, torch.float32, ("parts", 8.0, 4096)),
    (33, 2, 256, 256, "interleaved", None, torch.float32, ("stretch", 4.0)),
    (2, 40, 16, 16, "half", [4, 4], torch.float32, None),
    (1001, 1, 64, 32, "half", None, torch.bfloat16, None),
]


@pytest.mark.parametrize("T,H,d,rot,layout,sections,dtype,scaling", ROTARY)
@pytest.mark.parametrize("inverse", [False, True])
def test_rotary(lib, T, H, d, rot, layout, sections, dtype, scaling, inverse):
    g = gen(T * 7 + d)
    table = lib.rotary_table(rot, layout, sections=sections, scaling=scaling)
    x = randn(g, T, H, d).to(dtype)
    pos = torch.randint(-500, 1 << 20, (T, len(sections or [0])), generator=g, device="cuda", dtype=torch.int32)
    y = lib.cast_rotary(x, pos, table, inverse=inverse)
    ref, err = R.rotate(f64(x), pos.cpu().numpy(), rot, layout, inverse, sections=sections, scaling=scaling)
    within(f64(y), ref, err + (R.UBF * (np.abs(ref) + err) if dtype == torch.bfloat16 else 0), "rotary")
    assert torch.equal(y[..., rot:], x[..., rot:])


def test_rotary_at_the_ends_of_int32(lib):
    table = lib.rotary_table(64)
    pos = torch.tensor([0, 1, -1, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda")
    x = randn(gen(3), 5, 2, 64)
    y = lib.cast_rotary(x, pos, table)
    # frequencies are kept to 53 bits: at 2^31 the angle is off by 2^31 2^-53 radians, far below f32
    f, _, _ = R.frequencies(64)
    ref, err = R.rotate(f64(x), pos.cpu().numpy()[:, None], 64)
    within(f64(y), ref, err + 4e-6, "rotary")
    assert torch.equal(y[0], x[0])


def test_rotary_in_place_strided_and_on_another_stream(lib):
    table = lib.rotary_table(128, "interleaved")
    buf = randn(gen(5), 50, 3, 4, 128).to(torch.bfloat16)
    x = buf[:, 1]                                    # rows 3 * 4 * 128 apart
    pos = torch.arange(50, dtype=torch.int32, device="cuda")
    want = lib.cast_rotary(x.contiguous(), pos, table)
    before = buf.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    lib.cast_rotary(x, pos, table, out=x, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(x, want)
    assert torch.equal(buf[:, 0], before[:, 0]) and torch.equal(buf[:, 2], before[:, 2])


def test_rotary_inverse_is_the_gradient(lib):
    """<rotate(x), w> differentiated: by the formula's transpose (an exact inner product) and by
    differences along random directions (the map is linear, so differences have no truncation)."""
    g = gen(11)
    table = lib.rotary_table(64, "half", scaling=("parts", 4.0, 2048))
    pos = torch.randint(0, 9999, (40,), generator=g, device="cuda", dtype=torch.int32)
    x, w, dx = (randn(g, 40, 3, 96) for _ in range(3))
    grad = lib.cast_rotary(w, pos, table, inverse=True)
    ref, err = R.rotate(f64(w), pos.cpu().numpy()[:, None], 64, inverse=True, scaling=("parts", 4.0, 2048))
    within(f64(grad), ref, err, "gradient")
    moved = f64(lib.cast_rotary(x + dx, pos, table)) - f64(lib.cast_rotary(x, pos, table))
    by_difference, by_gradient = (moved * f64(w)).sum(), (f64(grad) * f64(dx)).sum()
    # every term carries a few roundings of its factors
    bound = 32 * R.U32 * (np.abs(f64(w)) * (np.abs(f64(x)) + np.abs(f64(dx)) + np.abs(moved))).sum() * 1.3
    assert abs(by_difference - by_gradient) <= bound


def test_rotary_of_no_tokens(lib):
    y = lib.cast_rotary(torch.empty((0, 2, 64), device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"), lib.rotary_table(64))
    assert y.shape == (0, 2, 64)


# ------------------------------------------------------------------------------------ a cache in use
class Pages:
    """A paged cache of B sequences with NaN wherever nothing was stored, pages in no order."""

    def __init__(self, lib, lens, H, d, page, f8, seed=0, spare=2, interleaved=False):
        g = gen(seed)
        self.lens, self.page, self.f8, self.H, self.d = list(lens), page, f8, H, d
        need = [-(-n // page) for n in lens]
        self.n_pages, per = sum(need) + spare, max(need + [1])
        order = torch.randperm(self.n_pages, generator=g, device="cuda").to(torch.int32)
        self.table = torch.full((len(lens), per), -1, dtype=torch.int32, device="cuda")
        at = 0
        for b, c in enumerate(need):
            self.table[b, :c] = order[at:at + c]
            at += c
        shape = (self.n_pages, page, 2, H, d) if interleaved else (2, self.n_pages, page, H, d)
        if f8:
            buf = torch.full(shape, 0x7f, dtype=torch.uint8, device="cuda").view(F8)
        else:
            buf = torch.full(shape, float("nan"), dtype=torch.bfloat16, device="cuda")
        self.k, self.v = (buf[:, :, 0], buf[:, :, 1]) if interleaved else (buf[0], buf[1])
        self.ks = torch.full((self.n_pages, H), float("nan"), device="cuda") if f8 else None
        self.vs = torch.full((self.n_pages, H), float("nan"), device="cuda") if f8 else None
        self.cache = lib.kv_cache(self.k, self.v, self.ks, self.vs)

    def len_tensor(self, lens=None):
        return torch.tensor(self.lens if lens is None else lens, dtype=torch.int32, device="cuda")

    def fill(self, seed, amp=1.0):
        """Random rows at every position below the lengths (8 bits: scales 2^-8 .. 2^-5)."""
        g = gen(seed)
        for b, n in enumerate(self.lens):
            for i in range(-(-n // self.page)):
                p, m = int(self.table[b, i]), min(self.page, n - i * self.page)
                for c, s in ((self.k, self.ks), (self.v, self.vs)):
                    x = randn(g, m, self.H, self.d)
                    if self.f8:
                        c.view(torch.uint8)[p, :m] = (x * 90).clamp(-448, 448).to(F8).view(torch.uint8)
                        s[p] = torch.exp2(torch.randint(-8, -4, (self.H,), generator=g, device="cuda").float()) * amp
                    else:
                        c[p, :m] = (x * amp).to(torch.bfloat16)
        return self

    def rows(self, b, n=None):
        """k, v [n, H, d] of sequence b in 64 bits, NaN where nothing is stored."""
        n = self.lens[b] if n is None else n
        pages = -(-n // self.page)
        t = self.table[b, :pages].cpu().numpy()
        out = []
        for c, s in ((self.k, self.ks), (self.v, self.vs)):
            x = f64(c.contiguous())
            if self.f8:
                x = x * f64(s)[:, None, :, None]
            x = np.where((t >= 0)[:, None, None, None], x[np.maximum(t, 0)], np.nan)
            out.append(x.reshape(-1, self.H, self.d)[:n])
        return out


# ------------------------------------------------------------------------------------ append
APPEND = [
    # lens before, new, H, H_q, d, page, rot, layout
    ([0], [1], 1, 0, 64, 16, 64, "half"),
    ([15, 0, 16, 33], [1, 1, 1, 1], 4, 16, 128, 16, 128, "half"),
    ([5, 130, 0, 64], [300, 1, 65, 0], 3, 12, 64, 32, 32, "interleaved"),
    ([100], [700], 12, 12, 128, 64, 128, "half"),
    ([1, 127], [129, 128], 9, 0, 128, 128, 64, "interleaved"),
]


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("before,new,H,Hq,d,page,rot,layout", APPEND)
def test_append(lib, before, new, H, Hq, d, page, rot, layout, f8):
    lens = [a + b for a, b in zip(before, new)]
    P = Pages(lib, lens, H, d, page, f8, seed=1, interleaved=H == 9)
    g = gen(17)
    table = lib.rotary_table(rot, layout)

    def step(start, count, amp):
        T = sum(count)
        k, v = ((amp * randn(g, T, H, d)).to(torch.bfloat16) for _ in range(2))
        q = randn(g, T, Hq, d).to(torch.bfloat16) if Hq else None
        cu = torch.tensor(np.concatenate([[0], np.cumsum(count)]), dtype=torch.int32, device="cuda")
        out = lib.cast_cache_append(k, v, P.cache, P.table, P.len_tensor([a + b for a, b in zip(start, count)]), cu_new=cu,
                                    max_new=max(count), rotary=table, q=q)
        return f64(k), f64(v), q, out

    old = step([0] * len(before), before, 1.0) if sum(before) else (np.zeros((0, H, d)),) * 2
    held = [P.rows(b, before[b]) for b in range(len(before))]
    scales = None if not f8 else (f64(P.ks), f64(P.vs))
    k, v, q, q_out = step(before, new, 3.0)
    lib.cast_check_device()
    at = 0
    for b in range(len(before)):
        p0, n = before[b], new[b]
        pos = np.arange(p0, p0 + n)[:, None]
        kr, kerr = R.rotate(k[at:at + n], pos, rot, layout)
        if Hq and n:
            qr, qerr = R.rotate(f64(q[at:at + n]), pos, rot, layout)
            within(f64(q_out[at:at + n]), qr, qerr + R.UBF * (np.abs(qr) + qerr), "q")
        for got, ref, err, was, sc in zip(P.rows(b), (kr, v[at:at + n]), (kerr, 0 * kerr), held[b],
                                          scales or (None, None)):
            if not f8:
                within(got[p0:], ref, err + R.UBF * (np.abs(ref) + err) * (err > 0), "row")
                assert np.array_equal(got[:p0], was)
                continue
            stored = f64(P.ks if ref is kr else P.vs)
            for i in range(p0 // page, -(-(p0 + n) // page) if n else 0):
                lo, hi, pg = max(i * page, p0), min(i * page + page, p0 + n), int(P.table[b, i])
                for h in range(H):
                    want = R.page_scale(np.abs(ref[lo - p0:hi - p0, h]).max())
                    if lo % page:
                        want = max(want, sc[pg, h])
                        ow = was[i * page:lo, h]
                        assert np.array_equal(got[i * page:lo, h], R.e4m3(ow / want) * want)
                    assert stored[pg, h] == want
                    x = ref[lo - p0:hi - p0, h] / want
                    half = R.e4m3_step(x) / 2
                    within(got[lo:hi, h] / want, x, half + err[lo - p0:hi - p0, h] / want, "code")
        at += n


def test_append_growing_scale_keeps_codes(lib):
    """Tokens that arrive one by one, each larger: what is held changes by subnormals only."""
    P = Pages(lib, [12], 2, 64, 16, True)
    g = gen(2)
    want = []
    for i in range(12):
        x = (randn(g, 1, 2, 64) * 2.0 ** i).to(torch.bfloat16)
        lib.cast_cache_append(x, x, P.cache, P.table, P.len_tensor([i + 1]))
        want.append(f64(x)[0])
    k, v = P.rows(0)
    scale = f64(P.ks)[int(P.table[0, 0])]
    for i, x in enumerate(want):
        # one rounding at the scale of the time, one more at the final scale (its subnormal step)
        tol = np.maximum(np.abs(x) * 2.0 ** -4, scale[:, None] * 2.0 ** -10) + scale[:, None] * 2.0 ** -10
        within(k[i], x, tol, "k")
        assert np.array_equal(k[i], v[i])


def test_append_of_values_that_are_not_finite_and_of_extremes(lib):
    P = Pages(lib, [4], 1, 64, 16, True)
    x = torch.zeros((4, 1, 64), dtype=torch.bfloat16, device="cuda")
    x[0, 0, 0], x[0, 0, 1], x[1, 0, 2], x[2, 0, 3] = float("inf"), float("nan"), 3.0e38, 1.0
    lib.cast_cache_append(x, torch.zeros_like(x), P.cache, P.table, P.len_tensor())
    k, v = P.rows(0)
    assert np.isnan(k[0, 0, :2]).all() and np.isfinite(k[1:]).all() and np.isfinite(k[0, 0, 2:]).all()
    assert abs(k[1, 0, 2] / 3.0e38 - 1) <= 2.0 ** -4
    assert (v == 0).all()
    lib.cast_check_device()


def test_append_leaves_out_what_is_out_of_range(lib):
    P = Pages(lib, [40, 10], 2, 64, 16, False)
    P.table[0, 1] = P.n_pages          # the sequence's second page does not exist
    before = P.k.clone()
    x = torch.ones((50, 2, 64), dtype=torch.bfloat16, device="cuda")
    cu = torch.tensor([0, 40, 50], dtype=torch.int32, device="cuda")
    lib.cast_cache_append(x, x, P.cache, P.table, P.len_tensor(), cu_new=cu, max_new=40)
    with pytest.raises(lib.CastError) as e:
        lib.cast_check_device()
    assert e.value.status == lib.ERR_INVALID_ARG
    lib.cast_check_device()
    done = {int(P.table[0, 0]), int(P.table[0, 2]), int(P.table[1, 0])}
    for p in range(P.n_pages):
        if p in done:
            assert not torch.equal(P.k[p].view(torch.int16), before[p].view(torch.int16))
        else:
            assert torch.equal(P.k[p].view(torch.int16), before[p].view(torch.int16))


# ------------------------------------------------------------------------------------ attention
ATTEND = [
    # lens, new, H, H_q, d, page, causal, window, sinks
    ([1], [1], 1, 1, 64, 16, True, 0, 0),
    ([17, 16, 300], [1, 1, 1], 2, 8, 64, 16, True, 0, 0),
    ([2500, 1, 777, 0], [1, 1, 1, 0], 4, 4, 128, 32, True, 0, 0),
    ([5000, 333], [1, 1], 1, 8, 128, 64, True, 1000, 37),
    ([1200, 64, 65], [3, 5, 2], 3, 9, 64, 128, True, 100, 4),
    ([1200, 64, 65], [3, 5, 2], 3, 9, 128, 16, False, 40, 200),
    ([5], [9], 2, 4, 64, 16, True, 0, 0),             # the first four rows see nothing
    ([0, 3], [4, 3], 2, 4, 128, 16, True, 2, 1),
    ([700, 90], [200, 90], 2, 4, 64, 16, True, 0, 0),
    ([900], [257], 1, 3, 128, 64, True, 130, 5),
    ([513, 1000], [130, 300], 2, 2, 128, 32, False, 0, 0),
    ([640], [640], 2, 10, 128, 128, True, 1, 0),
    ([2000], [150], 1, 1, 64, 64, False, 64, 100),
    ([400, 3, 1030], [33, 3, 1], 1, 24, 64, 32, True, 0, 0),
    ([200], [3], 1, 100, 128, 16, True, 0, 0),        # a group that fills most of a tile
    ([3000, 1500, 40], [700, 300, 40], 2, 6, 128, 64, True, 0, 0),
    ([4000, 1, 2600], [150, 1, 513], 3, 3, 64, 16, True, 900, 200),
    ([2900], [130], 2, 2, 128, 128, False, 0, 0),
    ([1400] * 20, [17 + i for i in range(20)], 1, 2, 64, 32, True, 0, 0),
]


def attend(lib, P, new, Hq, causal, window, sinks, seed=5, dtype=torch.bfloat16, amp=1.0, **kw):
    q = (amp * randn(gen(seed), sum(new), Hq, P.d)).to(torch.bfloat16)
    cu = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device="cuda")
    o, lse = lib.cast_cache_attention(q, P.cache, P.table, P.len_tensor(), cu_new=cu, max_new=max(new), causal=causal,
                                      window=window, sinks=sinks, want_lse=True, out_dtype=dtype, **kw)
    return q, o, lse


def check(P, q, o, lse, new, Hq, causal, window, sinks, scale=None):
    at = 0
    o, lse = f64(o).reshape(-1, Hq, P.d), f64(lse)
    for b, n in enumerate(new):
        k, v = P.rows(b)
        ref, rl, eo, el = R.attention(f64(q[at:at + n]), k, v, n, P.lens[b], causal, window, sinks, scale)
        within(o[at:at + n], ref, eo, f"o of sequence {b}")
        none = np.isneginf(rl)
        assert np.array_equal(none, np.isneginf(lse[at:at + n]))
        within(np.where(none, 0, lse[at:at + n]), np.where(none, 0, rl), el, f"lse of sequence {b}")
        at += n


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("lens,new,H,Hq,d,page,causal,window,sinks", ATTEND)
def test_attention(lib, lens, new, H, Hq, d, page, causal, window, sinks, f8):
    P = Pages(lib, lens, H, d, page, f8, seed=3, interleaved=H == 3).fill(4)
    q, o, lse = attend(lib, P, new, Hq, causal, window, sinks)
    lib.cast_check_device()
    check(P, q, o, lse, new, Hq, causal, window, sinks)


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("new", [1, 5, 200])
def test_pages_that_no_row_sees_are_not_read(lib, f8, new):
    """A sequence whose pages between the sinks and the window were given back."""
    P = Pages(lib, [3000], 2, 64, 32, f8, seed=8).fill(9)
    window, sinks = 300, 40
    lo = 3000 - new - window + 1
    for i in range(2, lo // 32):
        P.table[0, i] = -1
    q, o, lse = attend(lib, P, [new], 4, True, window, sinks)
    lib.cast_check_device()
    check(P, q, o, lse, [new], 4, True, window, sinks)


@pytest.mark.parametrize("new", [1, 6, 140])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_values_that_are_not_finite_stay_where_they_are_seen(lib, new, bad):
    """A key and a value row that only some of the rows see: the others are not touched by it."""
    L, window = 1000, 100
    P = Pages(lib, [L], 1, 128, 16, False, seed=8).fill(9)
    for pos in (L - 1, L - 3, L - new - window + 2):
        if pos < L:
            page, row = int(P.table[0, pos // 16]), pos % 16
            P.v[page, row, 0, 5] = bad
    q, o, lse = attend(lib, P, [new], 2, True, window, 0)
    lib.cast_check_device()
    o = f64(o).reshape(new, 2, 128)
    for i in range(new):
        p = L - new + i
        seen = [x for x in (L - 1, L - 3, L - new - window + 2) if x <= p and x > p - window]
        assert np.isfinite(np.delete(o[i], 5, axis=1)).all()
        assert np.isfinite(o[i, :, 5]).all() == (not seen), (i, seen)


def test_eight_bit_codes_of_every_kind(lib):
    """All finite codes, subnormal ones among them, at scales from tiny to large; and NaN is NaN."""
    P = Pages(lib, [64], 1, 64, 16, True).fill(1)
    codes = torch.arange(256, dtype=torch.int32, device="cuda").to(torch.uint8)
    codes[codes.int() % 128 == 127] = 0
    for i in range(4):
        p = int(P.table[0, i])
        P.v.view(torch.uint8)[p, :, 0] = codes.roll(i * 64 + 1).repeat(4).view(16, 64)
        P.vs[p, 0] = 2.0 ** [-100, -3, 7, 60][i]
        P.k.view(torch.uint8)[p].zero_()
    for scales in ([0, 0, 0, 0], [-100, -90, -98, -95], [9, 12, 10, 60]):
        for i in range(4):
            P.vs[int(P.table[0, i]), 0] = 2.0 ** scales[i]
        q, o, lse = attend(lib, P, [1], 1, True, 0, 0, dtype=torch.float32)
        check(P, q, o, lse, [1], 1, True, 0, 0)
    P.v.view(torch.uint8)[int(P.table[0, 2]), 3, 0, 7] = 0x7f
    for new in (1, 40):
        q, o, lse = attend(lib, P, [new], 1, False, 0, 0)
        bad = np.isnan(f64(o).reshape(new, 64))
        assert bad[:, 7].all() and bad.sum() == new


def test_large_logits_do_not_overflow(lib):
    for f8 in (False, True):
        for new in (1, 150):
            P = Pages(lib, [500], 1, 128, 64, f8).fill(2)
            q, o, lse = attend(lib, P, [new], 2, True, 0, 0, amp=300.0)
            check(P, q, o, lse, [new], 2, True, 0, 0)


def test_offsets_beyond_32_bits(lib):
    """Pages whose rows lie more than 2^32 elements from the cache's first."""
    H, d, page = 2, 128, 128
    n = (1 << 32) // (page * H * d) + 5
    k = torch.empty((n, page, H, d), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    cache = lib.kv_cache(k, v)
    table = torch.tensor([[n - 1, 0, n - 2]], dtype=torch.int32, device="cuda")
    g = gen(1)
    for new in (1, 380):
        x = randn(g, 380, H, d).to(torch.bfloat16)
        y = randn(g, 380, H, d).to(torch.bfloat16)
        lib.cast_cache_append(x, y, cache, table, torch.tensor([380], dtype=torch.int32, device="cuda"))
        q = randn(g, new, 4, d).to(torch.bfloat16)
        o = lib.cast_cache_attention(q, cache, table, torch.tensor([380], dtype=torch.int32, device="cuda"))
        ref, _, eo, _ = R.attention(f64(q), f64(x), f64(y), new, 380)
        within(f64(o).reshape(new, 4, d), ref, eo, "o")
    lib.cast_check_device()


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("new,Hq", [(1, 4), (90, 4)])
def test_attention_again_strided_in_f32_and_on_another_stream(lib, f8, new, Hq):
    """The same call twice gives the same bits; q may be a slice of wider rows; an own scale."""
    P = Pages(lib, [4000, 900], 2, 128, 16, f8, seed=3).fill(4)
    wide = randn(gen(6), 2 * new, 3, Hq, 128).to(torch.bfloat16)
    q = wide[:, 1]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    args = dict(causal=True, window=2100, sinks=9, scale=0.05, want_lse=True, out_dtype=torch.float32)
    with torch.cuda.stream(s):
        o, lse = lib.cast_cache_attention(q, P.cache, P.table, P.len_tensor(), stream=s, **args)
    torch.cuda.current_stream().wait_stream(s)
    again, lse2 = lib.cast_cache_attention(q.contiguous(), P.cache, P.table, P.len_tensor(), **args)
    assert torch.equal(o, again) and torch.equal(lse, lse2)
    check(P, q, o, lse, [new, new], Hq, True, 2100, 9, 0.05)


def test_attention_reports_what_is_out_of_range(lib):
    P = Pages(lib, [100], 1, 64, 16, False).fill(1)
    P.table[0, 2] = P.n_pages + 7
    for new in (1, 70):
        attend(lib, P, [new], 1, True, 0, 0)
        with pytest.raises(lib.CastError) as e:
            lib.cast_check_device()
        assert e.value.status == lib.ERR_INVALID_ARG
        lib.cast_check_device()


def test_attention_of_no_rows(lib):
    P = Pages(lib, [10], 1, 64, 16, False).fill(1)
    o = lib.cast_cache_attention(torch.empty((0, 2, 64), dtype=torch.bfloat16, device="cuda"), P.cache, P.table, P.len_tensor())
    assert o.shape == (0, 128)


def test_attention_in_a_graph_follows_the_lengths(lib):
    """Lengths and pages live on the device: a captured step replays at every length."""
    P = Pages(lib, [600], 2, 64, 16, False).fill(1)
    q = randn(gen(3), 1, 4, 64).to(torch.bfloat16)
    n = P.len_tensor([600])
    out = torch.empty((1, 256), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    lib.cast_cache_attention(q, P.cache, P.table, n, out=out, workspace=ws)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        lib.cast_cache_attention(q, P.cache, P.table, n, out=out, workspace=ws)
    for length in (600, 1, 333, 0):
        n.fill_(length)
        g.replay()
        k, v = P.rows(0)
        ref, _, eo, _ = R.attention(f64(q), k[:length], v[:length], 1, length)
        within(f64(out).reshape(1, 4, 64), ref, eo, f"length {length}")


@pytest.mark.parametrize("new", [1, 40])
def test_scales_far_apart_within_a_sequence(lib, new):
    """V pages whose scales differ by up to 2^80, the largest first, last and in between: what small pages
    weigh in the sum counts in full, and their values to the bound that the largest allows."""
    for order in ([40, -40, 0, -3], [-40, 0, 40, -3], [-40, -3, 0, 40], [-120, -120, -120, -120], [100, 98, 100, 99]):
        P = Pages(lib, [256], 1, 64, 64, True).fill(3)
        for i, e in enumerate(order):
            P.vs[int(P.table[0, i]), 0] = 2.0 ** e
        q, o, lse = attend(lib, P, [new], 2, True, 0, 0, dtype=torch.float32)
        check(P, q, o, lse, [new], 2, True, 0, 0)


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("new", [1, 3, 8, 30])
def test_many_sequences(lib, f8, new):
    """More sequences than a warp has lanes, of very different lengths."""
    lens = [max(new, (37 * i * i) % 1700) for i in range(70)]
    P = Pages(lib, lens, 1, 64, 16, f8, seed=2).fill(5)
    n = [min(new, 1 + i % new) for i in range(70)]
    q, o, lse = attend(lib, P, n, 4, True, 0, 0)
    lib.cast_check_device()
    check(P, q, o, lse, n, 4, True, 0, 0)


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("new", [2, 60])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_query_that_is_not_finite_stays_its_own(lib, f8, new, bad):
    P = Pages(lib, [500], 2, 128, 32, f8).fill(5)
    q = randn(gen(1), new, 4, 128).to(torch.bfloat16)
    want = lib.cast_cache_attention(q, P.cache, P.table, P.len_tensor())
    q[1, 2, 77] = bad
    got = lib.cast_cache_attention(q, P.cache, P.table, P.len_tensor())
    got, want = got.view(new, 4, 128), want.view(new, 4, 128)
    assert torch.isnan(got[1, 2]).all()
    got[1, 2] = want[1, 2]
    assert torch.equal(got, want)


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("new", [1, 90])
def test_table_is_a_slice_and_longer_than_needed(lib, f8, new):
    P = Pages(lib, [900, 333], 2, 64, 16, f8, seed=4).fill(5)
    wide = torch.full((2, 5000), -7, dtype=torch.int32, device="cuda")
    wide[:, 100:100 + P.table.shape[1]] = P.table
    P.table = wide[:, 100:4100]
    q, o, lse = attend(lib, P, [new, new], 2, True, 0, 0)
    lib.cast_check_device()
    check(P, q, o, lse, [new, new], 2, True, 0, 0)


@pytest.mark.parametrize("new", [1, 90])
def test_length_past_the_table_is_reported(lib, new):
    P = Pages(lib, [320], 1, 64, 16, False).fill(5)
    P.lens = [400]          # the table has room for 320
    attend(lib, P, [new], 1, False, 0, 0)
    with pytest.raises(lib.CastError) as e:
        lib.cast_check_device()
    assert e.value.status == lib.ERR_INVALID_ARG


@pytest.mark.parametrize("f8", [False, True])
def test_more_new_tokens_than_said_are_left_out(lib, f8):
    P = Pages(lib, [300, 300], 1, 64, 16, f8).fill(5)
    for said in (2, 60):
        n = [said, said + 5]
        cu = torch.tensor([0, n[0], sum(n)], dtype=torch.int32, device="cuda")
        q = randn(gen(2), sum(n), 2, 64).to(torch.bfloat16)
        out = torch.full((sum(n), 128), 5.0, dtype=torch.bfloat16, device="cuda")
        lib.cast_cache_attention(q, P.cache, P.table, P.len_tensor(), cu_new=cu, max_new=said, out=out)
        with pytest.raises(lib.CastError):
            lib.cast_check_device()
        assert (out[n[0] + said:] == 5).all() and not (out[:n[0] + said] == 5).all(1).any()


@pytest.mark.parametrize("bits", [8, 16])
def test_rollout_example(lib, bits):
    """The example's steps (frames, a control token, a routed chunk) against 64 bits."""
    from examples.cache_rollout import Rollout
    r = Rollout(H=2, H_q=4, d=64, grid=(8, 8), page=64, n_pages=16, bits=bits, window=150)
    sections = [32 - 2 * 12, 12, 12]
    keys, values = [], []
    for tokens, causal in ((64, False), (64, False), (1, True), (64, False), (64, False), (1, True)):
        (q, k, v, pos), turned, o = r.step(tokens, causal)
        for x, y in ((q, turned),):
            ref, err = R.rotate(f64(x), pos.cpu().numpy(), 64, sections=sections)
            within(f64(y), ref, err + R.UBF * (np.abs(ref) + err), "queries")
        kk, vv = [], []
        for c, s in ((r.k, r.cache._keep[2]), (r.v, r.cache._keep[3])):
            x = f64(c) if s is None else f64(c) * f64(s)[:, None, :, None]
            (kk if c is r.k else vv).append(x.reshape(-1, 2, 64)[:r.len])
        ref, _ = R.rotate(f64(k), pos.cpu().numpy(), 64, sections=sections)
        half = 2.0 ** -4 if bits == 8 else 2.0 ** -8
        within(kk[0][r.len - tokens:], ref, half * np.abs(ref) + 2.0 ** -7, "keys")
        want, _, eo, _ = R.attention(f64(turned), kk[0], vv[0], tokens, r.len, causal, 150, 64)
        within(f64(o).reshape(tokens, 4, 64), want, eo, "output")
    if bits == 16:
        out = r.routed_chunk(n_frames=3, anchors=(0, 2), K=2)
        assert torch.isfinite(out.float()).all()
    lib.cast_check_device()


def test_binding_refuses_tensors_that_are_not_on_the_gpu(lib):
    k, q = (torch.zeros(2, h, 64, dtype=torch.bfloat16, device="cuda") for h in (1, 2))
    pages = torch.zeros(2, 16, 1, 64, dtype=torch.bfloat16, device="cuda")
    cache, host_cache = lib.kv_cache(pages, pages.clone()), lib.kv_cache(pages.cpu(), pages.cpu())
    table, n = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((1, 2), (1,)))
    n += 2
    cu, pos, turns = torch.tensor([0, 2], dtype=torch.int32), torch.zeros(2, dtype=torch.int32), lib.rotary_table(64)
    calls = [lambda: lib.cast_rotary(k, pos, turns), lambda: lib.cast_rotary(k, pos.cuda(), turns, out=k.cpu())]
    for f, x in ((lambda *a, **kw: lib.cast_cache_append(a[0], a[0], *a[1:], **kw), k), (lib.cast_cache_attention, q)):
        calls += [lambda f=f, x=x, a=a, kw=kw: f(x if a[0] else x.cpu(), *a[1:], **kw) for a, kw in (
            ((0, cache, table, n), {}), ((1, host_cache, table, n), {}), ((1, cache, table.cpu(), n), {}),
            ((1, cache, table, n.cpu()), {}), ((1, cache, table, n), dict(cu_new=cu)))]
    calls += [lambda: lib.cast_cache_append(k, k.cpu(), cache, table, n), lambda: lib.cast_cache_append(k, k, cache, table, n, q=q.cpu()),
              lambda: lib.cast_cache_append(k, k, cache, table, n, q=q, q_out=q.cpu()),
              lambda: lib.cast_cache_append(k, k, cache, table, n, rotary=turns, positions=pos),
              lambda: lib.cast_cache_attention(q, cache, table, n, out=q.cpu()),
              lambda: lib.cast_cache_attention(q, cache, table, n, workspace=torch.empty(1 << 20, dtype=torch.uint8))]
    for call in calls:
        with pytest.raises(ValueError):
            call()


# Work that is dealt out in shares which begin and end inside units, of one query tile and of two, at their first
# key tiles, between units and at their last
CUT = [
    ([20000, 131, 4100, 257], [9, 20, 40, 64], 2, 8, 64, 64, True, 0, 0),
    ([9000] * 7, [5] * 7, 3, 15, 128, 16, True, 4000, 100),
    ([6000, 6100, 6200], [300, 129, 17], 2, 4, 128, 32, False, 0, 0),
    ([0, 12000, 1], [6, 40, 6], 1, 24, 128, 128, True, 0, 0),
    ([1100 + 130 * i for i in range(9)], [70 - 7 * i for i in range(9)], 5, 5, 64, 16, True, 0, 0),
]


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("lens,new,H,Hq,d,page,causal,window,sinks", CUT)
def test_units_cut_anywhere(lib, lens, new, H, Hq, d, page, causal, window, sinks, f8):
    P = Pages(lib, lens, H, d, page, f8, seed=8).fill(9)
    q, o, lse = attend(lib, P, new, Hq, causal, window, sinks)
    lib.cast_check_device()
    check(P, q, o, lse, new, Hq, causal, window, sinks)


def test_append_of_more_heads_than_are_fetched_ahead(lib):
    """Every number of heads from one to more than a CTA takes, into bf16 and 8-bit pages, the same rows as head by head."""
    for f8 in (False, True):
        for H in (1, 2, 3, 4, 5, 13, 25):
            P, one = (Pages(lib, [300], H, 64, 64, f8, seed=1) for _ in range(2))
            k, v = (randn(gen(s), 300, H, 64).to(torch.bfloat16) for s in (1, 2))
            lib.cast_cache_append(k, v, P.cache, P.table, P.len_tensor())
            for h in range(H):
                pages = [t[:, :, h:h + 1].contiguous() for t in (one.k, one.v)]
                scales = [t[:, h:h + 1].contiguous() for t in (one.ks, one.vs)] if f8 else []
                lib.cast_cache_append(k[:, h:h + 1].contiguous(), v[:, h:h + 1].contiguous(), lib.kv_cache(*pages, *scales),
                                      P.table, P.len_tensor())
                used = P.table[0, :5].long()
                for a, b in zip((P.k, P.v), pages):
                    a, b = (t[used].view(torch.uint8 if f8 else torch.int16) for t in (a[:, :, h:h + 1].contiguous(), b))
                    assert torch.equal(a.reshape(5 * 64, -1)[:300], b.reshape(5 * 64, -1)[:300]), (f8, H, h)
                for a, b in zip((P.ks, P.vs), scales):
                    assert torch.equal(a[used, h], b[used, 0])
    lib.cast_check_device()


@pytest.mark.parametrize("f8,H,d", [(True, 8, 128), (True, 16, 64), (True, 18, 64), (False, 8, 64), (False, 10, 64)])
@pytest.mark.parametrize("causal,window,sinks", [(True, 0, 0), (True, 1100, 20)])
def test_many_heads_of_short_rows(lib, f8, H, d, causal, window, sinks):
    """Heads whose rows are short, in sequences from nothing to over a thousand tokens."""
    lens = [(131 * i * i) % 1500 for i in range(16)]
    new = [1 + i % 2 for i in range(16)]
    lens = [max(m, n) for m, n in zip(lens, new)]
    lens[5], new[5], lens[6] = 0, 0, 1500
    P = Pages(lib, lens, H, d, 32, f8, seed=2).fill(5)
    q, o, lse = attend(lib, P, new, 3 * H, causal, window, sinks)
    lib.cast_check_device()
    check(P, q, o, lse, new, 3 * H, causal, window, sinks)
