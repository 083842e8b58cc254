"""The paged KV cache at the edges of its definitions, against 64 bits."""
import numpy as np
import pytest
import torch

from tests import cache_ref as R
from tests.test_gpu_cache import Pages, attend, check, f64, gen, randn, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("new,Hq,causal,window", [(40, 2, True, 0), (300, 2, True, 0), (300, 1, True, 70), (90, 3, False, 100)])
def test_zero_queries_see_no_hidden_zero_keys(lib, new, Hq, causal, window, page):
    """Padding at a prompt's end: queries of zeros, pages of zero keys at the scales that the append gives them (and
    at small ones).  A row of zeros is the mean of the values that it sees."""
    L = new + 400
    for e in (-120, -30):
        P = Pages(lib, [L], 1, 64, page, True).fill(9)
        for i in range((L - new) // page, -(-L // page)):
            p = int(P.table[0, i])
            P.k.view(torch.uint8)[p].zero_()
            P.ks[p] = 2.0 ** e
        q = randn(gen(5), new, Hq, 64).to(torch.bfloat16)
        q[new // 3:] = 0
        o, lse = lib.cast_cache_attention(q, P.cache, P.table, P.len_tensor(), causal=causal, window=window, want_lse=True,
                                          out_dtype=torch.float32)
        lib.cast_check_device()
        check(P, q, o, lse, [new], Hq, causal, window, 0)


# A page's place in its sequence (which rows see it follows from the lengths), and what it is larger by
HIDDEN = [
    # L, new, H_q, page, window, sinks, {page of the sequence: log2 of its scale}
    (300, 300, 2, 16, 0, 0, {i: 6 * i for i in range(19)}),                 # a prompt whose pages grow
    (300, 300, 1, 16, 0, 0, {i: 40 * (i % 2) for i in range(19)}),
    (132, 40, 2, 128, 0, 0, {1: 40}),                                        # the last four rows' page
    (1000, 200, 2, 16, 50, 0, {47: 40}),                                     # positions 752 .. 767, of the first rows' windows
    (1000, 200, 1, 32, 50, 40, {24: 60, 0: 0, 1: -20}),
    (5000, 150, 2, 64, 2000, 0, {44: 50, 45: 30}),                           # cut into parts
    (600, 8, 2, 16, 181, 0, {25: 40}),                                       # drafts: positions 400 .. 415, seen from 412 on by the first row
    (516, 8, 2, 16, 0, 0, {32: 40}),                                         # drafts: the last four rows' page
    (5016, 8, 2, 16, 3989, 0, {63: 40}),                                     # drafts, cut into parts: 1008 .. 1023, seen from 1020 on
    (5016, 8, 4, 32, 3989, 0, {31: 50, 32: 20}),                             # two products a head
]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("L,new,Hq,page,window,sinks,scales", HIDDEN)
def test_a_hidden_page_does_not_set_the_scale(lib, L, new, Hq, page, window, sinks, scales, d):
    """Values of pages that a row does not see cost its own no bits, however large they are."""
    P = Pages(lib, [L], 1, d, page, True).fill(3)
    for i, e in scales.items():
        P.vs[int(P.table[0, i])] = 2.0 ** e
    q, o, lse = attend(lib, P, [new], Hq, True, window, sinks, dtype=torch.float32)
    lib.cast_check_device()
    check(P, q, o, lse, [new], Hq, True, window, sinks)


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("new", [1, 40])
def test_sequences_that_share_one_table(lib, f8, new):
    """A table expanded over the sequences: the same bits as with a copy for each; and tokens stored through it."""
    P = Pages(lib, [900], 2, 64, 16, f8, seed=4).fill(5)
    lens = torch.tensor([900, 333, new, 850], dtype=torch.int32, device="cuda")
    q = randn(gen(1), 4 * new, 4, 64).to(torch.bfloat16)
    shared = P.table.expand(4, -1)
    assert shared.stride(0) == 0
    got = lib.cast_cache_attention(q, P.cache, shared, lens)
    assert torch.equal(got, lib.cast_cache_attention(q, P.cache, shared.contiguous(), lens))
    # each sequence ends a page of its own: tokens 16 b .. 16 b + 15
    k = randn(gen(2), 64, 2, 64).to(torch.bfloat16)
    ends = torch.tensor([16, 32, 48, 64], dtype=torch.int32, device="cuda")
    lib.cast_cache_append(k, k, P.cache, shared, ends)
    one = Pages(lib, [900], 2, 64, 16, f8, seed=4).fill(5)
    lib.cast_cache_append(k, k, one.cache, one.table, ends[3:])
    lib.cast_check_device()
    bits = torch.uint8 if f8 else torch.int16
    assert torch.equal(P.k.view(bits), one.k.view(bits)) and torch.equal(P.v.view(bits), one.v.view(bits))


def test_work_beyond_32_bits(lib):
    """65,536 sequences of two rows of 128 query heads over 2^20 positions (one page, again and again): the tiles that
    the call has to be dealt out by are more than 2^31."""
    B, G, d, L = 65536, 128, 64, 1 << 20
    g = gen(3)
    k, v = (randn(g, 1, 128, 1, d).to(torch.bfloat16) for _ in range(2))
    table = torch.zeros((B, L // 128), dtype=torch.int32, device="cuda")
    q = torch.randn((2 * B, G, d), generator=g, device="cuda", dtype=torch.bfloat16)
    out = torch.full((2 * B, G * d), float("nan"), dtype=torch.bfloat16, device="cuda")
    lib.cast_cache_attention(q, lib.kv_cache(k, v), table, torch.full((B,), L, dtype=torch.int32, device="cuda"), causal=False, out=out)
    lib.cast_check_device()
    rows = torch.arange(0, 2 * B, 997, device="cuda")
    # every position of the page has the same weight L / 128 times over
    ref, _, eo, _ = R.attention(f64(q[rows]), f64(k[0]), f64(v[0]), len(rows), 128, causal=False)
    # and the sums have L terms: cache_ref's bound has 128 U32 in their place
    part = R.attention(f64(q[rows]), f64(k[0]), np.abs(f64(v[0])), len(rows), 128, causal=False)[0]
    within(f64(out[rows]).reshape(-1, G, d), ref, eo + L * R.U32 * part, "o")
    assert not torch.isnan(out.view(torch.int16).view(B, -1)[:, ::1000].view(torch.bfloat16)).any()


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("start,new,said", [
    ([0, 10], [7, 7], 2),                # ends inside the page that it begins in
    ([60, 64], [9, 200], 5),             # ends inside the next page; would fill several
    ([3, 130], [64, 70], 64),            # one sequence at the bound
    ([-2, -4], [5, 4], 5),               # places before the sequence's beginning
    ([-3, -1], [40, 9], 6),              # and both
])
def test_append_leaves_out_what_was_not_said(lib, start, new, said, f8):
    """Tokens past max_new and places below zero: pages, scales and rotated queries are those of a call without them."""
    H, d, Hq, page = 2, 64, 4, 64
    lens = [max(s + n, 1) for s, n in zip(start, new)]
    P, want = (Pages(lib, lens, H, d, page, f8, seed=1).fill(2) for _ in range(2))
    g = gen(7)
    T = sum(new)
    k, v = ((3 * randn(g, T, H, d)).to(torch.bfloat16) for _ in range(2))
    q = randn(g, T, Hq, d).to(torch.bfloat16)
    turns = lib.rotary_table(d)
    got_q = torch.full_like(q, 5.0)
    want_q = got_q.clone()
    cu = torch.tensor([0, new[0], T], dtype=torch.int32, device="cuda")
    n = torch.tensor([s + c for s, c in zip(start, new)], dtype=torch.int32, device="cuda")
    lib.cast_cache_append(k, v, P.cache, P.table, n, cu_new=cu, max_new=said, rotary=turns, q=q, q_out=got_q)
    if max(new) > said:
        with pytest.raises(lib.CastError) as e:
            lib.cast_check_device()
        assert e.value.status == lib.ERR_INVALID_ARG
    lib.cast_check_device()
    at = 0
    for b in range(2):
        lo, hi = at + max(0, -start[b]), at + min(new[b], said)
        if lo < hi:
            rows = slice(lo, hi)
            end = torch.tensor([start[b] + hi - at], dtype=torch.int32, device="cuda")
            want_q[rows] = lib.cast_cache_append(k[rows], v[rows], want.cache, want.table[b:b + 1], end, rotary=turns, q=q[rows])
        at += new[b]
    lib.cast_check_device()
    bits = torch.uint8 if f8 else torch.int16
    for x, y in ((P.k, want.k), (P.v, want.v)):
        assert torch.equal(x.view(bits), y.view(bits))
    if f8:
        # (NaN where no page was)
        assert all(torch.equal(x.view(torch.int32), y.view(torch.int32)) for x, y in ((P.ks, want.ks), (P.vs, want.vs)))
    assert torch.equal(got_q.view(torch.int16), want_q.view(torch.int16))


@pytest.mark.parametrize("which", ["rotary", "append", "rows", "tiles", "lse"])
def test_outputs_on_another_stream_leave_memory_in_use_alone(lib, which):
    """A tensor that the current stream still reads was given back before a call on another stream."""
    P = Pages(lib, [3000], 2, 64, 16, False, seed=4).fill(5)
    new = 100 if which == "tiles" else 4
    T = 2048 if which in ("rotary", "append") else new
    turns, n = lib.rotary_table(64), P.len_tensor()
    q = randn(gen(1), T, 4, 64).to(torch.bfloat16)
    k = randn(gen(2), T, 2, 64).to(torch.bfloat16)
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    s = torch.cuda.Stream()

    def call():
        if which == "rotary":
            return lib.cast_rotary(q, pos, turns, stream=s)
        if which == "append":
            return lib.cast_cache_append(k, k, P.cache, P.table, n, rotary=turns, q=q, stream=s)
        out = lib.cast_cache_attention(q, P.cache, P.table, n, want_lse=True, stream=s)
        return out[which == "lse"]

    want = call()
    torch.cuda.synchronize()
    for _ in range(3):
        held = torch.full_like(want, 7.0)
        kept = torch.empty_like(want)
        torch.cuda.synchronize()
        torch.cuda._sleep(20_000_000)
        kept.copy_(held)
        del held
        got = call()
        torch.cuda.synchronize()
        assert (kept == 7).all() and torch.equal(got, want)
    lib.cast_check_device()


@pytest.mark.parametrize("f8", [False, True])
def test_a_workspace_of_earlier_calls(lib, f8):
    """Calls of other shapes leave their cuts and parts behind; whole units, shares of them and single units follow."""
    ws = torch.full((1 << 26,), 0x7f, dtype=torch.uint8, device="cuda")
    for L, new, H in ((3000, 900, 4), (2000, 700, 40), (4000, 130, 1), (2500, 128, 152), (2500, 128, 153), (3000, 900, 4)):
        P = Pages(lib, [L], H, 64, 64, f8).fill(3)
        q, o, lse = attend(lib, P, [new], H, False, 0, 0, workspace=ws)
        lib.cast_check_device()
        check(P, q, o, lse, [new], H, False, 0, 0)


@pytest.mark.parametrize("f8,H,d", [(True, 8, 64), (True, 10, 64), (True, 4, 128), (True, 6, 128), (False, 4, 64), (False, 6, 64)])
@pytest.mark.parametrize("causal,window,sinks", [(True, 0, 0), (False, 1100, 20)])
def test_heads_whose_rows_are_short_side_by_side(lib, f8, H, d, causal, window, sinks):
    """Rows of 512 to 1024 bytes, in sequences from nothing to over a thousand tokens."""
    lens = [max((131 * i * i) % 1500, 1 + i % 3) for i in range(34)]
    new = [1 + i % 3 for i in range(34)]
    lens[5], new[5], lens[6] = 0, 0, 1500
    P = Pages(lib, lens, H, d, 32, f8, seed=2).fill(5)
    q, o, lse = attend(lib, P, new, 2 * H, causal, window, sinks)
    lib.cast_check_device()
    check(P, q, o, lse, new, 2 * H, causal, window, sinks)
