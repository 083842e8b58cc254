"""4-bit pages on the GPU at the ends of what scales and queries may be, and units that a CTA takes whole."""
import numpy as np
import pytest
import torch

from tests.test_gpu_cache4 import Pages4, check_attention, gen, i32, randn

pytestmark = pytest.mark.gpu

# rows of a KV head: few (one and two eights), tiles of one query tile and of two
FORMS = [(1, 4, 128), (3, 8, 64), (3, 12, 64), (40, 4, 128), (300, 2, 64), (300, 4, 128)]
MASKS = [dict(), dict(window=200, sinks=9), dict(causal=False)]


@pytest.mark.parametrize("new,H_q,d", FORMS)
@pytest.mark.parametrize("kw", MASKS, ids=["causal", "window", "all"])
@pytest.mark.parametrize("scale,size", [(1e-8, 1e-34), (1e-30, 1e-20), (1e-38, 1e-6), (1e-38, 0.0)])
def test_a_row_whose_logits_are_next_to_nothing_is_the_mean(lib, new, H_q, d, kw, scale, size):
    """The scale times the row's power of two is below what f32 holds: hidden keys stay hidden."""
    c = Pages4(lib, [700], 2, d, 32, seed=8)
    held = c.fill(seed=9)
    q = (randn(gen(new), new, H_q, d) * size).to(torch.bfloat16)
    o, lse = lib.cast_cache_attention(q, c.cache, c.table, c.kv_len, scale=scale, want_lse=True, out_dtype=torch.float32, **kw)
    check_attention(lib, c, held, q, [new], o, lse, scale=scale, **kw)


@pytest.mark.parametrize("new,H_q,d", FORMS)
@pytest.mark.parametrize("scale,size", [(1e33, 1e-34), (1e35, 1e-36), (2e38, 1e-39), (1e-38, 1e38)])
def test_queries_at_the_ends_of_bf16(lib, new, H_q, d, scale, size):
    """Rows of subnormal numbers and of the largest, with a scale that makes ordinary logits of them."""
    c = Pages4(lib, [700], 2, d, 32, seed=8)
    held = c.fill(seed=9)
    q = (randn(gen(new), new, H_q, d).clamp(-3, 3).double() * size).to(torch.bfloat16)
    o, lse = lib.cast_cache_attention(q, c.cache, c.table, c.kv_len, scale=scale, want_lse=True, out_dtype=torch.float32)
    check_attention(lib, c, held, q, [new], o, lse, scale=scale)


@pytest.mark.parametrize("new,H_q,d", FORMS)
@pytest.mark.parametrize("kw", MASKS, ids=["causal", "window", "all"])
def test_keys_of_zeros_under_the_largest_queries_and_scales(lib, new, H_q, d, kw):
    """Every logit is 0 whatever multiplies it: the mean of the values."""
    c = Pages4(lib, [700], 2, d, 32, seed=8)
    (k, v), = c.fill(seed=9)
    c.ks.zero_()
    q = (randn(gen(new), new, H_q, d).clamp(-3, 3).double() * 1e38).to(torch.bfloat16)
    for scale in (1e5, 3e38):
        o, lse = lib.cast_cache_attention(q, c.cache, c.table, c.kv_len, scale=scale, want_lse=True, out_dtype=torch.float32, **kw)
        check_attention(lib, c, [(np.zeros_like(k), v)], q, [new], o, lse, scale=scale, **kw)


WHOLE = [
    # sequences, lengths up to, new, H, H_q, d, page, window, sinks
    (128, 2000, 1, 1, 4, 128, 16, 0, 0),       # 128 units of up to 125 blocks of 16
    (64, 2040, 2, 2, 14, 64, 64, 0, 0),        # ... of two eights of rows
    (48, 1900, 3, 3, 9, 128, 128, 0, 0),
    (384, 2900, 1, 1, 8, 64, 16, 0, 0),        # 384 of up to 182
    (97, 2990, 3, 4, 20, 128, 32, 0, 0),
    (129, 6000, 2, 1, 5, 128, 16, 1700, 40),   # bounded by the window instead of the table
    (200, 7000, 5, 2, 6, 64, 64, 2500, 100),
]


@pytest.mark.parametrize("B,most,new,H,H_q,d,page,window,sinks", WHOLE)
def test_units_that_ctas_take_whole(lib, B, most, new, H, H_q, d, page, window, sinks):
    """Many units of more than a thousand tokens: no workspace, which an empty one shows.  Ragged, with sequences of no
    tokens and of fewer than their new ones."""
    r = np.random.default_rng(B)
    lens = r.integers(1, 300, B)
    lens[::max(B // 12, 1)] = r.integers(1000, most, len(lens[::max(B // 12, 1)]))
    lens[1], lens[B // 2], lens[-1] = 0, new - 1, most
    n = [int(x) for x in r.integers(1, new + 1, B)]
    n[1], n[B // 2], n[-1] = new, new, new
    c = Pages4(lib, [int(x) for x in lens], H, d, page, seed=2)
    held = c.fill(seed=5)
    q = (1.5 * randn(gen(1), sum(n), H_q, d)).to(torch.bfloat16)
    kw = dict(window=window, sinks=sinks)
    o, lse = lib.cast_cache_attention(q, c.cache, c.table, c.kv_len, cu_new=i32(*np.concatenate([[0], np.cumsum(n)])), max_new=new,
                                      want_lse=True, workspace=torch.empty(0, dtype=torch.uint8, device="cuda"), **kw)
    lib.cast_check_device()
    check_attention(lib, c, held, q, n, o, lse, **kw)
