"""4-bit pages on the GPU at the ends of what scales and queries may be."""
import numpy as np
import pytest
import torch

from tests.test_gpu_cache4 import Pages4, check_attention, gen, randn

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
