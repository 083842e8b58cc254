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
