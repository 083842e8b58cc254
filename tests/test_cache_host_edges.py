"""The paged KV cache's entry points on the CPU, at the edges of what they take."""
import ctypes as C

import pytest
import torch

from tests.test_cache_host import _append, _attend, _batch, lib  # noqa: F401


class OnGpu:
    """What the binding asks a tensor for, of one on GPU `device` that is not there."""

    is_cuda = True

    def __init__(self, t, device=0):
        self.t, self.device_index = t, device

    def get_device(self):
        return self.device_index

    def __getattr__(self, name):
        return getattr(self.t, name)


def test_table_of_all_sequences(lib):  # noqa: F811
    """One table that several sequences share has a row stride of 0; rows that overlap otherwise are refused."""
    n = OnGpu(torch.zeros(3, dtype=torch.int32))
    table = torch.arange(40, dtype=torch.int32)

    def stride(t):
        return lib._batch(OnGpu(t), n, None, 3, None)[1]

    assert stride(table[None, :8].expand(3, -1)) == 0
    assert stride(table.as_strided((3, 8), (12, 1))) == 12
    for t in (table.as_strided((3, 8), (7, 1)), table.as_strided((3, 8), (1, 1)), table.as_strided((3, 8), (8, 2))):
        with pytest.raises(ValueError):
            stride(t)
    one = OnGpu(torch.zeros(1, dtype=torch.int32))
    assert lib._batch(OnGpu(table[None, :8].expand(1, -1)), one, None, 3, None)[1] == 8
    assert lib._batch(OnGpu(table.as_strided((1, 8), (0, 1))), one, None, 3, None)[1] == 8


@pytest.mark.parametrize("stride,status", [(0, 0), (8, 0), (7, 1), (1, 1), (-1, 1)])
def test_table_stride(lib, stride, status):  # noqa: F811
    b = _batch(lib, T=0, max_new=0, page_table_stride=stride)   # nothing to do: only the checks
    assert lib.library().cast_cache_append(C.byref(_append(lib, batch=b)), None) == status
    assert lib.library().cast_cache_attention(C.byref(_attend(lib, batch=b)), None, 0, None) == status
