"""The paged KV cache's entry points on the CPU, at the edges of what they take."""
import ctypes as C
import os
import re
import subprocess
import sys

import pytest
import torch

from tests.test_cache_host import _append, _attend, _batch, _cache, lib  # noqa: F401

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


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


def _calls(lib, on):  # noqa: F811
    """A call of each entry point whose tensors are on the GPUs on("name"); nothing is behind their addresses."""
    def t(name, *shape, dtype=torch.bfloat16):
        return OnGpu(torch.zeros(shape, dtype=dtype), on(name))

    pages = [t("cache", 2, 16, 1, 64), t("cache_v", 2, 16, 1, 64)]
    ints = dict(page_table=t("page_table", 1, 2, dtype=torch.int32), kv_len=t("kv_len", 1, dtype=torch.int32),
                cu_new=t("cu_new", 2, dtype=torch.int32))
    pos, table = t("positions", 2, dtype=torch.int32), lib.rotary_table(64)
    yield lambda: lib.cast_rotary(t("k", 2, 1, 64), pos, table, out=t("out", 2, 1, 64))
    yield lambda: lib.cast_cache_append(t("k", 2, 1, 64), t("v", 2, 1, 64), lib.kv_cache(*pages), rotary=table, positions=pos,
                                        q=t("q", 2, 2, 64), q_out=t("out", 2, 2, 64), **ints)
    yield lambda: lib.cast_cache_attention(t("q", 2, 2, 64), lib.kv_cache(*pages), out=t("out", 2, 128), workspace=t("workspace", 1 << 20),
                                           **ints)


class Launched(Exception):
    pass


@pytest.fixture
def no_launch(lib, monkeypatch):  # noqa: F811
    """A process whose current GPU is 1 and whose calls end where they would enter the library."""
    def enter(*a):
        raise Launched

    for f in ("cast_rotary", "cast_cache_append", "cast_cache_attention"):
        monkeypatch.setattr(lib._lib, f, enter)
    monkeypatch.setattr(lib, "_current_device", lambda: 1, raising=False)
    monkeypatch.setattr(lib, "_raw_stream", lambda device: 0)


def test_tensors_of_the_current_gpu_are_taken(lib, no_launch):  # noqa: F811
    for call in _calls(lib, lambda name: 1):
        with pytest.raises(Launched):
            call()


def test_tensors_of_another_gpu_are_refused(lib, no_launch):  # noqa: F811
    """All tensors on a GPU that is not the current one, or one of them on another than the rest: refused on the host."""
    for call in _calls(lib, lambda name: 0):
        with pytest.raises(ValueError):
            call()
    names = dict(rotary=("k", "positions", "out"), append=("k", "v", "cache", "cache_v", "page_table", "kv_len", "cu_new", "positions", "q", "out"),
                 attention=("q", "cache", "cache_v", "page_table", "kv_len", "cu_new", "out", "workspace"))
    for i, f in enumerate(names):
        for name in names[f]:
            call = list(_calls(lib, lambda n: 0 if n == name else 1))[i]
            with pytest.raises(ValueError):
                call()


def test_a_stream_of_another_gpu_is_refused(lib, no_launch):  # noqa: F811
    class Stream:
        cuda_stream = 0

        def __init__(self, device):
            self.device_index = device

    x, pos, table = OnGpu(torch.zeros(2, 1, 64), 1), OnGpu(torch.zeros(2, dtype=torch.int32), 1), lib.rotary_table(64)
    with pytest.raises(Launched):
        lib.cast_rotary(x, pos, table, out=x, stream=Stream(1))
    with pytest.raises(ValueError):
        lib.cast_rotary(x, pos, table, out=x, stream=Stream(0))


WORKSPACE = """
import ctypes as C
from paper_2609_34144_gb300 import native as lib
from tests.test_cache_host import _attend, _batch, _cache
for kw, b, c in (({"H_q": 2 * 129}, {}, {}), ({"H_q": 1 << 20}, {}, {}), ({}, {"B": 0}, {}), ({"H_q": 64}, {"B": 0}, {}), ({"H_q": 64}, {"B": -1}, {}),
                 ({"H_q": 3}, {}, {}), ({"H_q": 0}, {}, {}), ({}, {}, {"H": 0}), ({}, {}, {"d": 96}), ({}, {"T": -4}, {}), ({}, {"max_new": -1}, {}),
                 ({}, {"max_pages": -1}, {}), ({}, {}, {"page_size": 0})):
    a = _attend(lib, cache=_cache(lib, **c), batch=_batch(lib, **b), **kw)
    print(lib.library().cast_cache_attention_workspace_size(C.byref(a)))
print(lib.library().cast_cache_attention_workspace_size(None))
"""


def test_workspace_of_arguments_that_the_call_refuses_is_zero(lib):  # noqa: F811
    """In a process of its own: a division by zero would end it."""
    r = subprocess.run([sys.executable, "-c", WORKSPACE], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    assert r.stdout.split() == ["0"] * 14


def test_binding_refuses_heads_and_batches_that_the_library_refuses(lib, monkeypatch):  # noqa: F811
    """More than 128 query heads a KV head, and no sequences: an error, as from the library itself."""
    monkeypatch.setattr(lib, "_current_device", lambda: 0)
    monkeypatch.setattr(lib, "_raw_stream", lambda device: 0)
    pages = [OnGpu(torch.zeros(2, 16, 1, 64, dtype=torch.bfloat16)) for _ in range(2)]
    for heads, B, status in ((129, 1, lib.ERR_UNSUPPORTED), (64, 0, lib.ERR_INVALID_ARG)):
        q, out = (OnGpu(torch.zeros(2, heads * 64, dtype=torch.bfloat16).view(s)) for s in ((2, heads, 64), (2, heads * 64)))
        ints = [OnGpu(torch.zeros(s, dtype=torch.int32)) for s in ((B, 2), (B,))]
        with pytest.raises(lib.CastError) as e:
            lib.cast_cache_attention(q, lib.kv_cache(*pages), *ints, out=out)
        assert e.value.status == status


@pytest.mark.parametrize("lse", [0xa00001, 0xa00002, 0xa00003])
def test_lse_has_to_be_aligned(lib, lse):  # noqa: F811
    # (without a workspace, which a call that gets past the check would miss)
    a = _attend(lib, batch=_batch(lib, max_pages=1000, page_table_stride=1000), lse=lse)
    assert lib.library().cast_cache_attention(C.byref(a), None, 0, None) == lib.ERR_INVALID_ARG
    assert b"lse" in lib.library().cast_last_error_detail()


def _tiles_kernel():
    """The text of k_cache_tiles, without comments."""
    text = open(os.path.join(ROOT, "paper_2609_34144_gb300", "csrc", "cache_tiles.cu")).read()
    text = re.sub(r"//[^\n]*", "", text)
    start = text.index("k_cache_tiles(const __grid_constant__")
    return text[start:text.index("k_tiles_merge", start)]


def test_every_share_of_tiles_has_a_cut_before_the_first_wait():
    """The joining follows the cuts in the workspace also when a CTA gave up: each has to be written, or marked as
    none, before anything is waited for (whole units first: marked; else found with the share)."""
    text = _tiles_kernel()
    start = text[:text.index("mbar_wait")]
    assert "a.cuts[blockIdx.x].c0 = -1" in start
    assert re.search(r"unit_at\(a, d, at, stop, lane, d.rounds > 0 \? nullptr : a.cuts \+ blockIdx.x\)", start)


def test_copies_of_a_cta_that_gave_up_are_awaited():
    """Warps 0 and 2 begin the copies into shared memory; where the CTA gave up they wait (with a limit) for those
    that are on their way, and for the queries, before it leaves."""
    text = _tiles_kernel()
    assert text.count("fetch_pages<") == 1 and text.count("tma_load_3d(") == 1
    leave = text[text.index("tma_load_3d("):text.index("setmaxnreg_inc")]
    leave = leave[leave.rindex("another()"):]
    gave_up = leave[leave.index("aborted(bars)"):leave.index("tmem_dealloc")]
    assert re.search(r"for \(int j = max\(issued - .*mbar_wait\(&full\[.*lim\)", gave_up, re.S)
    assert re.search(r"mbar_wait\(F8 \? &bars->q_raw : &bars->q_full, 0, lim\)", gave_up)


@pytest.mark.parametrize("dtype,d,H,two", [("f8", 64, 8, True), ("f8", 64, 10, True), ("f8", 128, 4, True), ("bf16", 64, 4, True), ("bf16", 64, 8, True),
                                           ("f8", 64, 6, False), ("bf16", 128, 8, False)])
def test_two_heads_side_by_side_where_rows_are_short(lib, dtype, d, H, two):  # noqa: F811
    """Which calls take units of two KV heads shows in the workspace: twice the parts of an odd number of heads."""
    def need(heads):
        cache = _cache(lib, dtype=lib.F8E4M3 if dtype == "f8" else lib.BF16, H=heads, d=d, row_stride=heads * d)
        batch = _batch(lib, B=64, T=64, max_new=1, max_pages=1000, page_table_stride=1000)
        return lib.library().cast_cache_attention_workspace_size(C.byref(_attend(lib, cache=cache, batch=batch, H_q=heads)))

    assert need(H) == (2 if two else 1) * need(H + 1)
