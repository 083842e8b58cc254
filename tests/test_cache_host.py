"""The paged KV cache's entry points on the CPU: what they refuse before any CUDA call, and the rotary table."""
import ctypes as C
import math
import os
import shutil
import subprocess

import numpy as np
import pytest

from tests import cache_ref as R

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    from paper_2609_34144_gb300 import native
    return native


@pytest.mark.parametrize("rot,kw", [
    (64, {}),
    (128, dict(sections=[16, 24, 24])),
    (32, dict(scaling=("linear", 4.0))),
    (48, dict(scaling=("stretch", 2.0))),
    (64, dict(base=500000.0, scaling=("parts", 8.0, 4096))),
])
def test_table_holds_the_frequencies(lib, rot, kw):
    t = lib.rotary_table(rot, **kw)
    f, axis, amp = R.frequencies(rot, **kw)
    got = np.array([t.turn[i] for i in range(rot // 2)], dtype=np.float64) / 2.0 ** 64 * 2 * math.pi
    # a power and a few products in 64 bits
    assert np.all(np.abs(got - f) <= 1e-14 * f + 2.0 ** -60)
    assert [t.axis[i] for i in range(rot // 2)] == list(axis)
    assert abs(t.amplitude - amp) <= 2.0 ** -23


@pytest.mark.parametrize("rot,kw,status", [
    (0, {}, 1), (7, {}, 1), (24, {}, 2), (272, {}, 2),
    (64, dict(base=1.0), 1),
    (64, dict(sections=[16, 15]), 1),
    (64, dict(sections=[32, 0]), 1),
    (64, dict(scaling=("linear", 0.5)), 1),
    (64, dict(scaling=("parts", 2.0)), 1),
    (64, dict(sections=[31, 1], scaling=("stretch", 2.0)), 1),
])
def test_table_refusals(lib, rot, kw, status):
    with pytest.raises(lib.CastError) as e:
        lib.rotary_table(rot, **kw)
    assert e.value.status == status


def _fake(addr=0x10000):
    return C.c_void_p(addr)


def _rotary(lib, **kw):
    table = lib.rotary_table(64)
    a = lib.RotaryArgs(0x10000, 0x20000, 256, 256, 4, 2, 128, lib.BF16, 0x30000, C.pointer(table), 0)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("bad,status", [
    ({"x": None}, 1), ({"x": 0x10008}, 1), ({"out": None}, 1), ({"positions": None}, 1), ({"positions": 0x30002}, 1),
    ({"x_row_stride": 248}, 1), ({"out_row_stride": 260}, 1), ({"dtype": 2}, 1), ({"T": -1}, 1), ({"H": 0}, 1),
    ({"d": 48}, 1),                      # fewer channels than the table rotates
    ({"d": 72}, 2), ({"d": 512}, 2), ({"table": None}, 1),
])
def test_rotary_refusals(lib, bad, status):
    assert lib.library().cast_rotary(C.byref(_rotary(lib, **bad)), None) == status
    assert lib.library().cast_last_error_detail() != b""


def test_rotary_needs_a_table_that_was_made(lib):
    t = lib.RotaryTable()
    assert lib.library().cast_rotary(C.byref(_rotary(lib, table=C.pointer(t))), None) == 1
    assert lib.library().cast_rotary(C.byref(_rotary(lib, T=0)), None) == 0


def _cache(lib, **kw):
    c = lib.KvCache(lib.F8E4M3, 10, 16, 2, 64, 0x100000, 0x200000, 128, 0x300000, 0x400000)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _batch(lib, **kw):
    b = lib.CacheBatch(0x500000, 8, 8, 0x600000, None, 2, 6, 3)
    for k, v in kw.items():
        setattr(b, k, v)
    return b


CACHE_BAD = [
    ({"dtype": 0}, 1), ({"n_pages": 0}, 1), ({"page_size": 24}, 2), ({"page_size": 256}, 2), ({"H": 0}, 1), ({"d": 96}, 2),
    ({"k": None}, 1), ({"v": 0x200004}, 1), ({"row_stride": 120}, 1), ({"row_stride": 136}, 1), ({"k_scale": None}, 1),
    ({"v_scale": 0x400002}, 1),
]
BATCH_BAD = [
    ({"page_table": None}, 1), ({"kv_len": None}, 1), ({"page_table_stride": 7}, 1), ({"B": 0}, 1), ({"T": -1}, 1),
    ({"T": 7}, 1),                       # not a multiple of B without cu_new
    ({"max_new": 2}, 1),                 # T / B tokens each
    ({"max_pages": -1}, 1), ({"cu_new": 0x700002}, 1), ({"max_new": 0, "cu_new": 0x700000}, 1),
]


def _append(lib, cache=None, batch=None, **kw):
    table = lib.rotary_table(64)
    a = lib.AppendArgs(cache or _cache(lib), batch or _batch(lib), 0x800000, 0x900000, 128, 128, C.pointer(table), None,
                       0xa00000, 0xb00000, 256, 256, 4)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _attend(lib, cache=None, batch=None, **kw):
    a = lib.CacheAttnArgs(cache or _cache(lib), batch or _batch(lib), 0x800000, 256, 4, 1, 0, 0, 0.0, 0x900000, lib.BF16, None)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("which,bad,status", [("cache", b, s) for b, s in CACHE_BAD] + [("batch", b, s) for b, s in BATCH_BAD])
def test_cache_and_batch_refusals(lib, which, bad, status):
    kw = {which: (_cache if which == "cache" else _batch)(lib, **bad)}
    assert lib.library().cast_cache_append(C.byref(_append(lib, **kw)), None) == status
    assert lib.library().cast_last_error_detail() != b""
    assert lib.library().cast_cache_attention(C.byref(_attend(lib, **kw)), _fake(), 1 << 40, None) == status


@pytest.mark.parametrize("bad,status", [
    ({"k": None}, 1), ({"v": 0x900008}, 1), ({"k_row_stride": 120}, 1), ({"v_row_stride": 132}, 1),
    ({"q_out": None}, 1), ({"q": 0xa00004}, 1), ({"q_row_stride": 248}, 1), ({"H_q": 0}, 1), ({"positions": 0x700001}, 1),
    ({"rotary": None}, 1),               # queries without a table
])
def test_append_refusals(lib, bad, status):
    assert lib.library().cast_cache_append(C.byref(_append(lib, **bad)), None) == status
    assert lib.library().cast_last_error_detail() != b""


def test_append_axes_need_positions(lib):
    t = lib.rotary_table(64, sections=[16, 16])
    assert lib.library().cast_cache_append(C.byref(_append(lib, rotary=C.pointer(t))), None) == 1
    wide = lib.rotary_table(128)         # more channels than the heads have
    assert lib.library().cast_cache_append(C.byref(_append(lib, rotary=C.pointer(wide))), None) == 1


@pytest.mark.parametrize("bad,status", [
    ({"q": None}, 1), ({"q": 0x800008}, 1), ({"o": None}, 1), ({"q_row_stride": 200}, 1), ({"H_q": 3}, 1), ({"H_q": 0}, 1),
    ({"H_q": 2 * 129}, 2), ({"window": -1}, 1), ({"sinks": -1}, 1), ({"scale": float("nan")}, 1), ({"o_dtype": 2}, 1),
])
def test_attention_refusals(lib, bad, status):
    assert lib.library().cast_cache_attention(C.byref(_attend(lib, **bad)), _fake(), 1 << 40, None) == status
    assert lib.library().cast_last_error_detail() != b""


def test_attention_workspace_is_checked(lib):
    so = lib.library()
    a = _attend(lib, batch=_batch(lib, max_pages=1000, page_table_stride=1000))
    need = so.cast_cache_attention_workspace_size(C.byref(a))
    assert need > 0
    assert so.cast_cache_attention(C.byref(a), _fake(), need - 1, None) == 1
    assert so.cast_cache_attention(C.byref(a), None, need, None) == 1
    assert so.cast_cache_attention(C.byref(a), _fake(0x10010), need, None) == 1


def test_nothing_to_do_is_ok(lib):
    b = _batch(lib, T=0, max_new=0)
    assert lib.library().cast_cache_append(C.byref(_append(lib, batch=b, k=None, v=None, q=None)), None) == 0
    assert lib.library().cast_cache_attention(C.byref(_attend(lib, batch=b, q=None, o=None)), None, 0, None) == 0


def test_binding_refuses_tensors_of_another_form(lib):
    import torch
    t = lib.rotary_table(64)
    pos = torch.zeros(3, dtype=torch.int64)
    with pytest.raises(ValueError):
        lib.cast_rotary(torch.zeros(3, 2, 64), pos, t)
    with pytest.raises(ValueError):
        lib.cast_rotary(torch.zeros(3, 64, 2).transpose(1, 2), pos.int(), t)
    with pytest.raises(TypeError):
        lib.kv_cache(torch.zeros(2, 16, 1, 64), torch.zeros(2, 16, 1, 64))
    with pytest.raises(ValueError):
        lib.kv_cache(*(torch.zeros(2, 16, 1, 64, dtype=torch.uint8),) * 2)
    c = lib.kv_cache(*(torch.zeros(2, 16, 1, 64, dtype=torch.bfloat16),) * 2)
    x = torch.zeros(2, 1, 64, dtype=torch.bfloat16)
    table = torch.zeros(2, 1, dtype=torch.int32)
    with pytest.raises(ValueError):
        lib.cast_cache_append(x, x, c, table, torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError):
        lib.cast_cache_append(x, x[:1], c, table, torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        lib.cast_cache_attention(x.float(), c, table, torch.zeros(2, dtype=torch.int32))


def test_struct_layouts_match_the_header(lib, tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("no gcc")
    structs = {"cast_rotary_params": lib.RotaryParams, "cast_rotary_table": lib.RotaryTable, "cast_rotary_args": lib.RotaryArgs,
               "cast_kv_cache": lib.KvCache, "cast_cache_batch": lib.CacheBatch, "cast_append_args": lib.AppendArgs,
               "cast_cache_attn_args": lib.CacheAttnArgs}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "cast.h"', "int main(void) {"]
    for cname, py in structs.items():
        lines.append(f'printf("{cname} sizeof %zu\\n", sizeof({cname}));')
        lines += [f'printf("{cname} {f} %zu\\n", offsetof({cname}, {f}));' for f, _ in py._fields_]
    (tmp_path / "layout.c").write_text("\n".join(lines + ["return 0;", "}"]))
    subprocess.run(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), str(tmp_path / "layout.c"), "-o", str(tmp_path / "layout")],
                   check=True, capture_output=True)
    for line in subprocess.run([str(tmp_path / "layout")], check=True, capture_output=True, text=True).stdout.splitlines():
        cname, f, val = line.split()
        py = structs[cname]
        assert (C.sizeof(py) if f == "sizeof" else getattr(py, f).offset) == int(val), (cname, f)


def test_packed_arguments_are_the_structs(lib):
    """The bytes that the binding packs for a call lie as the ctypes classes (and so the header) do."""
    import torch
    k = torch.zeros(4, 16, 2, 64, dtype=torch.bfloat16)
    cache = lib.kv_cache(k, k)
    batch = (11, 12, 13, 14, 15, 16, 17, 18)
    assert lib._pack_rotary(1, 2, 3, 4, 5, 6, 7, 1, 9, 0, 1) == bytes(lib.RotaryArgs(1, 2, 3, 4, 5, 6, 7, 1, 9, None, 1))
    want = lib.AppendArgs(cache, lib.CacheBatch(*batch), 21, 22, 23, 24, None, 25, 26, 27, 28, 29, 30)
    assert lib._pack_append(cache.packed, *batch, 21, 22, 23, 24, 0, 25, 26, 27, 28, 29, 30) == bytes(want)
    want = lib.CacheAttnArgs(cache, lib.CacheBatch(*batch), 21, 22, 23, 1, 25, 26, 0.5, 28, 1, 30)
    assert lib._pack_attention(cache.packed, *batch, 21, 22, 23, 1, 25, 26, 0.5, 28, 1, 30) == bytes(want)
