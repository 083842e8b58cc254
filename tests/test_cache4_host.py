"""4-bit pages and the reading back on the CPU: what the entry points and the binding refuse before any CUDA call, the
arguments' layout, and the reference itself."""
import ctypes as C
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from tests import cache4_ref as R4
from tests.test_cache_host import BATCH_BAD, _append, _attend, _batch, _cache, _fake, lib  # noqa: F401
from tests.test_cache_host_edges import Launched, OnGpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _pages(lib, **kw):  # noqa: F811
    return _cache(lib, **dict(dtype=lib.F4E2M1, **kw))


def _read(lib, cache=None, batch=None, **kw):  # noqa: F811
    a = lib.CacheReadArgs(cache or _pages(lib), batch or _batch(lib), 0x800000, 0x900000, 128, 128, lib.BF16)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


PAGES_BAD = [
    ({"dtype": 4}, 1), ({"n_pages": 0}, 1), ({"page_size": 24}, 2), ({"page_size": 256}, 2), ({"H": 0}, 1), ({"d": 96}, 2), ({"d": 32}, 2),
    ({"k": None}, 1), ({"v": 0x200004}, 1), ({"row_stride": 120}, 1), ({"row_stride": 136}, 1), ({"row_stride": 0}, 1), ({"k_scale": None}, 1),
    ({"v_scale": None}, 1), ({"k_scale": 0x300008}, 1), ({"v_scale": 0x400004}, 1),
]


@pytest.mark.parametrize("bad,status", PAGES_BAD)
def test_pages_refusals(lib, bad, status):  # noqa: F811
    cache = _cache(lib, **dict(dict(dtype=lib.F4E2M1), **bad))
    so = lib.library()
    assert so.cast_cache_append(C.byref(_append(lib, cache=cache)), None) == status
    assert so.cast_last_error_detail() != b""
    assert so.cast_cache_attention(C.byref(_attend(lib, cache=cache)), _fake(), 1 << 40, None) == status
    assert so.cast_cache_read(C.byref(_read(lib, cache=cache)), None) == status


@pytest.mark.parametrize("bad,status", BATCH_BAD)
def test_read_batch_refusals(lib, bad, status):  # noqa: F811
    assert lib.library().cast_cache_read(C.byref(_read(lib, batch=_batch(lib, **bad))), None) == status
    assert lib.library().cast_last_error_detail() != b""


@pytest.mark.parametrize("bad,status", [
    ({"k_out": None, "v_out": None}, 1), ({"k_out": 0x800008}, 1), ({"v_out": 0x900004}, 1), ({"k_row_stride": 120}, 1),
    ({"v_row_stride": 132}, 1), ({"out_dtype": 2}, 1), ({"out_dtype": 3}, 1), ({"out_dtype": -1}, 1),
])
def test_read_refusals(lib, bad, status):  # noqa: F811
    assert lib.library().cast_cache_read(C.byref(_read(lib, **bad)), None) == status
    assert lib.library().cast_last_error_detail() != b""
    assert lib.library().cast_cache_read(None, None) == 1


def test_nothing_to_do_is_ok(lib):  # noqa: F811
    b = _batch(lib, T=0, max_new=0)
    c = _pages(lib)
    assert lib.library().cast_cache_read(C.byref(_read(lib, batch=b, k_out=None, v_out=None)), None) == 0
    assert lib.library().cast_cache_append(C.byref(_append(lib, cache=c, batch=b, k=None, v=None, q=None)), None) == 0
    assert lib.library().cast_cache_attention(C.byref(_attend(lib, cache=c, batch=b, q=None, o=None)), None, 0, None) == 0


def test_attention_workspace_is_checked(lib):  # noqa: F811
    so = lib.library()
    for new in (1, 100):
        a = _attend(lib, cache=_pages(lib), batch=_batch(lib, T=2 * new, max_new=new, max_pages=1000, page_table_stride=1000))
        need = so.cast_cache_attention_workspace_size(C.byref(a))
        assert need > 0
        assert so.cast_cache_attention(C.byref(a), _fake(), need - 1, None) == 1
        assert so.cast_cache_attention(C.byref(a), None, need, None) == 1
        assert so.cast_cache_attention(C.byref(a), _fake(0x10010), need, None) == 1


@pytest.mark.parametrize("B,H,H_q,max_pages,whole", [
    (1, 8, 32, 64, True),         # at most 1024 tokens
    (1, 8, 32, 65, False),
    (16, 8, 32, 128, True),       # 128 units of up to 2048
    (15, 8, 32, 128, False),
    (16, 8, 32, 129, False),
    (48, 8, 32, 192, True),       # 384 units of up to 3000
    (48, 8, 32, 193, False),
])
def test_where_a_cta_has_a_whole_unit(lib, B, H, H_q, max_pages, whole):  # noqa: F811
    """Which calls need no workspace: those whose units are not cut."""
    cache = _pages(lib, H=H, d=128, row_stride=H * 128)
    batch = _batch(lib, B=B, T=B, max_new=1, max_pages=max_pages, page_table_stride=max_pages)
    need = lib.library().cast_cache_attention_workspace_size(C.byref(_attend(lib, cache=cache, batch=batch, H_q=H_q)))
    assert (need == 0) == whole


def test_struct_layout_matches_the_header(lib, tmp_path):  # noqa: F811
    if shutil.which("gcc") is None:
        pytest.skip("no gcc")
    py, cname = lib.CacheReadArgs, "cast_cache_read_args"
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "cast.h"', "int main(void) {", f'printf("sizeof %zu\\n", sizeof({cname}));']
    lines += [f'printf("{f} %zu\\n", offsetof({cname}, {f}));' for f, _ in py._fields_]
    lines += ['printf("F4E2M1 %d\\n", CAST_F4E2M1);', "return 0;", "}"]
    (tmp_path / "layout.c").write_text("\n".join(lines))
    subprocess.run(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), str(tmp_path / "layout.c"), "-o", str(tmp_path / "layout")],
                   check=True, capture_output=True)
    for line in subprocess.run([str(tmp_path / "layout")], check=True, capture_output=True, text=True).stdout.splitlines():
        f, val = line.split()
        assert (C.sizeof(py) if f == "sizeof" else lib.F4E2M1 if f == "F4E2M1" else getattr(py, f).offset) == int(val), f


def _tensors(n=4, H=2, page=16, d=64, dtype=torch.uint8):
    k, v = (torch.zeros((n, H, page, d // 2), dtype=dtype) for _ in range(2))
    ks, vs = (torch.zeros((n, H, page, d // 16), dtype=torch.uint8) for _ in range(2))
    return k, v, ks, vs


def test_handle(lib):  # noqa: F811
    k, v, ks, vs = _tensors()
    c = lib.kv_cache(k, v, ks, vs)
    assert (c.dtype, c.n_pages, c.page_size, c.H, c.d, c.row_stride) == (lib.F4E2M1, 4, 16, 2, 64, 128) and c.heads == (2, 64)
    pool = torch.zeros((4, 2, 2, 16, 32), dtype=torch.uint8)     # K and V of a page side by side
    c = lib.kv_cache(pool[:, 0], pool[:, 1], ks, vs)
    assert c.row_stride == 256 and c.v - c.k == 2 * 16 * 32
    assert lib.kv_cache(*_tensors(n=1)).row_stride == 128
    # as before: 8-bit pages as bytes with f32 scales
    f8 = torch.zeros((4, 16, 2, 64), dtype=torch.uint8)
    assert lib.kv_cache(f8, f8, torch.ones(4, 2), torch.ones(4, 2)).dtype == lib.F8E4M3
    if hasattr(torch, "float4_e2m1fn_x2"):
        assert lib.kv_cache(k.view(torch.float4_e2m1fn_x2), v.view(torch.float4_e2m1fn_x2), ks, vs).dtype == lib.F4E2M1


def test_handle_refusals(lib):  # noqa: F811
    k, v, ks, vs = _tensors()
    wide = torch.zeros((4, 2, 16, 8), dtype=torch.uint8)
    for bad in ((k, v[:2], ks, vs), (k, v, ks, None), (k, v, ks, vs[:, :1]), (k, v, ks, vs.float()), (k, v, ks, wide[..., ::2]),
                (k.transpose(1, 2), v.transpose(1, 2), ks, vs), (k[..., ::2], v[..., ::2], ks, vs), (k, v.to(torch.int8), ks, vs),
                (k, torch.zeros((8, 2, 16, 32), dtype=torch.uint8)[::2], ks, vs)):
        with pytest.raises(ValueError):
            lib.kv_cache(*bad)


def test_packed_arguments_are_the_struct(lib):  # noqa: F811
    cache = lib.kv_cache(*_tensors())
    batch = (11, 12, 13, 14, 15, 16, 17, 18)
    want = lib.CacheReadArgs(cache, lib.CacheBatch(*batch), 21, 22, 23, 24, 1)
    assert lib._pack_read(cache.packed, *batch, 21, 22, 23, 24, 1) == bytes(want)


@pytest.fixture
def no_launch(lib, monkeypatch):  # noqa: F811
    """A process whose current GPU is 1 and whose reads end where they would enter the library."""
    def enter(*a):
        raise Launched

    monkeypatch.setattr(lib._lib, "cast_cache_read", enter)
    monkeypatch.setattr(lib, "_current_device", lambda: 1, raising=False)
    monkeypatch.setattr(lib, "_raw_stream", lambda device: 0)


def test_read_takes_tensors_of_the_current_gpu_alone(lib, no_launch):  # noqa: F811
    def call(on, **kw):
        def t(name, x):
            return OnGpu(x, on(name))

        pages = [t(f"cache{i}", x) for i, x in enumerate(_tensors())]
        out = torch.zeros((3, 2, 64), dtype=torch.bfloat16)
        return lib.cast_cache_read(lib.kv_cache(*pages), t("page_table", torch.zeros((1, 2), dtype=torch.int32)),
                                   t("kv_len", torch.zeros(1, dtype=torch.int32)), 3, cu_new=t("cu_new", torch.zeros(2, dtype=torch.int32)),
                                   k_out=t("k_out", out), v_out=t("v_out", out), **kw)

    with pytest.raises(Launched):
        call(lambda name: 1)
    with pytest.raises(ValueError):
        call(lambda name: 0)
    for other in ("cache0", "cache1", "cache2", "cache3", "page_table", "kv_len", "cu_new", "k_out", "v_out"):
        with pytest.raises(ValueError):
            call(lambda name: 0 if name == other else 1)

    class Stream:
        cuda_stream, device_index = 0, 0

    with pytest.raises(ValueError):
        call(lambda name: 1, stream=Stream())


def test_read_refuses_outputs_of_another_form(lib, no_launch):  # noqa: F811
    cache = lib.kv_cache(*(OnGpu(x, 1) for x in _tensors()))
    table, n = OnGpu(torch.zeros((1, 2), dtype=torch.int32), 1), OnGpu(torch.zeros(1, dtype=torch.int32), 1)
    good = torch.zeros((3, 2, 64), dtype=torch.bfloat16)
    for bad in (good.float(), good[:2], good.view(3, 4, 32), torch.zeros((3, 64, 2), dtype=torch.bfloat16).transpose(1, 2),
                torch.zeros((3, 2, 128), dtype=torch.bfloat16)[..., ::2]):
        with pytest.raises(ValueError):
            lib.cast_cache_read(cache, table, n, 3, k_out=OnGpu(bad, 1), values=False)
    with pytest.raises(ValueError):
        lib.cast_cache_read(cache, table, n, 3, keys=False, values=False)
    with pytest.raises(ValueError):
        lib.cast_cache_read(cache, OnGpu(torch.zeros((1, 2)), 1), n, 3, k_out=OnGpu(good, 1), values=False)


def test_every_scale_byte_is_the_upper_half_of_an_f16(lib):  # noqa: F811
    code = np.arange(256)
    f16 = (code.astype(np.uint16) << 7).view(np.float16).astype(np.float64)
    assert np.array_equal(R4.scale_value(code), f16, equal_nan=True)
    a = f16[:0xe3]
    assert np.array_equal(R4.scale_code(a), code[:0xe3])
    mid = (a[1:] + a[:-1]) / 2
    assert np.array_equal(R4.scale_code(mid), (code[:0xe2] + 1) & ~1)       # ties to the even code
    assert (R4.scale_code(mid * (1 + 1e-9)) == code[1:0xe3]).all() and (R4.scale_code(mid * (1 - 1e-9)) == code[:0xe2]).all()


def test_values_are_exact_in_f16_and_bf16(lib):  # noqa: F811
    v = np.outer(R4.VALUES, R4.scale_value(np.arange(0xe3)))
    assert np.array_equal(v, v.astype(np.float16).astype(np.float64))
    assert np.array_equal(v, torch.tensor(v).to(torch.bfloat16).double().numpy())


def test_reference_rounds_to_nearest(lib):  # noqa: F811
    r = np.random.default_rng(1)
    x = r.standard_normal((500, 2, 64)) * np.exp2(r.integers(-6, 6, (500, 2, 1)))
    v, s = R4.quantise(x)
    scale = np.repeat(R4.scale_value(s), 16, -1)
    every = np.concatenate([R4.VALUES, -R4.VALUES]) * scale[..., None]
    assert np.array_equal(np.abs(v - x), np.abs(every - x[..., None]).min(-1))
    R4.check_quantised(v, s, x, np.zeros_like(x))
    with pytest.raises(AssertionError):
        R4.check_quantised(v + scale, s, x, np.zeros_like(x))
