"""The paged cache's handle in C and C++: programs that set and read its scales, for 8- and for 4-bit pages."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CPP = r"""
#include <cstddef>
#include <cstdio>
#include <type_traits>
#include "cast.h"
static_assert(std::is_trivially_copyable<cast_kv_cache>::value && std::is_standard_layout<cast_kv_cache>::value, "a C struct");
static_assert(sizeof(cast_kv_cache) == 64 && offsetof(cast_kv_cache, k_scale) == 48 && offsetof(cast_kv_cache, v_scale) == 56, "as in C");
int main() {
  float f32[4] = {1, 2, 3, 4};
  unsigned char bytes[4] = {5, 6, 7, 8};
  void* any = bytes;
  cast_kv_cache c{};
  if (c.k_scale || c.v_scale) return 1;
  // 8-bit pages: set from and read as float*
  c.k_scale = f32;
  c.v_scale = f32 + 2;
  float* k = c.k_scale;
  const float* v = c.v_scale;
  if (k != f32 || v[1] != 4 || c.k_scale[1] != 2 || *c.v_scale != 3 || c.k_scale == c.v_scale || !c.k_scale) return 2;
  // 4-bit pages: set from bytes and read as void*
  c.k_scale = bytes;
  c.v_scale = any;
  void* b = c.k_scale;
  if (b != bytes || c.v_scale.bytes != any) return 3;
  c.v_scale = nullptr;
  if (c.v_scale) return 4;
  cast_kv_cache d = {CAST_F8E4M3, 1, 16, 1, 64, nullptr, nullptr, 64, f32, f32 + 1};
  if (d.k_scale != f32 || *d.v_scale != 2) return 5;
  cast_kv_cache e = {CAST_F4E2M1, 1, 16, 1, 64, nullptr, nullptr, 64, bytes, any};
  c = e;
  return c.k_scale.bytes == bytes ? 0 : 6;
}
"""

C = r"""
#include "cast.h"
int main(void) {
  float f32[2] = {1, 2};
  unsigned char bytes[2] = {3, 4};
  cast_kv_cache c = {0};
  c.k_scale = f32;
  float* k = c.k_scale;
  c.v_scale = bytes;
  unsigned char* v = c.v_scale;
  return k[1] == 2 && v[0] == 3 ? 0 : 1;
}
"""


@pytest.mark.parametrize("compiler,std,text", [("g++", "c++11", CPP), ("g++", "c++17", CPP), ("g++", "c++20", CPP), ("gcc", "c99", C), ("gcc", "c11", C)],
                         ids=["c++11", "c++17", "c++20", "c99", "c11"])
def test_scales_in_c_and_cpp(tmp_path, compiler, std, text):
    if shutil.which(compiler) is None:
        pytest.skip(f"no {compiler}")
    src = tmp_path / ("p.cpp" if compiler == "g++" else "p.c")
    src.write_text(text)
    subprocess.run([compiler, f"-std={std}", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "p")],
                   check=True)
    assert subprocess.run([str(tmp_path / "p")]).returncode == 0
