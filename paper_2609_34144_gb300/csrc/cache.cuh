// What the paged-cache kernels share: sequences and pages of a call, 8-bit pages, the rotation.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include "internal.h"

namespace cast {

namespace {
// Set when a page, a position or a token was left out: one word for each translation unit, so that its
// kernels name it themselves.
__device__ unsigned int g_left_out;
__device__ __forceinline__ void left_out() { atomicExch(&g_left_out, 1u); }
inline unsigned int read_left_out(cudaStream_t st, bool clear) {
  unsigned int v = 0;
  cudaMemcpyFromSymbolAsync(&v, g_left_out, sizeof(v), 0, cudaMemcpyDeviceToHost, st);
  cudaStreamSynchronize(st);
  if (clear && v) {
    const unsigned int z = 0;
    cudaMemcpyToSymbolAsync(g_left_out, &z, sizeof(z), 0, cudaMemcpyHostToDevice, st);
    cudaStreamSynchronize(st);
  }
  return v;
}
}  // namespace

// Sequence b of a call: its new tokens are rows t0 .. t0 + n_new - 1, its cache holds `len` tokens.
struct Sequence {
  int t0, n_new, len;
};
__device__ __forceinline__ Sequence sequence_of(const cast_cache_batch& a, int b) {
  Sequence s;
  if (a.cu_new) {
    // clamped, so that a table which does not ascend cannot lead out of the call's rows
    s.t0 = min(max(__ldg(a.cu_new + b), 0), a.T);
    s.n_new = min(max(__ldg(a.cu_new + b + 1), s.t0), a.T) - s.t0;
  } else {
    s.n_new = a.T / a.B;
    s.t0 = b * s.n_new;
  }
  s.len = max(__ldg(a.kv_len + b), 0);
  return s;
}

// Sum over a warp of numbers from 0 to 2^52 (the work of a call passes 32 bits)
__device__ __forceinline__ int64_t warp_sum(int64_t x) {
  const uint32_t low = __reduce_add_sync(0xffffffffu, (uint32_t)x & 0x3ffffffu);
  const uint32_t high = __reduce_add_sync(0xffffffffu, (uint32_t)(x >> 26));
  return ((int64_t)high << 26) + low;
}

// ------------------------------------------------------------------ rotation
// (cos, sin) * amplitude of the angle that pair i turns by at `pos`.  The table holds turns a
// position in units of 2^-64: the product modulo 2^64 is the turn's fraction, exactly, at any
// position, and its top 32 bits as a signed number lie in [-1/2, 1/2) turns.
__device__ __forceinline__ float2 rotary_cs(const cast_rotary_table& t, int i, int pos) {
  const uint64_t frac = (uint64_t)(int64_t)pos * t.turn[i];
  const float half_turns = (float)(int32_t)(frac >> 32) * 0x1p-31f;
  float s, c;
  sincospif(half_turns, &s, &c);
  return make_float2(c * t.amplitude, s * t.amplitude);
}

// A unit is 16 channels of one head in two runs of 8: for the half layout the two partners'
// runs, elsewhere 16 consecutive channels.  Units 0 .. rot/16-1 are rotated; pair 8u + i is
// (a[i], b[i]) in the half layout, (v[2i], v[2i+1]) in the interleaved one.
__device__ __forceinline__ void unit_channels(int u, int layout, int rot, int& c0, int& c1) {
  if (layout == CAST_ROTARY_HALF && u < rot / 16) {
    c0 = 8 * u;
    c1 = 8 * u + rot / 2;
  } else {
    c0 = 16 * u;
    c1 = 16 * u + 8;
  }
}
__device__ __forceinline__ void rotate_unit(float* v, const float2* cs, int layout) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 t = cs[i];
    if (layout == CAST_ROTARY_HALF) {
      const float a = v[i], b = v[8 + i];
      v[i] = a * t.x - b * t.y;
      v[8 + i] = b * t.x + a * t.y;
    } else {
      const float a = v[2 * i], b = v[2 * i + 1];
      v[2 * i] = a * t.x - b * t.y;
      v[2 * i + 1] = b * t.x + a * t.y;
    }
  }
}

// 8 bf16 channels <-> 8 floats
__device__ __forceinline__ void unpack8(const uint4& r, float* v) {
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ uint4 pack8(const float* v) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&b);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// ------------------------------------------------------------------ 8-bit pages
// Two floats within +-448 (or NaN) as e4m3 codes, to nearest even
__device__ __forceinline__ uint32_t code2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint2 encode8(const float* v) {
  return make_uint2(code2(v[0], v[1]) | code2(v[2], v[3]) << 16, code2(v[4], v[5]) | code2(v[6], v[7]) << 16);
}
// Asynchronous copies of 16 bytes to shared memory
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// Least e in [-120, 120] with amax <= 448 * 2^e (448 = 1.75 * 2^8)
__device__ __forceinline__ int scale_exponent(float amax) {
  if (!(amax > 0.f)) return -120;
  const uint32_t bits = __float_as_uint(amax);
  const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return min(max(e, -120), 120);
}
__device__ __forceinline__ float pow2f(int e) { return __int_as_float((e + 127) << 23); }

}  // namespace cast
