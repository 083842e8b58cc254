// What the paged-cache kernels share: sequences and pages of a call, 8- and 4-bit pages, the rotation.
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

// ------------------------------------------------------------------ 4-bit pages
// A page is [H][page_size][d / 2] bytes of codes (channel 2i in the low half of byte i), so that a head's rows
// lie together: 64-byte rows a KV head apart would cost memory half of its rate.  Its scales, [H][page_size][d / 16]
// bytes, are the upper eight bits of f16 numbers without sign (5 exponent, 3 mantissa bits): the range of a scale in
// f16 makes one for the page superfluous, a shift by 7 decodes it, and its four significant bits times a code's two
// are exact in f16 and in bf16.
constexpr uint32_t kScaleTop = 0xe2;    // 10240: six times it is the largest value within f16
constexpr uint32_t kScaleNan = 0xff;

// x / s for s of four bits or fewer and r = 1 / s to 2^-22: x r corrected once by its remainder, which is exact
// (Markstein's correction).  Where the quotient is half way between two codes, or scales, it comes out exactly: the
// correction is good to 2^-43 of it, and the halfway points have five bits at most.
__device__ __forceinline__ float over_scale(float x, float s, float r) {
  const float q = x * r;
  return fmaf(fmaf(-q, s, x), r, q);
}
__device__ __forceinline__ float about_inverse(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// The scale of 16 channels whose largest magnitude has these bits, as its byte: max / 6 to nearest even
__device__ __forceinline__ uint32_t scale4_code(uint32_t top) {
  if (top >= 0x7f800000u) return kScaleNan;
  const float a = over_scale(__uint_as_float(top), 6.f, 1.f / 6.f);
  if (a < 0x1p-14f) return (uint32_t)__float2int_rn(a * 0x1p17f);   // multiples of 2^-17
  uint32_t u = __float_as_uint(a);
  u += 0x7ffffu + ((u >> 20) & 1u);
  return min((u >> 20) - (uint32_t)((127 - 15) << 3), kScaleTop);
}
__device__ __forceinline__ float scale4_value(uint32_t code) {
  return __half2float(__ushort_as_half((unsigned short)(code << 7)));
}
// What the lowest four bits of `code` stand for with a scale, in f16 as pairs of them are formed
__device__ __forceinline__ float value4(uint32_t code, uint32_t scale) {
  const uint32_t m = code & 7u;
  const float v = m < 2 ? 0.5f * m : (float)(2u + (m & 1u)) * pow2f((int)(m >> 1) - 2);
  return __half2float(__float2half_rn((code & 8u ? -v : v) * scale4_value(scale)));
}
// Eight floats as codes, to nearest even (6 at most), the first in the lowest four bits
__device__ __forceinline__ uint32_t encode4(const float* v) {
  uint32_t r;
  asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
      "mov.b32 %0, {b0, b1, b2, b3};\n\t}"
      : "=r"(r) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
  return r;
}
// The four bytes of a word as f16 pairs (low half, high half of a byte)
__device__ __forceinline__ void half8(uint32_t w, uint32_t* h) {
  asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\tmov.b32 {b0, b1, b2, b3}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, b0;\n\tcvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, b2;\n\tcvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(w));
}
// A scale's byte (the lowest of w) as an f16 pair of it twice, and of two scales
__device__ __forceinline__ uint32_t scale4_pair(uint32_t w) { return __byte_perm(w, 0, 0x4040) << 7; }
__device__ __forceinline__ uint32_t scale4_pair(uint32_t low, uint32_t high) { return (low << 7) | (high << 23); }
__device__ __forceinline__ uint32_t times2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}

}  // namespace cast
