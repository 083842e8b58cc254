// What the two attention kernels of the paged cache share: the reading of 8-bit rows, and the form
// for many rows a sequence (cache_tiles.cu) as the entry point (cache_attention.cu) calls it.
#pragma once
#include "cache.cuh"

namespace cast {

struct TilesPlan {
  int tile_tokens, pairs;
  bool whole;      // a CTA has one whole unit; else units may be cut and are joined
  int64_t grid;
  size_t part_o_bytes, part_ml_bytes, total_bytes;
};
TilesPlan tiles_plan(const cast_cache_attn_args& a);
// Arguments must have been validated; ws holds tiles_plan(a).total_bytes.
cast_status launch_tiles(const cast_cache_attn_args& a, const TilesPlan& p, void* ws, cudaStream_t st);

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const __nv_bfloat162 x = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&x);
}
// Codes in the low and the high half of a word as f16 pairs
__device__ __forceinline__ void half4(uint32_t w, uint32_t& lo, uint32_t& hi) {
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\t"
      "cvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}"
      : "=r"(lo), "=r"(hi) : "r"(w));
}
// Whether a 16-byte chunk of V holds a value that is not finite: the carry out of an exponent (bf16) or of
// a magnitude (codes) that is all ones
template <bool F8>
__device__ __forceinline__ bool not_finite(const uint4& x) {
  constexpr uint32_t mask = F8 ? 0x7f7f7f7fu : 0x7f807f80u, one = F8 ? 0x01010101u : 0x00800080u;
  const uint32_t carry = ((x.x & mask) + one) | ((x.y & mask) + one) | ((x.z & mask) + one) | ((x.w & mask) + one);
  return (carry & (F8 ? 0x80808080u : 0x80008000u)) != 0u;
}

}  // namespace cast
