// What the two attention kernels of the paged cache share: the decoding of 8-bit rows, and the form
// for many rows a sequence (cache_tiles.cu) as the entry point (cache_attention.cu) calls it.
#pragma once
#include "cache.cuh"

namespace cast {

struct TilesPlan {
  int tile_tokens, pairs, n_split;
  size_t part_o_bytes, total_bytes;
};
TilesPlan tiles_plan(const cast_cache_attn_args& a);
// Arguments must have been validated; ws holds tiles_plan(a).total_bytes.
cast_status launch_tiles(const cast_cache_attn_args& a, const TilesPlan& p, void* ws, cudaStream_t st);

__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const __nv_bfloat162 x = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&x);
}
__device__ __forceinline__ uint32_t mul2(uint32_t a, uint32_t b) {
  uint32_t y;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(y) : "r"(a), "r"(b));
  return y;
}

// A page's scale as the two bf16 factors of the decoding: 2^120 * scale overflows bf16 from 2^8 on
struct Factor {
  uint32_t once, twice;   // bf16 pairs; `twice` is 1 unless the scale is above 128
  bool two;
};
__device__ __forceinline__ Factor factor_of(float scale) {
  Factor f;
  f.two = scale > 128.f;
  const float a = f.two ? 0x1p120f : scale * 0x1p120f;
  f.once = pack2(a, a);
  f.twice = pack2(scale, scale);
  return f;
}
// Codes 0, 2 (even) and 1, 3 (odd) of a word as bf16 pairs: a code's exponent and mantissa moved to
// bf16's fields are code * 2^-120, a subnormal code included.  The format's NaN (seven bits set) comes
// out as 480: see fix_nan.
__device__ __forceinline__ void decode4(uint32_t w, const Factor& f, uint32_t& even, uint32_t& odd) {
  even = ((w << 4) & 0x07f007f0u) | ((w << 8) & 0x80008000u);
  odd = ((w >> 4) & 0x07f007f0u) | (w & 0x80008000u);
  even = mul2(even, f.once);
  odd = mul2(odd, f.once);
  if (f.two) {
    even = mul2(even, f.twice);
    odd = mul2(odd, f.twice);
  }
}
__device__ __forceinline__ uint32_t nan_bits(uint32_t w) { return (w & 0x7f7f7f7fu) + 0x01010101u; }
__device__ __forceinline__ void fix_nan(uint32_t w, uint32_t& even, uint32_t& odd) {
  if ((w & 0x0000007fu) == 0x0000007fu) even |= 0x00007fffu;
  if ((w & 0x00007f00u) == 0x00007f00u) odd |= 0x00007fffu;
  if ((w & 0x007f0000u) == 0x007f0000u) even |= 0x7fff0000u;
  if ((w & 0x7f000000u) == 0x7f000000u) odd |= 0x7fff0000u;
}
// 16 codes, NaN included, with four consecutive ones in the order 0, 2, 1, 3
__device__ __forceinline__ void decode16(uint2 a, uint2 b, const Factor& f, uint4& oa, uint4& ob) {
  decode4(a.x, f, oa.x, oa.y);
  decode4(a.y, f, oa.z, oa.w);
  decode4(b.x, f, ob.x, ob.y);
  decode4(b.y, f, ob.z, ob.w);
  if (((nan_bits(a.x) | nan_bits(a.y) | nan_bits(b.x) | nan_bits(b.y)) & 0x80808080u) != 0u) {
    fix_nan(a.x, oa.x, oa.y);
    fix_nan(a.y, oa.z, oa.w);
    fix_nan(b.x, ob.x, ob.y);
    fix_nan(b.y, ob.z, ob.w);
  }
}
// Whether a 16-byte chunk of V holds a value that is not finite
template <bool F8>
__device__ __forceinline__ bool not_finite(const uint4& x) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (F8) bad |= (((w[i] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0u;
    else bad |= (w[i] & 0x7f80u) == 0x7f80u || (w[i] & 0x7f800000u) == 0x7f800000u;
  }
  return bad;
}

}  // namespace cast
