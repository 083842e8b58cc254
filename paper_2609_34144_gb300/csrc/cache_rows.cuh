// What the two kernels of the paged cache's attention for few rows a sequence share (cache_attention.cu, bf16 and
// 8-bit pages; cache4_attention.cu, 4-bit pages): what a unit's rows see, a CTA's share of the work, the joining.
#pragma once
#include "cache.cuh"
#include "cache_attention.cuh"

namespace cast {

struct RowsKArgs {
  cast_cache_batch batch;
  int n_pages, page_size, page_shift, H, H_q, group;   // page_size = 2^page_shift, group = H_q / H
  int causal, window, sinks, o_f32;
  int64_t row_stride, q_stride;
  const uint8_t *k, *v;
  const float *k_scale, *v_scale;
  const __nv_bfloat16* q;
  void* o;
  float* lse;
  float scale_log2;
  int row_tiles;      // units of ROWS rows that a sequence may have
  int least;          // blocks that a CTA takes at least
  int whole;          // every CTA has one whole unit
  int two, units;     // 1: units of two KV heads side by side, else 0; units of an entry
  float* part_o;      // [2 * grid][1 + two][ROWS][D]
  float2* part_ml;    // [2 * grid][1 + two][ROWS]
  struct RowsCut* cuts;   // 4-bit pages: [grid]
};
// What a CTA leaves for the joining (4-bit pages): the unit that its share begins inside of, which CTAs c0 .. c1 have
// blocks of (c0 = -1: it begins with a unit, or has none)
struct RowsCut {
  int c0, c1, h, tile, t0, n_rows;
};

namespace {

constexpr float kRescale = 8.f;   // the running maximum is renewed when a logit exceeds it by 2^8
// 8-bit pages: probabilities, at most 2^8 times a row's largest, are lifted by 2^7 to use f16's range
constexpr float kLift = 7.f;
constexpr float kLn2 = 0.69314718055994531f;
constexpr int kWarpsLog = 2, kWarps = 1 << kWarpsLog;

// What the rows of one unit see: blocks [0, n_sink) and [first, end) of BT positions, and within
// them the positions below `sinks` or from lo on, below hi.
struct Span {
  int n_sink, first, end;
  int lo, hi, sinks;
  int p0;        // position of the sequence's first new token
  int n_rows;    // rows of the sequence
  int t0;
  __device__ __forceinline__ int blocks() const { return n_sink + max(end - first, 0); }
  __device__ __forceinline__ int block(int i) const { return i < n_sink ? i : first + (i - n_sink); }
};
template <int BT = 16>
__device__ __forceinline__ Span span_of(const RowsKArgs& a, int b, int row_tile, int rows) {
  const Sequence s = sequence_of(a.batch, b);
  Span z;
  z.t0 = s.t0;
  z.p0 = s.len - s.n_new;
  const int kept = min(s.n_new, a.batch.max_new);
  if (kept < s.n_new) left_out();
  z.n_rows = kept * a.group;
  const int64_t room = (int64_t)a.batch.max_pages * a.page_size;
  if (s.len > room) left_out();
  const int len = (int)min((int64_t)s.len, room);
  const int r0 = row_tile * rows, r1 = min(r0 + rows, z.n_rows) - 1;
  z.n_sink = z.first = z.end = z.lo = z.hi = z.sinks = 0;
  if (r0 > r1) return z;
  z.hi = a.causal ? min(len, max(z.p0 + r1 / a.group + 1, 0)) : len;
  if (a.window > 0) {
    z.lo = min(max(z.p0 + r0 / a.group - a.window + 1, 0), z.hi);
    z.sinks = min(min(a.sinks, z.lo), z.hi);
  }
  z.first = z.lo / BT;
  z.end = (z.hi + BT - 1) / BT;
  z.n_sink = min((z.sinks + BT - 1) / BT, z.first);
  return z;
}

// ---------------------------------------------------------------- warp-level pieces
__device__ __forceinline__ void copy16_or_zero(uint32_t dst, const void* src, bool valid) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(valid ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t addr, uint32_t* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma16816(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma16816h(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack2h(float a, float b) {
  const __half2 x = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&x);
}
// Rows of units without any block get zeros (one CTA's threads do this)
template <int D, int ROWS>
__device__ __forceinline__ void zero_rows(const RowsKArgs& a, int e, int h0, int h1) {
  const Span z = span_of(a, e / a.row_tiles, e % a.row_tiles, ROWS);
  const int r0 = (e % a.row_tiles) * ROWS, n = max(min(r0 + ROWS, z.n_rows) - r0, 0), heads = h1 - h0;
  for (int i = threadIdx.x; i < n * heads * D; i += kWarps * 32) {
    const int c = i % D, h = h0 + i / D % heads, r = r0 + i / (D * heads);
    const int64_t row = (int64_t)(z.t0 + r / a.group) * a.H_q + h * a.group + r % a.group;
    if (a.o_f32) static_cast<float*>(a.o)[row * D + c] = 0.f;
    else static_cast<__nv_bfloat16*>(a.o)[row * D + c] = __float2bfloat16_rn(0.f);
    if (a.lse && c == 0) a.lse[row] = -INFINITY;
  }
}

// A CTA's share of the call's blocks: [at, stop), and the entry (sequence, row tile) it begins in, whose blocks
// begin at entry_at.  False for a CTA without one.  *size: blocks of a share (2^30 at most: no unit has as many).
template <int D, int ROWS, int BT = 16>
__device__ __forceinline__ bool share_of(const RowsKArgs& a, int& entry, int64_t& at, int64_t& stop, int64_t& entry_at,
                                         int* size = nullptr) {
  __shared__ int s_entry;
  __shared__ int64_t s_work[kWarps], s_before;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int entries = a.batch.B * a.row_tiles, units = a.units;
  entry_at = 0;
  if (size) *size = 1;
  if (a.whole) {
    entry = blockIdx.x / units;
    const int h = blockIdx.x - entry * units;
    const int nb = span_of<BT>(a, entry / a.row_tiles, entry % a.row_tiles, ROWS).blocks();
    if (nb == 0) {
      zero_rows<D, ROWS>(a, entry, h << a.two, (h + 1) << a.two);
      return false;
    }
    at = (int64_t)h * nb;
    stop = at + nb;
    return true;
  }
  int64_t mine = 0;
  int none = 0;
  for (int e = threadIdx.x; e < entries; e += kWarps * 32) {
    const int n = span_of<BT>(a, e / a.row_tiles, e % a.row_tiles, ROWS).blocks();
    mine += n;
    none |= n == 0;
  }
  mine = warp_sum(mine);
  if (lane == 0) s_work[warp] = mine;
  none = __syncthreads_or(none);
  int64_t total = 0;
  for (int w = 0; w < kWarps; ++w) total += s_work[w];
  total *= units;
  const int64_t share = max((int64_t)a.least, (total + gridDim.x - 1) / gridDim.x);
  if (size) *size = (int)min(share, (int64_t)1 << 30);
  at = blockIdx.x * share;
  stop = min(at + share, total);
  if (none && blockIdx.x == 0) {
    for (int e = 0; e < entries; ++e)
      if (span_of<BT>(a, e / a.row_tiles, e % a.row_tiles, ROWS).blocks() == 0) zero_rows<D, ROWS>(a, e, 0, a.H);
  }
  if (at >= stop) return false;
  if (warp == 0) {
    int64_t before = 0;
    for (int e0 = 0; e0 < entries; e0 += 32) {
      const int e = e0 + lane;
      const int n = e < entries ? span_of<BT>(a, e / a.row_tiles, e % a.row_tiles, ROWS).blocks() : 0;
      int64_t sum = n;
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += y;
      }
      const unsigned hit = __ballot_sync(0xffffffffu, (before + sum) * units > at);
      if (hit) {
        if (lane == __ffs(hit) - 1) {
          s_entry = e;
          s_before = before + sum - n;
        }
        break;
      }
      before += __shfl_sync(0xffffffffu, sum, 31);
    }
  }
  __syncthreads();
  entry = s_entry;
  entry_at = s_before * units;
  return true;
}

// Joins the warps of a unit (their unnormalised o [warp][row][D], maxima and sums [warp][row] in shared memory) into
// the rows' results, or into the part of the unit that this CTA leaves in `slot`.
template <int D, int ROWS>
__device__ __forceinline__ void join_warps(const RowsKArgs& a, const Span& z, int x, int tile, bool complete, int slot,
                                           const float* mo, const float2* ml) {
  const int two = a.two;
  for (int hw = 0; hw <= two; ++hw)
    for (int y = threadIdx.x; y < ROWS * D / 4; y += kWarps * 32) {
      const int rr = y / (D / 4), c = y % (D / 4) * 4;
      const int r = tile * ROWS + rr;
      if (r >= z.n_rows) continue;
      float top = -INFINITY;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) top = fmaxf(top, (w & two) == hw ? ml[w * ROWS + rr].x : -INFINITY);
      float sum = 0.f;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        // the other head's values are read and left out: no load waits for another
        const float2 v = ml[w * ROWS + rr];
        const float4 o4 = *reinterpret_cast<const float4*>(mo + (w * ROWS + rr) * D + c);
        const bool its = (w & two) == hw;
        const float f = v.x == -INFINITY ? 0.f : exp2_fast(v.x - top);
        sum = its ? fmaf(f, v.y, sum) : sum;
        acc.x = its ? fmaf(f, o4.x, acc.x) : acc.x;
        acc.y = its ? fmaf(f, o4.y, acc.y) : acc.y;
        acc.z = its ? fmaf(f, o4.z, acc.z) : acc.z;
        acc.w = its ? fmaf(f, o4.w, acc.w) : acc.w;
      }
      if (complete) {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        const int64_t row = (int64_t)(z.t0 + r / a.group) * a.H_q + ((x << two) + hw) * a.group + r % a.group;
        if (a.o_f32) {
          *reinterpret_cast<float4*>(static_cast<float*>(a.o) + row * D + c) =
              make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
        } else {
          *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.o) + row * D + c) =
              make_uint2(pack2(acc.x * inv, acc.y * inv), pack2(acc.z * inv, acc.w * inv));
        }
        if (a.lse && c == 0) a.lse[row] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
      } else {
        *reinterpret_cast<float4*>(a.part_o + ((((int64_t)slot << two) + hw) * ROWS + rr) * D + c) = acc;
        if (c == 0) a.part_ml[(((int64_t)slot << two) + hw) * ROWS + rr] = make_float2(top, sum);
      }
    }
}

// Joins the parts of rows lo .. hi-1 of the unit (h, tile) of a sequence that CTAs c0 .. c1 left: one warp a row and some of the parts
// (lanes: four channels each), then over the warps of a row.
constexpr int kMergeWarps = 16;
template <int D, int ROWS>
__device__ __forceinline__ void merge_unit(const RowsKArgs& a, int c0, int c1, int h, int tile, int t0, int n_rows, int lo = 0,
                                           int hi = ROWS) {
  constexpr int LANES = D / 4, GROUPS = 32 / LANES;   // GROUPS parts at a time in a warp
  __shared__ float4 s_o[kMergeWarps * GROUPS][LANES];
  __shared__ float2 s_ml[kMergeWarps * GROUPS];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // warps_per_row warps (a power of two) have every warps_per_row-th part of a row
  const int rows = min(hi, n_rows - tile * ROWS), parts = c1 - c0 + 1;
  int per_row = 1;
  while (per_row * 2 * (rows - lo) <= kMergeWarps && per_row * GROUPS < parts) per_row *= 2;
  for (int r0 = lo; r0 < rows; r0 += kMergeWarps / per_row) {
    const int rr = r0 + warp / per_row, mine = (warp % per_row) * GROUPS + lane / LANES, c = lane % LANES;
    const bool in = rr < rows;
    // CTA c0 began the unit (its second place), the others began inside it (their first place)
    float top = -INFINITY, l = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    if (in) {
      // of the CTAs' first places
      const float2* ml = a.part_ml + (((int64_t)c0 * 2 << a.two) + (h & a.two)) * ROWS + rr;
      const float* po = a.part_o + ((((int64_t)c0 * 2 << a.two) + (h & a.two)) * ROWS + rr) * D + c * 4;
      const int each = ROWS << a.two;   // rows from a CTA's first place to its second
#pragma unroll 4
      for (int i = mine; i < parts; i += per_row * GROUPS) {
        const int64_t rows_on = (int64_t)(2 * i + (i == 0 ? 1 : 0)) * each;
        const float2 v = ml[rows_on];
        const float4 y = *reinterpret_cast<const float4*>(po + rows_on * D);
        const float m = fmaxf(top, v.x);
        const float f0 = top == -INFINITY ? 0.f : exp2_fast(top - m), f1 = v.x == -INFINITY ? 0.f : exp2_fast(v.x - m);
        l = f0 * l + f1 * v.y;
        acc.x = f0 * acc.x + f1 * y.x; acc.y = f0 * acc.y + f1 * y.y;
        acc.z = f0 * acc.z + f1 * y.z; acc.w = f0 * acc.w + f1 * y.w;
        top = m;
      }
    }
    const int place = warp * GROUPS + lane / LANES;
    s_o[place][c] = acc;
    if (c == 0) s_ml[place] = make_float2(top, l);
    __syncthreads();
    if (in && mine == 0) {
      const int n = per_row * GROUPS, first = warp * GROUPS;
      for (int i = 0; i < n; ++i) top = fmaxf(top, s_ml[first + i].x);
      l = 0.f;
      acc = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int i = 0; i < n; ++i) {
        const float2 v = s_ml[first + i];
        const float f = v.x == -INFINITY ? 0.f : exp2_fast(v.x - top);
        const float4 y = s_o[first + i][c];
        l += f * v.y;
        acc.x += f * y.x; acc.y += f * y.y; acc.z += f * y.z; acc.w += f * y.w;
      }
      const float inv = l == 0.f ? 0.f : 1.f / l;
      const int r = tile * ROWS + rr;
      const int64_t row = (int64_t)(t0 + r / a.group) * a.H_q + h * a.group + r % a.group;
      if (a.o_f32) {
        *reinterpret_cast<float4*>(static_cast<float*>(a.o) + row * D + c * 4) =
            make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
      } else {
        *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.o) + row * D + c * 4) =
            make_uint2(pack2(acc.x * inv, acc.y * inv), pack2(acc.z * inv, acc.w * inv));
      }
      if (a.lse && c == 0) a.lse[row] = l == 0.f ? -INFINITY : (top + log2f(l)) * kLn2;
    }
    __syncthreads();
  }
}

// Joins the parts of the units that no single CTA of k_cache_rows had whole: one CTA a unit.
template <int D, int ROWS>
__global__ void __launch_bounds__(kMergeWarps * 32) k_cache_merge(const __grid_constant__ RowsKArgs a, int ctas) {
  __shared__ int64_t s_sum[kMergeWarps], s_before[kMergeWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int entries = a.batch.B * a.row_tiles;
  const int entry = blockIdx.x / a.H, h = blockIdx.x % a.H;
  int64_t sum = 0, before = 0;
  for (int e = threadIdx.x; e < entries; e += kMergeWarps * 32) {
    const int n = span_of(a, e / a.row_tiles, e % a.row_tiles, ROWS).blocks();
    sum += n;
    before += e < entry ? n : 0;
  }
  sum = warp_sum(sum);
  before = warp_sum(before);
  if (lane == 0) {
    s_sum[warp] = sum;
    s_before[warp] = before;
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  __syncthreads();
  int64_t total = 0, at = 0;
  for (int w = 0; w < kMergeWarps; ++w) {
    total += s_sum[w];
    at += s_before[w];
  }
  const int units = a.units;
  total *= units;
  const int64_t share = max((int64_t)a.least, (total + ctas - 1) / ctas);
  const int tile = entry % a.row_tiles;
  const Span z = span_of(a, entry / a.row_tiles, tile, ROWS);
  const int nb = z.blocks();
  at = at * units + (int64_t)(h >> a.two) * nb;
  if (nb == 0) return;
  const int c0 = (int)(at / share), c1 = (int)((at + nb - 1) / share);
  if (c0 == c1) return;   // written whole
  merge_unit<D, ROWS>(a, c0, c1, h, tile, z.t0, z.n_rows);
}

// The same by what the CTAs left of their shares' beginnings: CTA x takes the unit that the share of CTA x + 1 begins
// inside of, if that is the first such share; y: some of its rows, where units have many parts.  Nothing is searched for (48 sequences of 8 heads, windows of 4096 tokens
// of 4 bits 68.6 -> 66.6 us; 128 of 1k to 4k tokens 94 -> 87 us).
template <int D, int ROWS>
__global__ void __launch_bounds__(kMergeWarps * 32) k_cuts_merge(const __grid_constant__ RowsKArgs a) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const RowsCut u = a.cuts[blockIdx.x + 1];
  const int each = ROWS / gridDim.y, lo = blockIdx.y * each;
  if (u.c0 == (int)blockIdx.x && lo < u.n_rows - u.tile * ROWS)
    merge_unit<D, ROWS>(a, u.c0, u.c1, u.h, u.tile, u.t0, u.n_rows, lo, lo + each);
}

// A joining's launch behind the kernel that left the parts
template <class... A>
cast_status launch_joining(void (*kernel)(A...), int64_t grid, int rows, cudaStream_t st, A... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)grid, rows, 1);
  cfg.blockDim = dim3(kMergeWarps * 32, 1, 1);
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, kernel, args...) != cudaSuccess) return check_launch("cache attention merge");
  return check_launch("cache attention merge");
}

}  // namespace

struct RowsPlan {
  int mt, row_tiles, grid, least, two;   // mt: units of 16 * mt rows; 4-bit pages: of 8 * mt
  bool whole;            // a CTA takes a whole unit; else units may be split and are merged
  size_t part_o_bytes, part_ml_bytes, total_bytes;
};
// 4-bit pages (cache4_attention.cu): CTAs that an SM holds, and the launch
int rows4_ctas(int d, int mt);
cast_status launch_rows4(const RowsKArgs& k, const RowsPlan& p, int d, cudaStream_t st);

}  // namespace cast
