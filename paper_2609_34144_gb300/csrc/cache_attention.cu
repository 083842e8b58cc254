// Attention over the paged KV cache (cast_cache_attention).
//
// Few rows a sequence (single tokens, drafts): k_cache_rows.  A unit is 16 * MT rows of one sequence
// and KV head, a row being (token, query head of the KV head's group), so that the group's heads
// read a key once.  The keys that a unit's rows can see are a list of 16-token blocks (the sinks'
// blocks, then the window's), and all units' blocks in a row are the work of the call: every CTA
// takes an equal share of it, found from the lengths on the device, whatever they are.  A CTA whose
// share begins or ends inside a unit leaves that part (unnormalised o, running maximum and sum) in
// the workspace, and k_cache_merge joins the parts.
//
// Inside a CTA each warp works on its own blocks (w, w + 4, ...) with its own running maximum, sum
// and o in registers, so that there is no barrier between the loads and the end of the unit: its
// lanes fetch K and V rows with 16-byte asynchronous copies into a private ring of stages, in an
// order of 16-byte chunks that ldmatrix reads without bank conflicts, and rows that no row of the
// unit sees are filled with zeros instead of being read.  S = Q K^T and o += P V are m16n8k16
// products: at 16 rows the tensor cores wait for memory anyway.  Where a head's rows are short a unit is
// two KV heads side by side, two warps each, which read the same memory pages at the same time.
//
// 8-bit rows: codes become f16 (one conversion for two, exact) on the way from shared memory to the
// products, and the scales stay outside: a page's K scale multiplies its logits, and a row's o is kept in
// units of the largest V scale that it has seen so far over 2^7, a page's probabilities (f16) carrying its scale
// in those units in their exponent.  Queries are f16 too, each row times the power of two that brings its largest
// channel below 2^15: bf16's eight bits fit, and channels 2^30 below the largest are the first to lose
// one.  The order of channels inside a 16-wide step of Q K^T, and of o's columns, is that in which the
// codes lie in their 32-bit words.
// bf16 pages: a probability is two bf16 numbers, since memory leaves the time for the second product.
// Bound: memory for bf16 pages; for 8-bit ones memory and the latency of dependent instructions (390 a block
// of 16 tokens, issued in half of the slots: three CTAs of 165 registers a thread are what an SM holds).
// Measured, GB300: 48 sequences with windows of 4096, 8 KV heads of 128, 4 query heads each, bf16 (830 MB)
// 138 to 144 us, 5.9 TB/s; 24 sequences of 8k to 32k tokens in 8 bits (1.11 GB) 191 us, 5.8 TB/s.  The latter
// decoding everything to bf16 with integer operations 438 us; by f16 236 us with three CTAs an SM, 246 with two,
// 255 with four; then 205 us with copies that test a whole block at once and logits scaled inside the exponent,
// 190 us with two heads side by side, and 191 us with V units of a row's own.  Units of 32 rows (MT = 2) are for 64-channel heads, which leave the
// registers for it.
#include <cmath>

#include "cache.cuh"
#include "cache_attention.cuh"
#include "ptx.cuh"

namespace cast {
namespace {

constexpr float kRescale = 8.f;   // the running maximum is renewed when a logit exceeds it by 2^8
// 8-bit pages: probabilities, at most 2^8 times a row's largest, are lifted by 2^7 to use f16's range
constexpr float kLift = 7.f;
constexpr float kLn2 = 0.69314718055994531f;
constexpr int kWarpsLog = 2, kWarps = 1 << kWarpsLog;

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
  int row_tiles;      // units of 16 * MT rows that a sequence may have
  int least;          // blocks that a CTA takes at least
  int whole;          // every CTA has one whole unit
  int two, units;     // 1: units of two KV heads side by side, else 0; units of an entry
  float* part_o;      // [2 * grid][1 + two][16 * MT][D]
  float2* part_ml;    // [2 * grid][1 + two][16 * MT]
};

// What the rows of one unit see: blocks [0, n_sink) and [first, end) of 16 positions, and within
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
  z.first = z.lo / 16;
  z.end = (z.hi + 15) / 16;
  z.n_sink = min((z.sinks + 15) / 16, z.first);
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
template <int D, bool F8, int MT>
struct Cfg {
  static constexpr int ROWS = 16 * MT;
  static constexpr int ROWB = D * (F8 ? 1 : 2);        // bytes of a key row
  static constexpr int CHUNKS = ROWB / 16;
  static constexpr int LANE_ROWS = 32 / CHUNKS;        // rows that a warp's copy takes
  static constexpr int COPIES = 16 / LANE_ROWS;
  static constexpr int BLOCK = 16 * ROWB;              // K or V of a 16-token block
  static constexpr int CTAS = F8 ? 3 : 2;              // of an SM
  static constexpr int ROOM = F8 ? 16 * 1024 : 24 * 1024;   // a warp's ring at most
  static constexpr int STAGES = ROOM / (2 * BLOCK) > 8 ? 8 : ROOM / (2 * BLOCK);
  static constexpr int RING = STAGES * 2 * BLOCK;      // of one warp
  static constexpr int MERGE = kWarps * ROWS * (D + 2) * 4;
  static constexpr int SMEM = kWarps * RING > MERGE ? kWarps * RING : MERGE;
  static_assert(STAGES >= 2, "a block is fetched while another is used");
};

// Where chunk c of row r of a block lies: rows of 128 bytes or more permute their eight chunks by
// the row, so that the eight rows of an ldmatrix take eight bank groups; 64-byte rows by row pairs.
template <int ROWB>
__device__ __forceinline__ uint32_t chunk_at(int r, int c) {
  if constexpr (ROWB >= 128) return r * ROWB + ((c ^ (r & 7)) << 4);
  return r * ROWB + ((c ^ ((r >> 1) & 3)) << 4);
}

// Channel c of row r of a V block (8 bits: the code's value)
template <bool F8, int ROWB>
__device__ __forceinline__ float value_at(const uint8_t* block, int r, int c) {
  const uint8_t* p = block + chunk_at<ROWB>(r, c * (F8 ? 1 : 2) / 16) + c * (F8 ? 1 : 2) % 16;
  if constexpr (F8) {
    const __half h(__nv_cvt_fp8_to_halfraw(*p, __NV_E4M3));
    return __half2float(h);
  }
  return __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(p) << 16);
}

template <int D, bool F8, int MT>
__global__ void __launch_bounds__(kWarps * 32, Cfg<D, F8, MT>::CTAS) k_cache_rows(const __grid_constant__ RowsKArgs a) {
  using C = Cfg<D, F8, MT>;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int s_entry;
  __shared__ int64_t s_work[kWarps], s_before;
  __shared__ float2 s_scale[kWarps][C::STAGES];   // K and V scale of a stage's page
  __shared__ float s_prob[kWarps][C::ROWS][17];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = lane >> 2, q4 = lane & 3;
  const int entries = a.batch.B * a.row_tiles;
  // units of an entry; the warp's head in a unit, its first block and the step to its next
  const int two = a.two, units = a.units, head = warp & two, sub = warp >> two, step = kWarps >> two;

  // Rows of units without any block get zeros (one CTA's threads do this)
  auto zero_rows = [&](int e, int h0, int h1) {
    const Span z = span_of(a, e / a.row_tiles, e % a.row_tiles, C::ROWS);
    const int r0 = (e % a.row_tiles) * C::ROWS, n = max(min(r0 + C::ROWS, z.n_rows) - r0, 0), heads = h1 - h0;
    for (int i = threadIdx.x; i < n * heads * D; i += kWarps * 32) {
      const int c = i % D, h = h0 + i / D % heads, r = r0 + i / (D * heads);
      const int64_t row = (int64_t)(z.t0 + r / a.group) * a.H_q + h * a.group + r % a.group;
      if (a.o_f32) static_cast<float*>(a.o)[row * D + c] = 0.f;
      else static_cast<__nv_bfloat16*>(a.o)[row * D + c] = __float2bfloat16_rn(0.f);
      if (a.lse && c == 0) a.lse[row] = -INFINITY;
    }
  };

  // ---- this CTA's share of the call's blocks: [at, stop), and the entry (sequence, row tile) it
  // begins in, whose blocks begin at entry_at
  int entry;
  int64_t at, stop, entry_at = 0;
  if (a.whole) {
    entry = blockIdx.x / units;
    const int h = blockIdx.x - entry * units;
    const int nb = span_of(a, entry / a.row_tiles, entry % a.row_tiles, C::ROWS).blocks();
    if (nb == 0) {
      zero_rows(entry, h << two, (h + 1) << two);
      return;
    }
    at = (int64_t)h * nb;
    stop = at + nb;
  } else {
    int64_t mine = 0;
    int none = 0;
    for (int e = threadIdx.x; e < entries; e += kWarps * 32) {
      const int n = span_of(a, e / a.row_tiles, e % a.row_tiles, C::ROWS).blocks();
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
    at = blockIdx.x * share;
    stop = min(at + share, total);
    if (none && blockIdx.x == 0) {
      for (int e = 0; e < entries; ++e)
        if (span_of(a, e / a.row_tiles, e % a.row_tiles, C::ROWS).blocks() == 0) zero_rows(e, 0, a.H);
    }
    if (at >= stop) return;
    if (warp == 0) {
      int64_t before = 0;
      for (int e0 = 0; e0 < entries; e0 += 32) {
        const int e = e0 + lane;
        const int n = e < entries ? span_of(a, e / a.row_tiles, e % a.row_tiles, C::ROWS).blocks() : 0;
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
  }

  uint8_t* ring = smem + warp * C::RING;
  const uint32_t ring_at = smem_u32(ring);

  for (; at < stop; ++entry) {
    const int b = entry / a.row_tiles, tile = entry % a.row_tiles;
    const Span z = span_of(a, b, tile, C::ROWS);
    const int nb = z.blocks();
    const int* table = a.batch.page_table + (int64_t)b * a.batch.page_table_stride;
    for (int x = nb ? (int)((at - entry_at) / nb) : units; x < units && at < stop; ++x) {
      // blocks k0 .. k1-1 of unit (b, tile, x)
      const int64_t unit_at = entry_at + (int64_t)x * nb;
      const int h = (x << two) + head;
      const int k0 = (int)(at - unit_at);
      const int k1 = (int)min((int64_t)nb, stop - unit_at);

      // Q fragments: rows g and g + 8 of each 16
      uint32_t qf[MT][D / 16][4];
      int pos[MT][2];   // the rows' positions
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int r = tile * C::ROWS + m * 16 + j * 8 + g;
          const bool in = r < z.n_rows;
          const int i = r / a.group;
          pos[m][j] = in ? z.p0 + i : -1;
          const __nv_bfloat16* src =
              a.q + (int64_t)(z.t0 + (in ? i : 0)) * a.q_stride + (h * a.group + (in ? r - i * a.group : 0)) * D;
#pragma unroll
          for (int s = 0; s < D / 16; ++s) {
            uint32_t x, y;
            if constexpr (F8) {
              const uint2 w = __ldg(reinterpret_cast<const uint2*>(src + s * 16 + q4 * 4));
              x = w.x;
              y = w.y;
            } else {
              x = __ldg(reinterpret_cast<const uint32_t*>(src + s * 16 + q4 * 2));
              y = __ldg(reinterpret_cast<const uint32_t*>(src + s * 16 + q4 * 2 + 8));
            }
            qf[m][s][j] = in ? x : 0u;
            qf[m][s][2 + j] = in ? y : 0u;
          }
        }
      float unit[MT][2];   // what a row's logits are multiplied by
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          unit[m][j] = a.scale_log2;
          if constexpr (F8) {
            auto low = [](uint32_t w) { return __uint_as_float(w << 16); };
            auto high = [](uint32_t w) { return __uint_as_float(w & 0xffff0000u); };
            float top = 0.f;
#pragma unroll
            for (int s = 0; s < D / 16; ++s)
#pragma unroll
              for (int e = 0; e < 4; e += 2) {
                const uint32_t w = qf[m][s][e + j];
                top = fmaxf(top, fmaxf(fabsf(low(w)), fabsf(high(w))));
              }
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            // 2^-e with the largest channel in [2^14, 2^15); subnormal, zero and infinite rows as they are
            const int e = (int)(__float_as_uint(top) >> 23) - 127 - 14;
            const bool plain = e < -126 || e > 112;
            const float down = plain ? 1.f : pow2f(-e);
            if (!plain) unit[m][j] *= pow2f(e);
#pragma unroll
            for (int s = 0; s < D / 16; ++s)
#pragma unroll
              for (int e2 = 0; e2 < 4; e2 += 2) {
                const uint32_t w = qf[m][s][e2 + j];
                qf[m][s][e2 + j] = pack2h(low(w) * down, high(w) * down);
              }
          }
        }
      // positions that every row sees: [all_lo, all_hi); the others' blocks are masked
      int all_lo = 0, all_hi = z.hi;
      {
        const int r1 = min(tile * C::ROWS + C::ROWS, z.n_rows) - 1;
        if (a.causal) all_hi = min(z.hi, max(z.p0 + tile * C::ROWS / a.group + 1, 0));
        if (a.window > 0) all_lo = max(z.p0 + r1 / a.group - a.window + 1, 0);
      }

      float o[MT][D / 8][4], m_ref[MT][2], l[MT][2];
      // 8-bit pages: a row's o is in units of 2^(e_ref - kLift), e_ref log2 of the largest V scale that the row has
      // seen so far (its own: a page that it does not see must not cost its values bits)
      float e_ref[MT][2];
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        e_ref[m][0] = e_ref[m][1] = -INFINITY;
#pragma unroll
        for (int t = 0; t < D / 8; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[m][t][e] = 0.f;
        m_ref[m][0] = m_ref[m][1] = -INFINITY;
        l[m][0] = l[m][1] = 0.f;
      }

      // The page of block i of the unit (-1: out of range, reads as zeros)
      auto page_of = [&](int i) {
        const int g0 = (z.block(i) * 16) >> a.page_shift;
        int p = __ldg(table + g0);
        if (p < 0 || p >= a.n_pages) {
          if (lane == 0) left_out();
          p = -1;
        }
        return p;
      };
      // fetches block i of the unit into stage st: in copy c lane l has chunk l % CHUNKS of row
      // c * LANE_ROWS + l / CHUNKS
      const int64_t row_bytes = a.row_stride * (F8 ? 1 : 2), copy_step = row_bytes * C::LANE_ROWS;
      const int64_t lane_off = (lane / C::CHUNKS) * row_bytes + lane % C::CHUNKS * 16 + (int64_t)h * C::ROWB;
      auto fetch = [&](int i, int st, int page) {
        const int base = z.block(i) * 16;
        const int64_t row0 = (int64_t)max(page, 0) * a.page_size + (base & (a.page_size - 1));
        const uint8_t* ks = a.k + row0 * row_bytes + lane_off;
        const uint8_t* vs = ks + (a.v - a.k);
        const uint32_t dst = ring_at + st * 2 * C::BLOCK;
        if (page >= 0 && base + 16 <= z.hi && (base >= z.lo || base + 16 <= z.sinks)) {
#pragma unroll
          for (int c = 0; c < C::COPIES; ++c) {
            const uint32_t to = dst + chunk_at<C::ROWB>(c * C::LANE_ROWS + lane / C::CHUNKS, lane % C::CHUNKS);
            copy16(to, ks + c * copy_step);
            copy16(to + C::BLOCK, vs + c * copy_step);
          }
        } else {
#pragma unroll
          for (int c = 0; c < C::COPIES; ++c) {
            const int r = c * C::LANE_ROWS + lane / C::CHUNKS, p = base + r;
            const bool in = page >= 0 && p < z.hi && (p >= z.lo || p < z.sinks);
            const uint32_t to = dst + chunk_at<C::ROWB>(r, lane % C::CHUNKS);
            copy16_or_zero(to, in ? ks + c * copy_step : a.k, in);
            copy16_or_zero(to + C::BLOCK, in ? vs + c * copy_step : a.v, in);
          }
        }
        if constexpr (F8) {
          // lanes 0 and 1: the page's scales, 4 bytes behind the same group of copies
          if (lane < 2) {
            const float* src = (lane ? a.v_scale : a.k_scale) + (int64_t)max(page, 0) * a.H + h;
            copy4(smem_u32(&s_scale[warp][st]) + 4 * lane, src);
          }
        }
      };
      const int n = k1 - k0 > sub ? (k1 - k0 - sub + step - 1) >> (kWarpsLog - two) : 0;   // blocks of this warp
      const int i0 = k0 + sub;
      __syncwarp();
      for (int st = 0; st < C::STAGES - 1; ++st) {
        if (st < n) fetch(i0 + st * step, st, page_of(i0 + st * step));
        copy_commit();
      }
      int next_page = C::STAGES - 1 < n ? page_of(i0 + (C::STAGES - 1) * step) : -1;

      int st = 0, into = C::STAGES - 1;
      for (int it = 0; it < n; ++it) {
        copy_wait<C::STAGES - 2>();
        __syncwarp();
        // the stage used one block ago takes the block STAGES - 1 ahead
        const int ahead = it + C::STAGES - 1;
        if (ahead < n) fetch(i0 + ahead * step, into, next_page);
        copy_commit();
        if (ahead + 1 < n) next_page = page_of(i0 + (ahead + 1) * step);
        const uint32_t kt = ring_at + st * 2 * C::BLOCK, vt = kt + C::BLOCK;
        float s[MT][2][4];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[m][t][e] = 0.f;
        float2 sc = make_float2(1.f, 1.f);   // scales of the block's page
        if constexpr (F8) {
          sc = s_scale[warp][st];
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int c = 0; c < D / 16; c += 4) {
              uint32_t w[4];
              ldsm4(kt + chunk_at<C::ROWB>(t * 8 + (lane & 7), c + (lane >> 3)), w);
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                uint32_t b0, b1;
                half4(w[j], b0, b1);
#pragma unroll
                for (int m = 0; m < MT; ++m) mma16816h(s[m][t], qf[m][c + j], b0, b1);
              }
            }
        } else {
#pragma unroll
          for (int c = 0; c < D / 16; ++c) {
            uint32_t w[4];
            ldsm4(kt + chunk_at<C::ROWB>((lane >> 4) * 8 + (lane & 7), 2 * c + ((lane >> 3) & 1)), w);
#pragma unroll
            for (int m = 0; m < MT; ++m) {
              mma16816(s[m][0], qf[m][c], w[0], w[1]);
              mma16816(s[m][1], qf[m][c], w[2], w[3]);
            }
          }
        }
        const int base = z.block(i0 + it * step) * 16;
        const bool whole = base + 16 <= all_hi && (base >= all_lo || base + 16 <= z.sinks);
        float times[MT][2];
        bool grows = false;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int j = 0; j < 2; ++j) times[m][j] = unit[m][j] * sc.x;
        if (!whole) {
#pragma unroll
          for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
#pragma unroll
              for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                  const int p = base + t * 8 + q4 * 2 + e, r = pos[m][j];
                  const bool see = p < z.hi && (!a.causal || p <= r) && (a.window <= 0 || p > r - a.window || p < a.sinks);
                  s[m][t][2 * j + e] = see ? s[m][t][2 * j + e] * times[m][j] : -INFINITY;
                }
              times[m][j] = 1.f;
            }
        }
        float top[MT][2];   // this lane's largest logit of the row
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            top[m][j] = fmaxf(fmaxf(s[m][0][2 * j], s[m][0][2 * j + 1]), fmaxf(s[m][1][2 * j], s[m][1][2 * j + 1])) * times[m][j];
            grows = grows || top[m][j] > m_ref[m][j] + kRescale;
          }
        if (__any_sync(0xffffffffu, grows)) {
#pragma unroll
          for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              float x = top[m][j];
              x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
              x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
              if (x > m_ref[m][j]) {
                const float f = exp2_fast(m_ref[m][j] - x);
                m_ref[m][j] = x;
                l[m][j] *= f;
#pragma unroll
                for (int t = 0; t < D / 8; ++t) {
                  o[m][t][2 * j] *= f;
                  o[m][t][2 * j + 1] *= f;
                }
              }
            }
        }
        // 8-bit pages: probabilities carry the page's V scale in o's units; a scale 2^60 below the largest
        // adds nothing to o, and everything to the sum
        float weight[MT][2], back[MT][2];   // log2, and its inverse for the sum
        const float e = F8 ? __log2f(sc.y) : 0.f;
        if constexpr (F8) {
          bool more = false;
#pragma unroll
          for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int j = 0; j < 2; ++j) more = more || e > e_ref[m][j];
          if (more) {
            const int last = min(base + 15, z.hi - 1);
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                // whether the row sees any of the block
                const int r = pos[m][j], up = a.causal ? min(last, r) : last;
                const bool some = whole || (base <= up && (a.window <= 0 || up > r - a.window || base < a.sinks));
                if (some && e > e_ref[m][j]) {
                  const float f = exp2_fast(e_ref[m][j] - e);
                  e_ref[m][j] = e;
#pragma unroll
                  for (int t = 0; t < D / 8; ++t) {
                    o[m][t][2 * j] *= f;
                    o[m][t][2 * j + 1] *= f;
                  }
                }
              }
          }
        }
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            // (a page that the row does not see may have a larger scale)
            weight[m][j] = F8 ? kLift + fmaxf(fminf(e - e_ref[m][j], 0.f), -60.f) : 0.f;
            back[m][j] = F8 ? exp2_fast(-weight[m][j]) : 1.f;
          }
        // bf16 pages: a probability is two bf16 numbers (16 bits of it); memory leaves the time for the
        // second product
        uint32_t pf[MT][4], rest[MT][4];
#pragma unroll
        for (int m = 0; m < MT; ++m) {
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            // a row that has seen nothing yet: exp2(-inf - 0) = 0
            const float ref = weight[m][j] - (m_ref[m][j] == -INFINITY ? 0.f : m_ref[m][j]);
            float sum = 0.f;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const float p = exp2_fast(fmaf(s[m][t][2 * j + e], times[m][j], ref));
                s[m][t][2 * j + e] = p;
                sum += p;
              }
            l[m][j] = fmaf(sum, back[m][j], l[m][j]);
          }
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const float x = s[m][t][2 * j], y = s[m][t][2 * j + 1];
              pf[m][2 * t + j] = F8 ? pack2h(x, y) : pack2(x, y);
              if constexpr (!F8)
                rest[m][2 * t + j] = pack2(x - __uint_as_float(pf[m][2 * t + j] << 16),
                                           y - __uint_as_float(pf[m][2 * t + j] & 0xffff0000u));
            }
        }
        // A block that the rows do not all see, with a value that is not finite: 0 times it would
        // reach the rows that do not see it, so its tokens are added one by one where they are seen.
        bool apart = false;
        if (!whole) {
          for (int x = lane; x < C::BLOCK / 16; x += 32)
            apart |= not_finite<F8>(*reinterpret_cast<const uint4*>(ring + st * 2 * C::BLOCK + C::BLOCK + x * 16));
          apart = __any_sync(0xffffffffu, apart);
        }
        if (apart) {
#pragma unroll
          for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                s_prob[warp][m * 16 + (e >> 1) * 8 + g][t * 8 + q4 * 2 + (e & 1)] = s[m][t][e];
          __syncwarp();
#pragma unroll 1
          for (int t = 0; t < 16; ++t) {
            const int p = base + t;
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                const int r = pos[m][j];
                const bool see = p < z.hi && (!a.causal || p <= r) && (a.window <= 0 || p > r - a.window || p < a.sinks);
                if (!see) continue;
                const float w = s_prob[warp][m * 16 + j * 8 + g][t];
#pragma unroll
                for (int c = 0; c < D / 8; ++c)
#pragma unroll
                  for (int e = 0; e < 2; ++e) {
                    const int n = F8 ? (c >> 1) * 16 + 2 * (q4 * 2 + e) + (c & 1) : c * 8 + q4 * 2 + e;
                    o[m][c][2 * j + e] += w * value_at<F8, C::ROWB>(ring + st * 2 * C::BLOCK + C::BLOCK, t, n);
                  }
              }
          }
        } else if constexpr (F8) {
          // words of V hold tokens 2 q4 and 2 q4 + 1 of channels 2 g and 2 g + 1
#pragma unroll
          for (int c = 0; c < D / 16; c += 2) {
            uint32_t w[4];
            ldsm4t(vt + chunk_at<C::ROWB>(((lane >> 3) & 1) * 8 + (lane & 7), c + (lane >> 4)), w);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              uint32_t e0, e1, d0, d1;
              half4(__byte_perm(w[2 * j], 0, 0x3120), e0, d0);
              half4(__byte_perm(w[2 * j + 1], 0, 0x3120), e1, d1);
#pragma unroll
              for (int m = 0; m < MT; ++m) {
                mma16816h(o[m][2 * (c + j)], pf[m], e0, e1);
                mma16816h(o[m][2 * (c + j) + 1], pf[m], d0, d1);
              }
            }
          }
        } else {
#pragma unroll
          for (int c = 0; c < D / 16; ++c) {
            uint32_t w[4];
            ldsm4t(vt + chunk_at<C::ROWB>(((lane >> 3) & 1) * 8 + (lane & 7), 2 * c + (lane >> 4)), w);
#pragma unroll
            for (int m = 0; m < MT; ++m) {
              mma16816(o[m][2 * c], pf[m], w[0], w[1]);
              mma16816(o[m][2 * c + 1], pf[m], w[2], w[3]);
              mma16816(o[m][2 * c], rest[m], w[0], w[1]);
              mma16816(o[m][2 * c + 1], rest[m], w[2], w[3]);
            }
          }
        }
        __syncwarp();
        into = st;
        st = st + 1 == C::STAGES ? 0 : st + 1;
      }
      copy_wait<0>();
      __syncthreads();   // every warp is done with its ring: the merge takes the space

      // ---- join the warps of a head
      float* mo = reinterpret_cast<float*>(smem);                        // [warp][row][D]
      float2* ml = reinterpret_cast<float2*>(mo + kWarps * C::ROWS * D); // [warp][row]
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          float x = l[m][j];
          x += __shfl_xor_sync(0xffffffffu, x, 1);
          x += __shfl_xor_sync(0xffffffffu, x, 2);
          const int r = m * 16 + j * 8 + g;
          if (q4 == 0) ml[warp * C::ROWS + r] = make_float2(m_ref[m][j], x);
          float* dst = mo + (warp * C::ROWS + r) * D;
          if constexpr (F8) {
            const float f = exp2_fast(e_ref[m][j]) * 0x1p-7f;
#pragma unroll
            for (int c = 0; c < D / 16; ++c)
              *reinterpret_cast<float4*>(dst + c * 16 + q4 * 4) =
                  make_float4(o[m][2 * c][2 * j] * f, o[m][2 * c + 1][2 * j] * f, o[m][2 * c][2 * j + 1] * f,
                              o[m][2 * c + 1][2 * j + 1] * f);
          } else {
#pragma unroll
            for (int t = 0; t < D / 8; ++t)
              *reinterpret_cast<float2*>(dst + t * 8 + q4 * 2) = make_float2(o[m][t][2 * j], o[m][t][2 * j + 1]);
          }
        }
      __syncthreads();
      const bool complete = k0 == 0 && k1 == nb;
      // a share that begins inside the unit leaves its part in the CTA's first place
      const int slot = 2 * blockIdx.x + (k0 > 0 ? 0 : 1);
      for (int hw = 0; hw <= two; ++hw)
        for (int y = threadIdx.x; y < C::ROWS * D / 4; y += kWarps * 32) {
          const int rr = y / (D / 4), c = y % (D / 4) * 4;
          const int r = tile * C::ROWS + rr;
          if (r >= z.n_rows) continue;
          float top = -INFINITY;
#pragma unroll
          for (int w = 0; w < kWarps; ++w) top = fmaxf(top, (w & two) == hw ? ml[w * C::ROWS + rr].x : -INFINITY);
          float sum = 0.f;
          float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
          for (int w = 0; w < kWarps; ++w) {
            // the other head's values are read and left out: no load waits for another
            const float2 v = ml[w * C::ROWS + rr];
            const float4 o4 = *reinterpret_cast<const float4*>(mo + (w * C::ROWS + rr) * D + c);
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
            *reinterpret_cast<float4*>(a.part_o + ((((int64_t)slot << two) + hw) * C::ROWS + rr) * D + c) = acc;
            if (c == 0) a.part_ml[(((int64_t)slot << two) + hw) * C::ROWS + rr] = make_float2(top, sum);
          }
        }
      __syncthreads();   // the space goes back to the rings
      at = unit_at + k1;
    }
    entry_at += (int64_t)nb * units;
  }
}

// Joins the parts of the units that no single CTA of k_cache_rows had whole: one CTA a unit, one warp a
// row and some of the parts (lanes: four channels each), then over the warps of a row.
constexpr int kMergeWarps = 16;
template <int D, int MT>
__global__ void __launch_bounds__(kMergeWarps * 32) k_cache_merge(const __grid_constant__ RowsKArgs a, int ctas) {
  constexpr int ROWS = 16 * MT, LANES = D / 4, GROUPS = 32 / LANES;   // GROUPS parts at a time in a warp
  __shared__ int64_t s_sum[kMergeWarps], s_before[kMergeWarps];
  __shared__ float4 s_o[kMergeWarps * GROUPS][LANES];
  __shared__ float2 s_ml[kMergeWarps * GROUPS];
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
  // warps_per_row warps (a power of two) have every warps_per_row-th part of a row
  const int rows = min(ROWS, z.n_rows - tile * ROWS), parts = c1 - c0 + 1;
  int per_row = 1;
  while (per_row * 2 * rows <= kMergeWarps && per_row * GROUPS < parts) per_row *= 2;
  for (int r0 = 0; r0 < rows; r0 += kMergeWarps / per_row) {
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
      const int64_t row = (int64_t)(z.t0 + r / a.group) * a.H_q + h * a.group + r % a.group;
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

// ---------------------------------------------------------------- host side
struct RowsPlan {
  int mt, row_tiles, grid, least, two;
  bool whole;            // a CTA takes a whole unit; else units may be split and are merged
  size_t part_o_bytes, total_bytes;
};
RowsPlan rows_plan(const cast_cache_attn_args& a) {
  RowsPlan p{};
  const int group = a.H_q / a.cache.H;
  const int max_new = a.batch.max_new < a.batch.T ? a.batch.max_new : a.batch.T;
  p.mt = (int64_t)max_new * group > 16 ? 2 : 1;   // 16 rows of a product, or two of them for the same keys
  const int rows = 16 * p.mt;
  p.row_tiles = (int)(((int64_t)max_new * group + rows - 1) / rows);
  int dev = 0, nsm = 152;
  if (cudaGetDevice(&dev) == cudaSuccess) cudaDeviceGetAttribute(&nsm, cudaDevAttrMultiProcessorCount, dev);
  p.grid = (a.cache.dtype == CAST_F8E4M3 ? Cfg<128, true, 1>::CTAS : Cfg<128, false, 1>::CTAS) * (nsm < 1 ? 1 : nsm);
  p.least = 16;
  // Blocks that a unit has at most.  Up to 64 (a thousand tokens: four blocks' latency a warp's ring)
  // a CTA takes a whole unit and nothing is joined.  Measured, shares / whole units, us: one sequence of 301
  // tokens 12.5 / 6.9; 1000 tokens, 32 units 15.9 / 16.1, 384 units 48 / 46, ragged 38 / 34; but 4000 tokens (250
  // blocks), 32 units 23 / 57, 384 units 131 / 147.
  const int64_t room = (int64_t)a.batch.max_pages * a.cache.page_size;
  int64_t most = room / 16;
  if (a.window > 0) {
    const int64_t seen = ((int64_t)a.window + rows) / 16 + 2 + ((int64_t)a.sinks + 15) / 16;
    if (seen < most) most = seen;
  }
  p.whole = most <= 64;
  if (p.whole) {
    const int64_t units = (int64_t)a.batch.B * p.row_tiles * a.cache.H;
    p.grid = units > 0x7fffffff ? 0 : (int)units;
    return p;
  }
  // Units of two KV heads side by side, where one head's rows are at most 128 bytes in rows of 512 or more: what
  // a fetch takes of a memory page is little otherwise.  Measured, one head / two, us: 24 sequences of 8k to 32k
  // tokens, 8 bits, 8 heads of 128 205 / 191 (on another box 192 / 191), 8 heads of 64 165 / 127, 10 of 64
  // 237 / 155, 16 of 64 358 to 400 / 240; bf16, 8 heads of 64 207 / 185; 32 sequences, 6 heads of 128 in 8 bits
  // 190 / 181, of 64 in bf16 197 / 178; 48 sequences, rows of 512 bytes: 8 bits, 4 heads of 128 189 / 188, windows
  // of 4096 53.5 / 53.9, 8 heads of 64 69 / 64; bf16, 4 of 64 178 / 175, windows 8 of 64 87.5 / 82.5, 12 of 64
  // 128 / 113, but 8 of 128 (256 bytes each) 144 / 145.  A unit's parts are twice as many: with 64 units 73 / 72, 32 units 44 / 46.
  const int row = a.cache.d * (a.cache.dtype == CAST_F8E4M3 ? 1 : 2);
  p.two = row <= 128 && a.cache.H % 2 == 0 && (int64_t)a.cache.H * row >= 512 && (int64_t)a.batch.B * p.row_tiles * a.cache.H >= 128;
  p.least >>= p.two;
  p.part_o_bytes = align_up(((size_t)2 * p.grid << p.two) * rows * a.cache.d * sizeof(float));
  p.total_bytes = p.part_o_bytes + align_up(((size_t)2 * p.grid << p.two) * rows * sizeof(float2));
  return p;
}

cast_status validate_attention(const cast_cache_attn_args* a, const char* who) {
  if (!a) return fail(CAST_ERR_INVALID_ARG, "%s: args is NULL", who);
  cast_status s = validate_cache(a->cache, who);
  if (s) return s;
  if ((s = validate_batch(a->batch, who))) return s;
  if (a->H_q < 1 || a->H_q % a->cache.H)
    return fail(CAST_ERR_INVALID_ARG, "%s: H_q %d is not a multiple of the cache's %d heads", who, a->H_q, a->cache.H);
  if (a->H_q / a->cache.H > 128) return fail(CAST_ERR_UNSUPPORTED, "%s: %d query heads a KV head", who, a->H_q / a->cache.H);
  if (a->window < 0 || a->sinks < 0)
    return fail(CAST_ERR_INVALID_ARG, "%s: window %d and sinks %d must be >= 0", who, a->window, a->sinks);
  if (!std::isfinite(a->scale)) return fail(CAST_ERR_INVALID_ARG, "%s: scale is not finite", who);
  if (a->o_dtype != CAST_BF16 && a->o_dtype != CAST_F32)
    return fail(CAST_ERR_INVALID_ARG, "%s: o_dtype %d", who, a->o_dtype);
  if (a->batch.T == 0) return CAST_OK;
  if (!a->q || !aligned16(a->q) || !a->o || !aligned16(a->o))
    return fail(CAST_ERR_INVALID_ARG, "%s: q or o is NULL or not 16-byte aligned", who);
  if (reinterpret_cast<uintptr_t>(a->lse) % sizeof(float))
    return fail(CAST_ERR_INVALID_ARG, "%s: lse is not 4-byte aligned", who);
  if (a->q_row_stride < (int64_t)a->H_q * a->cache.d || a->q_row_stride % 8)
    return fail(CAST_ERR_INVALID_ARG, "%s: q row stride %lld must be >= H_q*d and a multiple of 8", who,
                (long long)a->q_row_stride);
  return CAST_OK;
}

template <int D, bool F8, int MT>
cast_status launch_rows(const RowsKArgs& k, const RowsPlan& p, cudaStream_t st) {
  using C = Cfg<D, F8, MT>;
  static std::atomic<uint64_t> attr_done{0};
  if (!once_per_device(attr_done, [&] {
        return cudaFuncSetAttribute(k_cache_rows<D, F8, MT>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM) ==
               cudaSuccess;
      }))
    return check_launch("cache attention smem attribute");
  k_cache_rows<D, F8, MT><<<p.grid, kWarps * 32, C::SMEM, st>>>(k);
  cast_status s = check_launch("cache attention");
  if (s || p.whole) return s;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(k.batch.B * k.row_tiles * k.H), 1, 1);
  cfg.blockDim = dim3(kMergeWarps * 32, 1, 1);
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, k_cache_merge<D, MT>, k, p.grid) != cudaSuccess) return check_launch("cache attention merge");
  return check_launch("cache attention merge");
}

}  // namespace

unsigned int cache_rows_error_word(cudaStream_t st, bool clear) { return read_left_out(st, clear); }

}  // namespace cast

using namespace cast;

extern "C" {

// Up to 16 rows a sequence and KV head go to k_cache_rows, more to the tiles of 128 (cache_tiles.cu),
// except that heads of 64 with up to 32 rows stay where there are 64 units or more (two products of 16 rows
// on the same keys).  Measured, tiles / rows, heads of 64, us, 8 bits and bf16: 256 units of 5k tokens with 32
// rows 101 / 82, 95 / 81; 108 units of 2.4k with 18 rows 36 / 30, 35 / 31; 64 units of 20k with 32 rows 80 / 79,
// 84 / 79; 32 units of 20k 49 / 54, 51 / 52; 16 units of 60k 64 / 72, 68 / 68; 8 units of 3k 19 / 22, 17 / 21.
// Heads of 128 have not the registers for two products (8 bits spill 650 bytes; bf16 takes 255): 32 rows, 16 units
// of 60k 71 / 188, 90 / 108; 256 units of 5k 112 / 240, 123 / 129.
static bool by_tiles(const cast_cache_attn_args& a) {
  const int max_new = a.batch.max_new < a.batch.T ? a.batch.max_new : a.batch.T;
  const int64_t rows = (int64_t)max_new * (a.H_q / a.cache.H);
  return rows > 32 || (rows > 16 && (a.cache.d != 64 || (int64_t)a.batch.B * a.cache.H < 64));
}

size_t cast_cache_attention_workspace_size(const cast_cache_attn_args* a) {
  // 0 for what the call refuses: the plans divide by the sequences, and by 128 rows over the group
  if (!a || a->batch.T < 1 || a->batch.B < 1 || a->batch.max_new < 1 || a->batch.max_pages < 0 || a->cache.page_size < 1 || a->cache.H < 1 ||
      a->H_q < a->cache.H || a->H_q / a->cache.H > 128 || (a->cache.d != 64 && a->cache.d != 128))
    return 0;
  return by_tiles(*a) ? tiles_plan(*a).total_bytes : rows_plan(*a).total_bytes;
}

cast_status cast_cache_attention(const cast_cache_attn_args* a, void* ws, size_t ws_bytes, void* stream) {
  clear_error_detail();
  const char* who = "cast_cache_attention";
  cast_status s = validate_attention(a, who);
  if (s) return s;
  if (a->batch.T == 0) return CAST_OK;
  const bool tiles = by_tiles(*a);
  const TilesPlan tp = tiles ? tiles_plan(*a) : TilesPlan{};
  const RowsPlan p = tiles ? RowsPlan{} : rows_plan(*a);
  const size_t need = tiles ? tp.total_bytes : p.total_bytes;
  if (ws_bytes < need || (need && !ws))
    return fail(CAST_ERR_INVALID_ARG, "%s: workspace %zu B < %zu B", who, ws_bytes, need);
  if (reinterpret_cast<uintptr_t>(ws) % kWsAlign)
    return fail(CAST_ERR_INVALID_ARG, "%s: workspace not 256-byte aligned", who);
  if (tiles) return launch_tiles(*a, tp, ws, static_cast<cudaStream_t>(stream));
  const cast_kv_cache& c = a->cache;
  if ((int64_t)a->batch.B * p.row_tiles * c.H > 0x7fffffff)
    return fail(CAST_ERR_UNSUPPORTED, "%s: too many units", who);
  RowsKArgs k{};
  k.batch = a->batch;
  k.n_pages = c.n_pages;
  k.page_size = c.page_size;
  while ((1 << k.page_shift) < c.page_size) ++k.page_shift;
  k.H = c.H;
  k.H_q = a->H_q;
  k.group = a->H_q / c.H;
  k.causal = a->causal ? 1 : 0;
  // a window as long as a sequence can be hides nothing
  k.window = a->window < (int64_t)a->batch.max_pages * c.page_size ? a->window : 0;
  k.sinks = k.window > 0 ? a->sinks : 0;
  k.o_f32 = a->o_dtype == CAST_F32;
  k.row_stride = c.row_stride;
  k.q_stride = a->q_row_stride;
  k.k = static_cast<const uint8_t*>(c.k);
  k.v = static_cast<const uint8_t*>(c.v);
  k.k_scale = c.k_scale;
  k.v_scale = c.v_scale;
  k.q = static_cast<const __nv_bfloat16*>(a->q);
  k.o = a->o;
  k.lse = a->lse;
  k.scale_log2 = (a->scale > 0.f ? a->scale : 1.f / sqrtf((float)c.d)) * 1.4426950408889634f;
  k.row_tiles = p.row_tiles;
  k.least = p.least;
  k.whole = p.whole;
  k.two = p.two;
  k.units = c.H >> p.two;
  k.part_o = static_cast<float*>(ws);
  k.part_ml = reinterpret_cast<float2*>(static_cast<char*>(ws) + p.part_o_bytes);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (p.mt == 2)   // heads of 64 only
    return c.dtype == CAST_F8E4M3 ? launch_rows<64, true, 2>(k, p, st) : launch_rows<64, false, 2>(k, p, st);
  if (c.dtype == CAST_F8E4M3)
    return c.d == 128 ? launch_rows<128, true, 1>(k, p, st) : launch_rows<64, true, 1>(k, p, st);
  return c.d == 128 ? launch_rows<128, false, 1>(k, p, st) : launch_rows<64, false, 1>(k, p, st);
}

}  // extern "C"
