// Attention over 4-bit pages for few rows a sequence (single tokens, drafts): k_cache_rows4.  Units, shares of the
// work and the joining are those of k_cache_rows (cache_attention.cu); inside a CTA each warp works on its own blocks
// of 64 tokens with its own running maximum, sum and o in registers.
//
// The codes become f16 in registers (a conversion and a product with the scale for two, both exact), so the issue of
// instructions is what bounds the kernel beside memory, and everything follows from it:
// - Tokens are the products' first operand: S^T = K Q^T and o^T += V^T P^T as m16n8k16, 16 tokens (channels) by 8 rows,
//   half of the products and of the exponentials that 16 rows would take.  P^T comes from S^T by a transposition of
//   8x8 tiles of f16 (movmatrix).
// - The channels' order inside S's sum is free: a lane takes a quarter of a token's row, one or two scales, as one
//   load.  So is the order of o's channels: a lane has D / 8 of them, one scale, for all of its tokens.  The order of
//   tokens inside the products is chosen so that these loads meet few bank conflicts (token_of).
// - V's products want two tokens of one channel side by side: the halves of two words are exchanged while they are
//   codes (six instructions for 16 values).
// A query is f16 times a power of two (its largest channel below 2^15), a probability f16 lifted by 2^7.
//
// Hidden tokens of a block that the rows do not all see: logits become -inf; their V scales, the only thing that can
// make a value not finite, become 0, and tokens whose scales are not finite are added one by one where they are seen.
// A page out of range is scales of 0.
//
// Bound: memory, and issue (530 instructions for 32 tokens, of which the conversions are 128 and the products with the
// scales 128).  Measured, GB300: 24 sequences of 8k to 32k tokens, 8 KV heads of 128, 4 query heads each (626 MB) 111 us,
// 5.6 TB/s; 48 sequences with windows of 4096 on pages of 16 (234 MB) 59 us, of which 20 are first loads, ends of units and
// the joining; one sequence of 301 tokens 7 us.
#include <cmath>

#include "cache.cuh"
#include "cache_attention.cuh"
#include "cache_rows.cuh"
#include "ptx.cuh"

namespace cast {
namespace {

constexpr int BT = 64, SUB = BT / 16;   // tokens of a block: four products' sixteen

// NT: units of 8 NT rows
template <int D, int NT>
struct Cfg4 {
  static constexpr int ROWS = 8 * NT;
  static constexpr int ROWB = D / 2, SROWB = D / 16;      // bytes of a token's codes and scales
  static constexpr int BLOCK = BT * ROWB, SBLOCK = BT * SROWB;
  static constexpr int STAGE = 2 * (BLOCK + SBLOCK);      // codes of K, of V, scales of K, of V
  // Fewer CTAs and larger blocks: what a block costs besides its products is a third of the instructions at 32 tokens
  // (24 sequences of 8k to 32k tokens, heads of 128, 32 tokens and four CTAs 130 us, 64 and three 115, and two 126;
  // heads of 64 85 and 77; 9 rows a KV head 170 and 163, of 64 114 and 100)
  static constexpr int CTAS = D == 128 ? (NT == 1 ? 3 : 2) : (NT == 1 ? 4 : 3);   // of an SM
  // 16 rows: their queries in shared memory, which leaves the registers to the loop (at 32 tokens 176 -> 169 us, heads of
  // 64 120 -> 112); with 8 rows there are enough (130 -> 134)
  static constexpr bool QS = NT > 1;
  static constexpr int STAGES = D == 128 ? 2 : 3;   // of a warp's ring (16 rows: one more would fit; not measured)
  static constexpr int RING = STAGES * STAGE;
  static constexpr int MERGE = kWarps * ROWS * (D + 2) * 4;
  static constexpr int OFF_Q = kWarps * RING > MERGE ? kWarps * RING : MERGE;
  static constexpr int SMEM = OFF_Q + (QS ? NT * (D / 16) * 32 * 8 : 0);
  static_assert((SMEM + 1024 + 256) * CTAS <= 228 * 1024, "CTAs of an SM");
};

// The block's token that lane group g's row of a product is (and token + 8 that row g + 8 is): token 4 j + (q ^ j) for
// row 2 q + j, so that neither the eight lanes that load K together nor those of V meet more than two to a bank.
__device__ __forceinline__ int token_of(int row) { return 4 * (row & 1) + ((row >> 1) ^ (row & 1)); }

__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// SMALL: a block has several pages; else it lies in one
template <int D, int NT, bool SMALL>
__global__ void __launch_bounds__(kWarps * 32, Cfg4<D, NT>::CTAS) k_cache_rows4(const __grid_constant__ RowsKArgs a) {
  using C = Cfg4<D, NT>;
  constexpr int KW = D / 32;   // words of a lane's part of a K row; a V row's part has D / 64
  constexpr int VW = D / 64;
  extern __shared__ __align__(128) uint8_t smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = lane >> 2, q4 = lane & 3;
  int entry;
  int64_t at, stop, entry_at;
  int share;
  // the joining may be put in place as CTAs leave (it waits for all of them)
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  // until the share is known no cut: the workspace may hold an earlier call's
  if (!a.whole && threadIdx.x == 0) a.cuts[blockIdx.x].c0 = -1;
  if (!share_of<D, C::ROWS, BT>(a, entry, at, stop, entry_at, &share)) return;

  uint8_t* ring = smem + warp * C::RING;
  const uint32_t ring_at = smem_u32(ring);
  const int kt0 = token_of(g);                       // this lane's K tokens: kt0 and kt0 + 8
  const int vt0 = q4, vt1 = 4 + (q4 ^ 1);            // ... and V tokens: these, and 8 further on
  const int64_t page_bytes = (int64_t)a.page_size * a.row_stride / 2;
  const uint8_t* kscale = reinterpret_cast<const uint8_t*>(a.k_scale);
  const uint8_t* vscale = reinterpret_cast<const uint8_t*>(a.v_scale);

  for (; at < stop; ++entry) {
    const int b = entry / a.row_tiles, tile = entry % a.row_tiles;
    const Span z = span_of<BT>(a, b, tile, C::ROWS);
    const int nb = z.blocks();
    const int* table = a.batch.page_table + (int64_t)b * a.batch.page_table_stride;
    for (int h = nb ? (int)((at - entry_at) / nb) : a.H; h < a.H && at < stop; ++h) {
      // blocks k0 .. k1-1 of unit (b, tile, h)
      const int64_t unit_at = entry_at + (int64_t)h * nb;
      const int k0 = (int)(at - unit_at);
      const int k1 = (int)min((int64_t)nb, stop - unit_at);
      // (k0 > 0: the share begins inside the unit)
      if (k0 > 0 && threadIdx.x == 0)
        a.cuts[blockIdx.x] = RowsCut{(int)blockIdx.x - (k0 + share - 1) / share, (int)blockIdx.x + (nb - 1 - k0) / share, h, tile, z.t0, z.n_rows};

      // The page of block i (-1: out of range, reads as zeros); small pages: lane group lane / LANES has that of its
      // sixteen tokens (-1 too where no row sees any of them)
      constexpr int LANES = SMALL ? 32 / SUB : 32;
      const int group = lane / LANES;
      auto page_of = [&](int i) {
        const int p = z.block(i) * BT + (SMALL ? 16 * group : 0);
        int page = -1;
        if (!SMALL || (p < z.hi && (p + 16 > z.lo || p < z.sinks))) {
          page = __ldg(table + (p >> a.page_shift));
          if ((unsigned)page >= (unsigned)a.n_pages) {
            if (lane % LANES == 0) left_out();
            page = -1;
          }
        }
        return page;
      };
      // A lane's part of a block: 16 bytes of each 512 of its codes (small pages: of each 128 or 256 of its sixteen's), K's
      // and V's at the same distance, and of the scales: K's, behind them V's
      const int64_t to_v = a.v - a.k, to_vs = vscale - kscale;
      constexpr int SCH = C::SBLOCK / 16, EACH = SCH / SUB;   // chunks of K's (V's) scales, and of a sixteen's
      constexpr bool BOTH = SCH == 32;                        // a lane copies a chunk of each
      const uint8_t* my_codes = a.k + (int64_t)h * a.page_size * C::ROWB + lane % LANES * 16;
      const uint8_t* my_scales = (BOTH || lane < SCH ? kscale : vscale) + (int64_t)h * a.page_size * C::SROWB + (lane & (SCH - 1)) * 16;
      const int64_t page_scales = (int64_t)a.H * a.page_size * C::SROWB;
      const int scale_group = (lane & (SCH - 1)) / EACH;
      // fetches block i of the unit into stage st
      auto fetch = [&](int i, int st, int page) {
        const int base = z.block(i) * BT;
        const uint32_t dst = ring_at + st * C::STAGE;
        // (small pages shorter than a block: its sixteens begin at rows 0, 16 or 32 of theirs)
        const int row = (base + (SMALL ? 16 * group : 0)) & (a.page_size - 1);
        constexpr int PART = SMALL ? C::BLOCK / SUB : C::BLOCK;
        if (page >= 0) {
          const uint8_t* from = my_codes + (page * page_bytes + row * C::ROWB);
          const uint32_t to = dst + (SMALL ? group * PART : 0) + lane % LANES * 16;
#pragma unroll
          for (int c = 0; c < PART; c += LANES * 16) {
            copy16(to + c, from + c);
            copy16(to + C::BLOCK + c, from + to_v + c);
          }
        }
        // the scales' page and row: this lane's, or, where a lane has one chunk of K or V, that of the chunk's sixteen
        int s_page = page, s_row = row;
        if constexpr (SMALL && !BOTH) {
          s_page = __shfl_sync(0xffffffffu, page, scale_group * LANES);
          s_row = (base + 16 * scale_group) & (a.page_size - 1);
        }
        const uint8_t* from = my_scales + (max(s_page, 0) * page_scales + (s_row - (SMALL ? 16 * scale_group : 0)) * C::SROWB);
        const uint32_t to = dst + 2 * C::BLOCK + lane * 16;
        if (lane < 2 * SCH) copy16_or_zero(to, from, s_page >= 0);
        if (BOTH) copy16_or_zero(to + C::SBLOCK, from + to_vs, s_page >= 0);
      };
      const int n = k1 - k0 > warp ? (k1 - k0 - warp + kWarps - 1) >> kWarpsLog : 0;   // blocks of this warp
      const int i0 = k0 + warp;
      __syncwarp();
      for (int st = 0; st < C::STAGES - 1; ++st) {
        if (st < n) fetch(i0 + st * kWarps, st, page_of(i0 + st * kWarps));
        copy_commit();
      }
      int next_page = C::STAGES - 1 < n ? page_of(i0 + (C::STAGES - 1) * kWarps) : -1;

      // Q^T fragments: row g of each 8 (product s takes channels (D / 4) q4 + 4 s .. + 3 of lane group q4)
      uint32_t qf[NT][D / 16][2];
      uint2* qs = reinterpret_cast<uint2*>(smem + C::OFF_Q) + lane;   // [NT][D / 16][lane]
      float unit[NT][2];   // what the logits of rows 2 q4 and 2 q4 + 1 are multiplied by
      int pos[NT][2];      // their positions
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const int r = tile * C::ROWS + t * 8 + g;
        const bool in = r < z.n_rows;
        const int i = r / a.group;
        const __nv_bfloat16* src =
            a.q + (int64_t)(z.t0 + (in ? i : 0)) * a.q_stride + (h * a.group + (in ? r - i * a.group : 0)) * D + q4 * (D / 4);
        uint32_t top = 0;   // magnitudes order as their bits
#pragma unroll
        for (int s = 0; s < D / 16; s += 2) {
          const uint4 w = __ldg(reinterpret_cast<const uint4*>(src + s * 4));
          qf[t][s][0] = in ? w.x : 0u;
          qf[t][s][1] = in ? w.y : 0u;
          qf[t][s + 1][0] = in ? w.z : 0u;
          qf[t][s + 1][1] = in ? w.w : 0u;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t x = qf[t][s + (e >> 1)][e & 1];
            top = max(top, max(x & 0x7fff0000u, (x << 16) & 0x7fff0000u));
          }
        }
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        // 2^-e with the largest channel in [2^14, 2^15), 2^126 at most; rows that are not finite as they are
        const int e = max((int)(top >> 23) - 127 - 14, -126);
        const bool plain = e > 113;
        // (never infinite: keys of zeros give logits of 0)
        const float down = plain ? 1.f : pow2f(-e), up = fminf(a.scale_log2 * (plain ? 1.f : pow2f(e)), 0x1.fffffep127f);
#pragma unroll
        for (int s = 0; s < D / 16; ++s)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const uint32_t w = qf[t][s][j];
            qf[t][s][j] = pack2h(__uint_as_float(w << 16) * down, __uint_as_float(w & 0xffff0000u) * down);
          }
        if constexpr (C::QS) {
          // the warps' are alike: each leaves some
#pragma unroll
          for (int s = 0; s < D / 16; ++s)
            if ((s & (kWarps - 1)) == warp) qs[(t * (D / 16) + s) * 32] = make_uint2(qf[t][s][0], qf[t][s][1]);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          unit[t][j] = __shfl_sync(0xffffffffu, up, (2 * q4 + j) * 4);
          const int rr = tile * C::ROWS + t * 8 + 2 * q4 + j;
          pos[t][j] = rr < z.n_rows ? z.p0 + rr / a.group : -1;
        }
      }
      if constexpr (C::QS) __syncthreads();
      // positions that every row sees: [all_lo, all_hi); the others' blocks are masked
      int all_lo = 0, all_hi = z.hi;
      {
        const int r1 = min(tile * C::ROWS + C::ROWS, z.n_rows) - 1;
        if (a.causal) all_hi = min(z.hi, max(z.p0 + tile * C::ROWS / a.group + 1, 0));
        if (a.window > 0) all_lo = max(z.p0 + r1 / a.group - a.window + 1, 0);
      }
      auto sees = [&](int p, int r) { return p < z.hi && (!a.causal || p <= r) && (a.window <= 0 || p > r - a.window || p < a.sinks); };

      float o[NT][D / 16][4], m_ref[NT][2], l[NT][2];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[t][i][e] = 0.f;
        m_ref[t][0] = m_ref[t][1] = -INFINITY;
        l[t][0] = l[t][1] = 0.f;
      }

      int st = 0, into = C::STAGES - 1;
      for (int it = 0; it < n; ++it) {
        copy_wait<C::STAGES - 2>();
        __syncwarp();
        // the stage used one block ago takes the block STAGES - 1 ahead
        const int ahead = it + C::STAGES - 1;
        if (ahead < n) fetch(i0 + ahead * kWarps, into, next_page);
        copy_commit();
        if (ahead + 1 < n) next_page = page_of(i0 + (ahead + 1) * kWarps);
        const uint8_t* kt = ring + st * C::STAGE;
        const uint8_t* vt = kt + C::BLOCK;
        const uint8_t* ks = kt + 2 * C::BLOCK;
        const uint8_t* vs = ks + C::SBLOCK;

        // ---- S^T = K Q^T, 16 tokens after 16
        float s[NT][SUB][4];
#pragma unroll
        for (int part = 0; part < SUB; ++part) {
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[t][part][e] = 0.f;
          uint32_t kw[2][KW], sc[2][2];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int token = 16 * part + kt0 + 8 * j;
            const uint8_t* p = kt + token * C::ROWB + q4 * (D / 8);
            if constexpr (D == 128) {
              const uint4 w = *reinterpret_cast<const uint4*>(p);
              kw[j][0] = w.x; kw[j][1] = w.y; kw[j][2] = w.z; kw[j][3] = w.w;
              const uint32_t two = *reinterpret_cast<const uint16_t*>(ks + token * C::SROWB + q4 * 2);
              sc[j][0] = scale4_pair(two);
              sc[j][1] = __byte_perm(two, 0, 0x4141) << 7;
            } else {
              const uint2 w = *reinterpret_cast<const uint2*>(p);
              kw[j][0] = w.x; kw[j][1] = w.y;
              sc[j][0] = scale4_pair(ks[token * C::SROWB + q4]);
            }
          }
#pragma unroll
          for (int w = 0; w < KW; ++w) {
            uint32_t x[4], y[4];
            half8(kw[0][w], x);
            half8(kw[1][w], y);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              x[e] = times2(x[e], sc[0][w / 2]);
              y[e] = times2(y[e], sc[1][w / 2]);
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              const uint32_t f[4] = {x[2 * u], y[2 * u], x[2 * u + 1], y[2 * u + 1]};
#pragma unroll
              for (int t = 0; t < NT; ++t) {
                if constexpr (C::QS) {
                  const uint2 q = qs[(t * (D / 16) + 2 * w + u) * 32];
                  mma16816h(s[t][part], f, q.x, q.y);
                } else {
                  mma16816h(s[t][part], f, qf[t][2 * w + u][0], qf[t][2 * w + u][1]);
                }
              }
            }
          }
        }

        const int base = z.block(i0 + it * kWarps) * BT;
        const bool whole = base + BT <= all_hi && (base >= all_lo || base + BT <= z.sinks);
        if (!whole) {
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int part = 0; part < SUB; ++part)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                s[t][part][e] = sees(base + 16 * part + kt0 + (e & 2 ? 8 : 0), pos[t][e & 1]) ? s[t][part][e] * unit[t][e & 1] : -INFINITY;
        }

        // ---- running maximum; what is left of a logit's factor
        float times[NT][2], top[NT][2];
        bool grows = false;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            times[t][j] = whole ? unit[t][j] : 1.f;
            float x = fmaxf(s[t][0][j], s[t][0][2 + j]);
#pragma unroll
            for (int k = 1; k < SUB; ++k) x = fmaxf(x, fmaxf(s[t][k][j], s[t][k][2 + j]));
            top[t][j] = x * times[t][j];
            grows = grows || top[t][j] > m_ref[t][j] + kRescale;
          }
        if (__any_sync(0xffffffffu, grows)) {
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              float x = top[t][j];
              x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
              x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
              x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
              if (x > m_ref[t][j]) {
                const float f = exp2_fast(m_ref[t][j] - x);
                m_ref[t][j] = x;
                l[t][j] *= f;
#pragma unroll
                for (int i = 0; i < D / 16; ++i) {
                  o[t][i][j] *= f;
                  o[t][i][2 + j] *= f;
                }
              }
            }
        }
        // ---- P^T, 2^kLift times the probabilities; l is the sum of them as they are before the rounding
        uint32_t pf[NT][SUB][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            // a row that has seen nothing yet: exp2(-inf - 0) = 0
            const float ref = kLift - (m_ref[t][j] == -INFINITY ? 0.f : m_ref[t][j]);
#pragma unroll
            for (int part = 0; part < SUB; ++part) {
              s[t][part][j] = exp2_fast(fmaf(s[t][part][j], times[t][j], ref));
              s[t][part][2 + j] = exp2_fast(fmaf(s[t][part][2 + j], times[t][j], ref));
            }
            float sum = s[t][0][j] + s[t][0][2 + j];
#pragma unroll
            for (int k = 1; k < SUB; ++k) sum += s[t][k][j] + s[t][k][2 + j];
            l[t][j] += sum;
          }
#pragma unroll
          for (int part = 0; part < SUB; ++part) {
            pf[t][part][0] = transposed(pack2h(s[t][part][0], s[t][part][1]));
            pf[t][part][1] = transposed(pack2h(s[t][part][2], s[t][part][3]));
          }
        }

        // ---- o^T += V^T P^T
#pragma unroll
        for (int part = 0; part < SUB; ++part) {
          uint32_t vw[4][VW], vc[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int token = 16 * part + (j & 1 ? vt1 : vt0) + (j & 2 ? 8 : 0);
            const uint8_t* p = vt + token * C::ROWB + g * (D / 16);
            if constexpr (D == 128) {
              const uint2 w = *reinterpret_cast<const uint2*>(p);
              vw[j][0] = w.x;
              vw[j][1] = w.y;
              vc[j] = vs[token * C::SROWB + g];
            } else {
              vw[j][0] = *reinterpret_cast<const uint32_t*>(p);
              vc[j] = vs[token * C::SROWB + (g >> 1)];
            }
          }
          bool apart = false;
          if (!whole) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const int p = base + 16 * part + (j & 1 ? vt1 : vt0) + (j & 2 ? 8 : 0);
              if (!(p < z.hi && (p >= z.lo || p < z.sinks))) vc[j] = 0;   // nobody's
              apart |= vc[j] > kScaleTop;
            }
            apart = __any_sync(0xffffffffu, apart);
          }
          if (apart) {
            // tokens one by one, where they are seen: P's column of a token is in the lanes that have it as a K token
#pragma unroll 1
            for (int token = 0; token < 16; ++token) {
              // the lane group whose K token this is: row 2 q + j of token 4 j + (q ^ j)
              const int k = token & 7, from = (2 * ((k & 3) ^ (k >> 2)) + (k >> 2)) * 4 + q4;
              const int p = base + 16 * part + token;
#pragma unroll
              for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                  const float w0 = __shfl_sync(0xffffffffu, s[t][part][j], from), w1 = __shfl_sync(0xffffffffu, s[t][part][2 + j], from);
                  if (!sees(p, pos[t][j])) continue;
                  const float w = token < 8 ? w0 : w1;
                  const uint32_t scale = vs[(16 * part + token) * C::SROWB + (D == 128 ? g : g >> 1)];
#pragma unroll
                  for (int i = 0; i < D / 16; ++i) {
                    const uint32_t two = vt[(16 * part + token) * C::ROWB + g * (D / 16) + i];
                    o[t][i][j] += w * value4(two, scale);
                    o[t][i][2 + j] += w * value4(two >> 4, scale);
                  }
                }
            }
          } else {
            const uint32_t s0 = scale4_pair(vc[0], vc[1]), s1 = scale4_pair(vc[2], vc[3]);
#pragma unroll
            for (int w = 0; w < VW; ++w) {
              constexpr uint32_t low = 0x0f0f0f0fu;
              // bytes of two tokens' codes of one channel: channels 0 2 4 6, and 1 3 5 7, of the word's eight
              uint32_t x[4], y[4], u[4], v[4];
              half8((vw[0][w] & low) | ((vw[1][w] << 4) & ~low), x);
              half8(((vw[0][w] >> 4) & low) | (vw[1][w] & ~low), y);
              half8((vw[2][w] & low) | ((vw[3][w] << 4) & ~low), u);
              half8(((vw[2][w] >> 4) & low) | (vw[3][w] & ~low), v);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const uint32_t f[4] = {times2(x[e], s0), times2(y[e], s0), times2(u[e], s1), times2(v[e], s1)};
#pragma unroll
                for (int t = 0; t < NT; ++t) mma16816h(o[t][4 * w + e], f, pf[t][part][0], pf[t][part][1]);
              }
            }
          }
        }
        __syncwarp();
        into = st;
        st = st + 1 == C::STAGES ? 0 : st + 1;
      }
      copy_wait<0>();
      __syncthreads();   // every warp is done with its ring: the merge takes the space

      float* mo = reinterpret_cast<float*>(smem);                        // [warp][row][D]
      float2* ml = reinterpret_cast<float2*>(mo + kWarps * C::ROWS * D); // [warp][row]
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          float x = l[t][j];
          x += __shfl_xor_sync(0xffffffffu, x, 4);
          x += __shfl_xor_sync(0xffffffffu, x, 8);
          x += __shfl_xor_sync(0xffffffffu, x, 16);
          const int r = t * 8 + 2 * q4 + j;
          if (g == 0) ml[warp * C::ROWS + r] = make_float2(m_ref[t][j], x * 0x1p-7f);
          float* dst = mo + (warp * C::ROWS + r) * D + g * (D / 8);
#pragma unroll
          for (int i = 0; i < D / 16; i += 2)
            *reinterpret_cast<float4*>(dst + 2 * i) = make_float4(o[t][i][j] * 0x1p-7f, o[t][i][2 + j] * 0x1p-7f,
                                                                  o[t][i + 1][j] * 0x1p-7f, o[t][i + 1][2 + j] * 0x1p-7f);
        }
      __syncthreads();
      // a share that begins inside the unit leaves its part in the CTA's first place
      join_warps<D, C::ROWS>(a, z, h, tile, k0 == 0 && k1 == nb, 2 * blockIdx.x + (k0 > 0 ? 0 : 1), mo, ml);
      __syncthreads();   // the space goes back to the rings
      at = unit_at + k1;
    }
    entry_at += (int64_t)nb * a.H;
  }
}

template <int D, int NT, bool SMALL>
cast_status launch_pages(const RowsKArgs& k, const RowsPlan& p, cudaStream_t st) {
  using C = Cfg4<D, NT>;
  static std::atomic<uint64_t> attr_done{0};
  if (!once_per_device(attr_done, [&] {
        return cudaFuncSetAttribute(k_cache_rows4<D, NT, SMALL>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM) == cudaSuccess;
      }))
    return check_launch("cache attention smem attribute");
  k_cache_rows4<D, NT, SMALL><<<p.grid, kWarps * 32, C::SMEM, st>>>(k);
  cast_status s = check_launch("cache attention");
  if (s || p.whole) return s;
  if (p.grid < 2) return CAST_OK;
  // two rows a CTA of the joining where units have 16 parts or more on average
  const int64_t units = (int64_t)k.batch.B * k.row_tiles * k.H;
  return launch_joining(k_cuts_merge<D, C::ROWS>, p.grid - 1, p.grid >= 16 * units ? C::ROWS / 2 : 1, st, k);
}

template <int D, int NT>
cast_status launch(const RowsKArgs& k, const RowsPlan& p, cudaStream_t st) {
  return k.page_size < BT ? launch_pages<D, NT, true>(k, p, st) : launch_pages<D, NT, false>(k, p, st);
}

}  // namespace

int rows4_ctas(int d, int mt) {
  if (d == 128) return mt == 1 ? Cfg4<128, 1>::CTAS : Cfg4<128, 2>::CTAS;
  return mt == 1 ? Cfg4<64, 1>::CTAS : Cfg4<64, 2>::CTAS;
}

cast_status launch_rows4(const RowsKArgs& k, const RowsPlan& p, int d, cudaStream_t st) {
  if (d == 128) return p.mt == 1 ? launch<128, 1>(k, p, st) : launch<128, 2>(k, p, st);
  return p.mt == 1 ? launch<64, 1>(k, p, st) : launch<64, 2>(k, p, st);
}

unsigned int cache_rows4_error_word(cudaStream_t st, bool clear) { return read_left_out(st, clear); }

}  // namespace cast
