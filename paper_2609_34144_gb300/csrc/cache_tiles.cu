// Attention over the paged KV cache for many rows a sequence (chunks of frames, prompts) on the
// tensor cores' tcgen05 form.
//
// Rows of one KV head are (token, query head of the group) pairs, G of them a token: a tile of 128
// rows holds 128 / G whole tokens, a unit two consecutive tiles (Q0, Q1) of one sequence, so that each
// K/V tile of 128 positions fetched feeds 256 rows.  The positions a unit's rows can see are a list
// of tiles (the sinks', then the window's).  All units' lists in a row are the work of the call: one CTA
// an SM takes an equal share of it, found from the lengths on the device, and walks through the units it
// touches.  A unit that no CTA had whole leaves parts (unnormalised o, maxima and sums), which
// k_tiles_merge joins.  Short lists (8 tiles) are not cut: a CTA has one unit.
//
// Roles (one CTA an SM): warp 0 fetches Q and the K pages, warp 2 the V pages (TMA boxes of one page x
// 64 channels into a two-stage ring of 128-byte-swizzled tiles; a page that no row sees or that is
// out of range is fetched from beyond the cache's end, which reads as zeros), warp 1 issues the
// products in the order S0 S1 | PV0 S0' PV1 S1' | ..., and two warpgroups hold one query row a thread:
// S from TMEM, mask, running maximum (renewed when a logit exceeds it by 2^8) and sum, P as bf16 back
// to TMEM, where the P V product reads it (bf16 as V is: the two operands of a product have one type, and P in
// two pieces would be a second product where products bound; the sum is of the unrounded P.  The error is 1.4
// times that of the output's rounding alone).  The products of one thread complete in order, so a
// thread that has S of tile j may change o, which holds tiles 0 .. j-1, before it hands over P.
//
// 0 times a value that is not finite is not 0: rows of V that no row of the unit sees are zeroed in
// shared memory (warp 3), and in tiles that the rows do not all see alike a V row holding NaN or
// infinity is zeroed too and its token added by the rows that do see it, one by one.
//
// 8-bit pages: K is multiplied as it lies, in the 8-bit form of the products.  A bf16 query is the sum of
// two e4m3 numbers, exactly: times the power of two that brings its row's largest channel to 448 at
// most, its first four bits and the rest are one each (channels 2^10 below the largest keep 2^-19 of
// it).  So S is the sum of two products at twice the rate, and each page's scale multiplies its columns
// of S.  V codes become f16 tiles (one conversion for two, by a fourth warpgroup, with the zeroing on the
// way) and P is f16: a row's o is kept in units of the largest V scale that it has seen so far over 2^7, and a
// page's probabilities carry its scale in those units in their exponent.  f16 ends at 2^-25: of a token that
// loses 2^-32 of what its codes would be at that scale, at most.
//
// A unit of one tile (few rows, or a sequence's odd last tile) gives even key tiles to one softmax
// warpgroup and odd ones to the other, each with its own S, o, maximum and sum, so that the products of one
// overlap the softmax of the other; the two are joined at the end.
//
// Bound: products and exponentials, about 1 us each of the 1.6 us (8 bits: 1.9 us) that a key tile of two query
// tiles takes; with one query tile of few rows the products of 128 rows (1 us a key tile, of which memory
// needs 0.73 us).  A CTA's first key tile is done 7 to 10 us after its start.  Measured, GB300: 3520 rows of 24
// heads of 128 over 28160 positions, bf16 807 us, 1508 TFLOP/s, 8 bits 912 us, 1335 TFLOP/s; 1560 rows of 12 heads
// over 12480 of 24960 positions, bf16 108 us; 4 sequences of 35 rows and 60011 positions, 4 heads, 8 bits (246 MB)
// 76 us.  Registers (control, softmax, decoding warps): the splits that fit and differ by one step are 0.4 to
// 1 % slower.
#include <cmath>
#include <type_traits>

#include "cache.cuh"
#include "cache_attention.cuh"
#include "ptx.cuh"

namespace cast {
namespace {

__device__ unsigned int g_tiles_error;

constexpr int BM = 128, BN = 128, kStages = 2;
// 8-bit pages: probabilities, at most 2^8 times a row's largest, are lifted by 2^7 to use f16's range
constexpr float kLift = 7.f;
constexpr int kTmemCols = 512;   // S0/P0 at 0, S1/P1 at 128, O0 at 256, O1 at 384

template <int HD, bool F8>
struct Cfg {
  static constexpr int THREADS = F8 ? 512 : 384;
  // registers a thread at launch, and after the hand-over: control warps, softmax, decoders
  static constexpr int LAUNCH = F8 ? 128 : 168;
  static constexpr int REGS_CTL = F8 ? 72 : 96;
  static constexpr int REGS_SOFTMAX = F8 ? 184 : 200;
  static constexpr int REGS_DECODE = 72;
  static_assert(128 * REGS_CTL + 256 * REGS_SOFTMAX + (F8 ? 128 * REGS_DECODE : 0) <= THREADS * LAUNCH,
                "register split exceeds the launch allocation");
  static constexpr int Q_BYTES = BM * HD * 2;               // 8 bits: two pieces of BM * HD
  static constexpr int K_BYTES = BN * HD * (F8 ? 1 : 2);
  static constexpr int V_BYTES = BN * HD * 2;
  static constexpr int RAW_BYTES = F8 ? BN * HD : 0;
  static constexpr int K_STAGES = F8 ? 4 : 2;   // 4 against 2: 8 bits, 35 rows 82 -> 79 us, frames of 3520 tokens 929 -> 924 us
  static constexpr int OFF_Q = 0;
  static constexpr int OFF_K = OFF_Q + 2 * Q_BYTES;
  static constexpr int OFF_V = OFF_K + K_STAGES * K_BYTES;
  static constexpr int OFF_RAW = OFF_V + kStages * V_BYTES;   // V codes
  static constexpr int OFF_BAR = OFF_RAW + kStages * RAW_BYTES;
  static_assert(kStages * V_BYTES >= BM * HD * 4, "o of one warpgroup passes through the V tiles");
  static constexpr int SMEM = OFF_BAR + 1664 + 1024;
  static_assert(SMEM <= 232448, "shared memory of a CTA");
};

struct TilesKArgs {
  cast_cache_batch batch;
  int n_pages, page_size, page_shift, H, H_q, group, tile_tokens;   // tile_tokens = 128 / group
  int causal, window, sinks, o_f32;
  int64_t row_stride;
  const uint8_t* v;
  const float *k_scale, *v_scale;
  void* o;
  float* lse;
  float scale_log2;
  int pairs;         // pairs of tiles that a head may have
  int most_pairs;    // of a sequence
  int whole;         // a CTA has one whole unit
  int least;         // work that a CTA takes at least
  float4* part_o;    // [2 * grid][HD / 4][256]
  float2* part_ml;   // [2 * grid][256]
  struct Cut* cuts;  // [grid]
  unsigned long long wait_ns;
};

// One unit, tokens i0 .. of sequence b, KV head h, and a CTA's part of it
struct Unit {
  int b, h, t0, i0, n_new, p0;
  int k0, n_tiles;          // its key tiles k0 .. k0 + n_tiles - 1
  int work;                 // its work (see unit_work)
  int slot;                 // where the part's result goes; -1: the part is the whole unit
  int lo, hi, sinks;        // positions that some row sees: below sinks, or lo .. hi-1
  int lo_all, hi_all;       // ... that every row sees: lo_all .. hi_all-1 (or below sinks)
  int n_sink, first, tiles; // tiles of 128 positions: 0 .. n_sink-1, then first ..
  int valid;
};
// What CTA c leaves for the joining: the unit that its share begins inside of, which CTAs c0 .. c1 have
// tiles of (c0 = -1: it begins with a unit)
struct Cut {
  int h, t0, i0, n_new, c0, c1;
};
// position of the first key of tile j of the unit's list
__device__ __forceinline__ int tile_pos(const Unit& u, int j) {
  return (j < u.n_sink ? j : u.first + (j - u.n_sink)) * BN;
}
__device__ __forceinline__ bool all_see(const Unit& u, int pos) {
  return pos + BN <= u.hi_all && (pos >= u.lo_all || pos + BN <= u.sinks);
}
__device__ __forceinline__ bool some_see(const Unit& u, int p) { return p < u.hi && (p >= u.lo || p < u.sinks); }

// The positions that unit u.i0 of sequence `s` sees
__device__ __forceinline__ void place_unit(const TilesKArgs& a, Unit& u, const Sequence& s) {
  u.t0 = s.t0;
  u.n_new = min(s.n_new, a.batch.max_new);
  u.p0 = s.len - s.n_new;
  const int64_t room = (int64_t)a.batch.max_pages * a.page_size;
  if (s.len > room || s.n_new > a.batch.max_new) left_out();
  const int len = (int)min((int64_t)s.len, room);
  const int i1 = min(u.i0 + 2 * a.tile_tokens, u.n_new) - 1;
  u.hi = a.causal ? min(len, max(u.p0 + i1 + 1, 0)) : len;
  u.hi_all = a.causal ? min(len, max(u.p0 + u.i0 + 1, 0)) : len;
  u.lo = u.lo_all = u.sinks = 0;
  if (a.window > 0) {
    u.lo = min(max(u.p0 + u.i0 - a.window + 1, 0), u.hi);
    u.lo_all = max(u.p0 + i1 - a.window + 1, 0);
    u.sinks = min(min(a.sinks, u.lo), u.hi);
  }
  u.first = u.lo / BN;
  u.n_sink = min((u.sinks + BN - 1) / BN, u.first);
  u.tiles = u.n_sink + max((u.hi + BN - 1) / BN - u.first, 0);
}
// Work, in items of about half a microsecond: a key tile of two query tiles takes 1.6 to 1.9 us, of one query
// tile 1 us, and a CTA that goes over to another unit has the first key tile's softmax done ~10 us later, half of
// which other CTAs' memory traffic gains (kBegin 0, 16 and 24 when it was chosen: decode of 35 rows, 60k
// positions, 8 bits, 85, 81, 83 us; window of 1560 frame tokens 114, 110, 113 us; frames of 3520 tokens 925, 929,
// 930 us).
constexpr int kBegin = 16, kPair = 4, kSingle = 2;
__device__ __forceinline__ int tile_work(const TilesKArgs& a, const Unit& u) {
  return u.i0 + a.tile_tokens < u.n_new ? kPair : kSingle;
}
__device__ __forceinline__ int unit_work(const TilesKArgs& a, const Unit& u) {
  return u.tiles ? kBegin + u.tiles * tile_work(a, u) : 1;
}

// Work of units lane, lane + 32, ... or, `serial`, of all units of sequence b
__device__ __forceinline__ int64_t sequence_work(const TilesKArgs& a, int b, int lane, bool serial) {
  if (b >= a.batch.B) return 0;
  const Sequence s = sequence_of(a.batch, b);
  const int n = min(s.n_new, a.batch.max_new), per = 2 * a.tile_tokens;
  Unit u{};
  int64_t w = 0;
  for (u.i0 = serial ? 0 : lane * per; u.i0 < n; u.i0 += serial ? per : 32 * per) {
    place_unit(a, u, s);
    w += unit_work(a, u);
  }
  return w;
}
// Lane l's answer is the work of sequence b0 + l: one sequence a lane, or, where there are fewer of them
// than units in one, one after the other by all lanes
__device__ __forceinline__ int64_t chunk_work(const TilesKArgs& a, int b0, int lane) {
  if (a.batch.B >= a.most_pairs) return sequence_work(a, b0 + lane, 0, true);
  int64_t mine = 0;
  for (int b = b0; b < min(b0 + 32, a.batch.B); ++b) {
    const int64_t w = warp_sum(sequence_work(a, b, lane, false));
    if (b0 + lane == b) mine = w;
  }
  return mine;
}
template <class T>
__device__ __forceinline__ T scan(T x, int lane) {   // inclusive
  for (int o = 1; o < 32; o <<= 1) {
    const T y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  return x;
}
// How the call's work is dealt out.  Units of equal work are first dealt whole, a round of one for each
// CTA (heads slowest: what runs together reads one head's keys); what is left, or everything where units
// differ, is a row of work items from `base` on, of which CTA c has share * c .. share * (c + 1) - 1.
struct Deal {
  int64_t per_head;      // work of a head
  int each, rounds;      // of a unit that is dealt whole, and how many a CTA has
  int64_t base, share, total;
};
__device__ __forceinline__ Deal deal(const TilesKArgs& a, int ctas, int lane) {   // one warp; every lane has it
  Deal d{};
  if (a.batch.B == 1) {
    const Sequence s = sequence_of(a.batch, 0);
    const int n = min(s.n_new, a.batch.max_new), per = 2 * a.tile_tokens;
    Unit u{};
    int low = 0x7fffffff, high = 0;
    for (u.i0 = lane * per; u.i0 < n; u.i0 += 32 * per) {
      place_unit(a, u, s);
      const int w = unit_work(a, u);
      d.per_head += w;
      low = min(low, w);
      high = max(high, w);
    }
    d.per_head = warp_sum(d.per_head);
    low = __reduce_min_sync(0xffffffffu, low);
    high = __reduce_max_sync(0xffffffffu, high);
    d.total = d.per_head * a.H;
    if (low == high) {
      d.each = high;
      d.rounds = (int)(d.total / high / ctas);
      d.base = (int64_t)d.rounds * ctas * high;
    }
  } else {
    for (int b0 = 0; b0 < a.batch.B; b0 += 32) d.per_head += warp_sum(chunk_work(a, b0, lane));
    d.total = d.per_head * a.H;
  }
  d.share = max((int64_t)a.least, (d.total - d.base + ctas - 1) / ctas);
  return d;
}

// Unit `x` of the call, whole (one warp; every lane has it), heads slowest: those that run together read
// one head's keys.
__device__ __forceinline__ Unit unit_of(const TilesKArgs& a, int x, int lane) {
  Unit u{};
  u.h = x / a.pairs;
  int pair = x - u.h * a.pairs;
  const int per = 2 * a.tile_tokens;
  for (int b0 = 0; b0 < a.batch.B; b0 += 32) {
    const int b = b0 + lane;
    const int n = b < a.batch.B ? (min(sequence_of(a.batch, b).n_new, a.batch.max_new) + per - 1) / per : 0;
    const int sum = scan(n, lane);
    const unsigned hit = __ballot_sync(0xffffffffu, sum > pair);
    if (hit) {
      const int l = __ffs(hit) - 1;
      u.b = b0 + l;
      u.i0 = (pair - __shfl_sync(0xffffffffu, sum - n, l)) * per;
      u.valid = 1;
      break;
    }
    pair -= __shfl_sync(0xffffffffu, sum, 31);
  }
  if (!u.valid) return u;
  place_unit(a, u, sequence_of(a.batch, u.b));
  u.n_tiles = u.tiles;
  u.work = unit_work(a, u);
  u.slot = -1;
  return u;
}

// The first unit of which items at .. stop-1 have a tile, and that part of it (one warp; every lane has it).  A
// unit's tile k is at item kBegin + k * tile_work.  Its first part (with tile 0) goes to the CTA's second
// place, others to its first.
__device__ __forceinline__ Unit unit_at(const TilesKArgs& a, const Deal& d, int64_t at, int64_t stop, int lane, Cut* cut) {
  Unit u{};
  if (cut && lane == 0) cut->c0 = -1;
  const int64_t from = at;
  const int per = 2 * a.tile_tokens;
  while (at < stop) {
    const int h = (int)(at / d.per_head);
    int64_t r = at - h * d.per_head;
    int b = a.batch.B == 1 ? 0 : -1;
    for (int b0 = 0; b < 0 && b0 < a.batch.B; b0 += 32) {
      const int64_t w = chunk_work(a, b0, lane);
      const int64_t sum = scan(w, lane);
      const unsigned hit = __ballot_sync(0xffffffffu, sum > r);
      if (hit) {
        const int l = __ffs(hit) - 1;
        r -= __shfl_sync(0xffffffffu, sum - w, l);
        b = b0 + l;
      } else {
        r -= __shfl_sync(0xffffffffu, sum, 31);
      }
    }
    if (b < 0) return u;
    const Sequence s = sequence_of(a.batch, b);
    const int n = min(s.n_new, a.batch.max_new);
    bool found = false;
    for (int i0 = 0; i0 < n; i0 += 32 * per) {
      u.i0 = i0 + lane * per;
      int w = 0;
      if (u.i0 < n) {
        place_unit(a, u, s);
        w = unit_work(a, u);
      }
      const int64_t sum = scan((int64_t)w, lane);
      const unsigned hit = __ballot_sync(0xffffffffu, sum > r);
      if (hit) {
        const int l = __ffs(hit) - 1;
        r -= __shfl_sync(0xffffffffu, sum - w, l);
        u.i0 = i0 + l * per;
        found = true;
        break;
      }
      r -= __shfl_sync(0xffffffffu, sum, 31);
    }
    if (!found) return u;
    u.b = b;
    u.h = h;
    place_unit(a, u, s);
    const int in = (int)r;   // items of the unit before `at`
    const int w = unit_work(a, u), each = tile_work(a, u), some = (int)min((int64_t)(w - in), stop - at);
    u.k0 = (max(in - kBegin, 0) + each - 1) / each;
    u.n_tiles = u.tiles ? (max(in + some - kBegin, 0) + each - 1) / each - u.k0 : 0;
    if (u.n_tiles > 0 || u.tiles == 0) {
      u.valid = 1;
      u.work = (int)(at - from) + some;
      u.slot = u.n_tiles == u.tiles ? -1 : 2 * (int)blockIdx.x + (u.k0 > 0 ? 0 : 1);
      if (cut && lane == 0 && u.k0 > 0) {
        const int64_t first = at - r - d.base + kBegin;   // of tile 0
        *cut = Cut{u.h, u.t0, u.i0, u.n_new, (int)(first / d.share), (int)((first + (u.tiles - 1) * each) / d.share)};
      }
      break;
    }
    at += some;
  }
  return u;
}

struct Bars {
  uint64_t q_full, q_raw;              // q_raw: 8-bit pages, the queries as they are, in the V tiles' place
  uint64_t k_full[4], k_empty[4], v_full[kStages], v_empty[kStages];
  uint64_t s_full[2], p_full[2];
  // bf16 pages: V of a stage's tile that not all rows see is ready.  One phase for each such tile of
  // the stage; the next cannot begin before the products, and so the softmax threads, are past this one.
  uint64_t v_fixed[kStages];
  uint64_t raw_full[4], raw_empty[4];   // 8-bit pages: V codes
  uint64_t fin;
  uint32_t tmem_base;
  int abort;
  int issued[2];                       // of a CTA that gave up: key tiles whose K (V) copies have begun, else many
  uint32_t apart[kStages][4];          // V rows of a stage's tile that are added one by one
  float2 ml[BM];                       // maximum and sum of the second warpgroup's rows
  Unit unit, next;                     // of this segment and the next
};
static_assert(sizeof(Bars) <= 1664, "barriers and the unit");

__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
template <bool F8>
__device__ __forceinline__ void init_barriers(Bars* bars) {
  mbar_init(&bars->q_full, F8 ? 256 : 1);
  mbar_init(&bars->q_raw, 1);
  for (int s = 0; s < 4; ++s) {
    mbar_init(&bars->k_full[s], 1);
    mbar_init(&bars->k_empty[s], 1);
    mbar_init(&bars->raw_full[s], 1);
    mbar_init(&bars->raw_empty[s], 128);
  }
  for (int s = 0; s < kStages; ++s) {
    mbar_init(&bars->v_full[s], F8 ? 128 : 1);
    mbar_init(&bars->v_empty[s], F8 ? 1 : 2);   // the products, and warp 3 that saw the tile
    mbar_init(&bars->v_fixed[s], 32);
  }
  for (int t = 0; t < 2; ++t) {
    mbar_init(&bars->s_full[t], 1);
    mbar_init(&bars->p_full[t], 128);
  }
  mbar_init(&bars->fin, 1);
  fence_barrier_init();
}
__device__ __forceinline__ void drop(uint64_t* bar) {
  asm volatile("mbarrier.inval.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void drop_barriers(Bars* bars) {
  drop(&bars->q_full);
  drop(&bars->q_raw);
  for (int s = 0; s < 4; ++s) {
    drop(&bars->k_full[s]);
    drop(&bars->k_empty[s]);
    drop(&bars->raw_full[s]);
    drop(&bars->raw_empty[s]);
  }
  for (int s = 0; s < kStages; ++s) {
    drop(&bars->v_full[s]);
    drop(&bars->v_empty[s]);
    drop(&bars->v_fixed[s]);
  }
  for (int t = 0; t < 2; ++t) {
    drop(&bars->s_full[t]);
    drop(&bars->p_full[t]);
  }
  drop(&bars->fin);
}
template <int N>
__device__ __forceinline__ void end_barrier() {
  asm volatile("barrier.sync 1, %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ bool aborted(const Bars* b) {
  return *reinterpret_cast<const volatile int*>(&b->abort) != 0;
}
__device__ __forceinline__ void set_abort(Bars* b) {
  atomicExch(&b->abort, 1);
  atomicExch(&g_tiles_error, 1u);
}
__device__ __forceinline__ uint64_t join(uint32_t low, uint32_t high) {
  uint64_t x;
  asm volatile("mov.b64 %0, {%1, %2};" : "=l"(x) : "r"(low), "r"(high));
  return x;
}
__device__ __forceinline__ uint32_t tmem_ld_1(uint32_t taddr) {
  uint32_t r;
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];\n\ttcgen05.wait::ld.sync.aligned;"
               : "=r"(r) : "r"(taddr) : "memory");
  return r;
}

// The page that holds position `p` of the unit's sequence, or n_pages (which reads as zeros) where no
// row of the unit sees any of it or it is out of range.
__device__ __forceinline__ int page_at(const TilesKArgs& a, const Unit& u, int p) {
  if (!(p < u.hi && (p < u.sinks || p + a.page_size > u.lo))) return a.n_pages;
  const int page = __ldg(a.batch.page_table + (int64_t)u.b * a.batch.page_table_stride + (p >> a.page_shift));
  if (page >= 0 && page < a.n_pages) return page;
  left_out();
  return a.n_pages;
}

// Fetches the pages of a K or V tile at `pos` (one warp; lane i < 128 / page_size has page i).  ROWB: bytes
// of a row; CODES: the tile is 8-bit.
template <int ROWB, bool CODES>
__device__ __forceinline__ void fetch_pages(const TilesKArgs& a, const Unit& u, const CUtensorMap* map, uint8_t* dst,
                                            uint64_t* full, int pos, int lane) {
  const int n = BN >> a.page_shift;
  const int page = lane < n ? page_at(a, u, pos + (lane << a.page_shift)) : 0;
  __syncwarp();
  if (lane == 0) mbar_arrive_expect_tx(full, BN * ROWB);
  __syncwarp();
  if (lane < n) {
    if (CODES) {
      tma_load_3d(dst + (lane << a.page_shift) * ROWB, map, full, u.h * ROWB, 0, page);
    } else {
#pragma unroll
      for (int b = 0; b < ROWB / 128; ++b)
        tma_load_3d(dst + b * BN * 128 + (lane << a.page_shift) * 128, map, full, u.h * (ROWB / 2) + b * 64, 0, page);
    }
  }
}

template <int HD, bool F8>
__global__ void __launch_bounds__(F8 ? 512 : 384, 1)
    k_cache_tiles(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                  const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ TilesKArgs a) {
  using C = Cfg<HD, F8>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  uint8_t* smem = smem_raw + (((raw + 1023u) & ~1023u) - raw);
  uint8_t* sQ = smem + C::OFF_Q;
  uint8_t* sK = smem + C::OFF_K;
  uint8_t* sV = smem + C::OFF_V;
  uint8_t* sRaw = smem + C::OFF_RAW;
  Bars* bars = reinterpret_cast<Bars*>(smem + C::OFF_BAR);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // V codes: two stages, and two more in the place of a second query tile that a unit does not have
  auto raw_stage = [&](int s) { return s < 2 ? sRaw + s * C::RAW_BYTES : sQ + C::Q_BYTES + (s - 2) * C::RAW_BYTES; };

  if (warp == 2 && lane == 0) {
    tma_prefetch_desc(&tm_q);
    tma_prefetch_desc(&tm_k);
    tma_prefetch_desc(&tm_v);
  }
  // warp 0: the CTA's share of the work, and its first unit
  Deal d{};
  int64_t at = 0, stop = 0;
  int round = 0;
  if (warp == 0) {
    Unit u;
    if (a.whole) {
      u = unit_of(a, blockIdx.x, lane);
    } else {
      d = deal(a, gridDim.x, lane);
      // whole units come first: should the CTA give up before its share, the joining must find no cut that the
      // workspace held before
      if (d.rounds > 0 && lane == 0) a.cuts[blockIdx.x].c0 = -1;
      at = d.rounds > 0 ? (int64_t)blockIdx.x * d.each : blockIdx.x * d.share;
      stop = d.rounds > 0 ? at + d.each : min(at + d.share, d.total);
      // with the share comes what it begins inside of, for the joining
      u = unit_at(a, d, at, stop, lane, d.rounds > 0 ? nullptr : a.cuts + blockIdx.x);
    }
    if (lane == 0) bars->unit = u;
  }
  if (warp == 1) {
    tmem_alloc(&bars->tmem_base, kTmemCols);
    tmem_relinquish();
    tc_fence_before();
    if (lane == 0) {
      init_barriers<F8>(bars);
      bars->abort = 0;
      bars->issued[0] = bars->issued[1] = 0x7fffffff;
    }
  }
  __syncthreads();
  tc_fence_after();
  const Unit& u = bars->unit;
  const uint32_t tmem = bars->tmem_base;
  const uint64_t lim = a.wait_ns;
  if (!u.valid) {
    if (warp == 1) tmem_dealloc(tmem, kTmemCols);
    return;
  }

  // Segments: the CTA's parts of units, one after the other.  Between two of them the CTA meets twice, and
  // its barriers begin anew in between.  Unit data is read from shared memory where it is needed.
  auto another = [&] {
    tc_fence_before();
    fence_proxy_async_smem();   // what was staged in the tiles' places, before copies land there again
    end_barrier<C::THREADS>();
    if (threadIdx.x == 32 && !aborted(bars)) {
      drop_barriers(bars);
      init_barriers<F8>(bars);
      bars->unit = bars->next;
    }
    end_barrier<C::THREADS>();
    tc_fence_after();
    return !aborted(bars) && u.valid != 0;
  };

  if (warp < 4) {
    setmaxnreg_dec<C::REGS_CTL>();
    for (;;) {
    const int k0 = u.k0, n_tiles = u.n_tiles;
    const bool has_q1 = u.i0 + a.tile_tokens < u.n_new;   // else the warpgroups share the key tiles
    if (warp == 0 || warp == 2) {
      // ------------------------------------------------------------ Q and K pages / V pages
      const bool is_k = warp == 0;
      const CUtensorMap* map = is_k ? &tm_k : &tm_v;
      if (lane == 0) {
        if (is_k && n_tiles > 0) {
          const uint32_t bytes = (uint32_t)a.tile_tokens * a.group * HD * 2;
          uint64_t* bar = F8 ? &bars->q_raw : &bars->q_full;
          uint8_t* to = F8 ? sV : sQ;
          mbar_arrive_expect_tx(bar, (has_q1 ? 2 : 1) * bytes);
          for (int t = 0; t < (has_q1 ? 2 : 1); ++t)
#pragma unroll
            for (int b = 0; b < HD / 64; ++b)
              tma_load_3d(to + t * C::Q_BYTES + b * BM * 128, &tm_q, bar, b * 64, u.h * a.group,
                          u.t0 + u.i0 + t * a.tile_tokens);
        }
      }
      __syncwarp();
      const bool codes = F8 && !is_k;   // V codes go to the raw ring
      uint64_t* full = is_k ? bars->k_full : codes ? bars->raw_full : bars->v_full;
      uint64_t* empty = is_k ? bars->k_empty : codes ? bars->raw_empty : bars->v_empty;
      uint8_t* dst = is_k ? sK : sV;
      const int bytes = is_k ? C::K_BYTES : codes ? C::RAW_BYTES : C::V_BYTES;
      const int log_stages = is_k ? (C::K_STAGES == 4 ? 2 : 1) : codes && !has_q1 ? 2 : 1;
      for (int j = 0; j < n_tiles; ++j) {
        const int s = j & ((1 << log_stages) - 1);
        bool ok = mbar_wait(&empty[s], ((uint32_t)(j >> log_stages) & 1u) ^ 1u, lim);
        ok = !aborted(bars) && ok;
        if (!__all_sync(0xffffffffu, ok)) {
          if (lane == 0) bars->issued[is_k ? 0 : 1] = j;
          set_abort(bars);
          break;
        }
        uint8_t* to = codes ? raw_stage(s) : dst + s * bytes;
        fetch_pages<HD * (F8 ? 1 : 2), F8>(a, u, map, to, &full[s], tile_pos(u, k0 + j), lane);
      }
      if (is_k) {
        // all keys are under way: the next unit (none where CTAs have one unit: stop = 0)
        at += u.work;
        Cut* cut = nullptr;
        if (at >= stop && round < d.rounds) {
          if (++round == d.rounds) cut = a.cuts + blockIdx.x;
          at = round < d.rounds ? ((int64_t)round * gridDim.x + blockIdx.x) * d.each : d.base + blockIdx.x * d.share;
          stop = round < d.rounds ? at + d.each : min(at + d.share, d.total);
        }
        if (at >= stop) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
        const Unit next = unit_at(a, d, at, stop, lane, cut);
        if (lane == 0) bars->next = next;
      }
    } else if (warp == 3 && !F8) {
      // ------------------------------------------------------------ V of tiles that not all rows see
      // It waits for every tile in turn and gives every stage back, so that it can be neither ahead
      // of a phase nor overtaken.
      for (int j = 0; j < n_tiles; ++j) {
        const int pos = tile_pos(u, k0 + j), s = j % kStages;
        bool ok = mbar_wait(&bars->v_full[s], (uint32_t)(j / kStages) & 1u, lim);
        ok = !aborted(bars) && ok;
        if (!__all_sync(0xffffffffu, ok)) { set_abort(bars); break; }
        if (!all_see(u, pos)) {
          uint8_t* tile = sV + s * C::V_BYTES;
          for (int i = 0; i < 4; ++i) {
            // lane: row 32 i + lane
            const int r = 32 * i + lane;
            const bool some = some_see(u, pos + r);
            bool bad = false;
            if (some) {
#pragma unroll 4
              for (int c = 0; c < HD / 8; ++c) {
                const uint4 w = *reinterpret_cast<const uint4*>(tile + (c / 8) * BN * 128 + r * 128 + ((c ^ r) & 7) * 16);
                bad |= not_finite<false>(w);
              }
            }
            const uint32_t apart = __ballot_sync(0xffffffffu, bad);
            if (lane == 0) bars->apart[s][i] = apart;
            if (bad || !some)
#pragma unroll 4
              for (int c = 0; c < HD / 8; ++c)
                *reinterpret_cast<uint4*>(tile + (c / 8) * BN * 128 + r * 128 + ((c ^ r) & 7) * 16) = make_uint4(0, 0, 0, 0);
          }
          fence_proxy_async_smem();
          mbar_arrive(&bars->v_fixed[s]);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars->v_empty[s]);
      }
    } else if (warp == 1 && lane == 0) {
      // ------------------------------------------------------------ products
      constexpr uint32_t idesc_qk = F8 ? idesc_e4m3_f32(BM, BN) : idesc_bf16_f32(BM, BN, false, false);
      constexpr uint32_t idesc_pv = F8 ? idesc_f16_f32(BM, HD, false, true) : idesc_bf16_f32(BM, HD, false, true);
      // a k-slice, query tile or stage further on adds its byte offset / 16 to the start address
      static_assert(C::SMEM + 1024 <= 256 * 1024, "descriptor start-address field would carry");
      constexpr bool kNarrow = F8 && HD == 64;   // 64-byte rows
      // descriptors as their low words (the start address / 16 and the leading offset); the high ones are
      // the same for a kind of operand
      const uint64_t dq = kNarrow ? sdesc_sw64(smem_u32(sQ), 16, 512) : sdesc_sw128(smem_u32(sQ), 16, 1024);
      const uint64_t dk = kNarrow ? sdesc_sw64(smem_u32(sK), 16, 512) : sdesc_sw128(smem_u32(sK), 16, 1024);
      const uint64_t dv = sdesc_sw128(smem_u32(sV), BN * 128, 1024);
      const uint32_t ql = (uint32_t)dq, kl = (uint32_t)dk, vl = (uint32_t)dv;
      constexpr uint32_t kHigh = kNarrow ? (uint32_t)(512 >> 4) | (1u << 14) | (4u << 29) : (uint32_t)(1024 >> 4) | (1u << 14) | (2u << 29);
      constexpr uint32_t kHighV = (uint32_t)(1024 >> 4) | (1u << 14) | (2u << 29);
      // S_t = Q_q K_j^T
      auto qk = [&](int t, int q, int j) {
        const uint32_t aq = ql + (uint32_t)((q * C::Q_BYTES) >> 4);
        const uint32_t bk = kl + (uint32_t)(((j % C::K_STAGES) * C::K_BYTES) >> 4);
        if constexpr (F8) {
#pragma unroll
          for (int piece = 0; piece < 2; ++piece)
#pragma unroll
            for (int kk = 0; kk < HD / 32; ++kk)
              umma_f8_ss(tmem + t * BN, join(aq + ((piece * BM * HD + kk * 32) >> 4), kHigh), join(bk + ((kk * 32) >> 4), kHigh),
                         idesc_qk, piece + kk > 0 ? 1u : 0u);
        } else {
#pragma unroll
          for (int kk = 0; kk < HD / 16; ++kk) {
            const uint32_t off = ((kk >> 2) * (BM * 128) + (kk & 3) * 32) >> 4;
            umma_bf16_ss(tmem + t * BN, join(aq + off, kHigh), join(bk + off, kHigh), idesc_qk, kk > 0 ? 1u : 0u);
          }
        }
        umma_commit(&bars->s_full[t]);
      };
      // o is zeroed by the softmax threads before the first P, so it always accumulates
      auto pv = [&](int t, int j) {
        const uint32_t bv = vl + (uint32_t)(((j % kStages) * C::V_BYTES) >> 4);
#pragma unroll
        for (int kk = 0; kk < BN / 16; ++kk)
          umma_bf16_ts(tmem + 256 + t * 128, tmem + t * BN + kk * 8, join(bv + ((kk * 16 * 128) >> 4), kHighV), idesc_pv, 1u);
      };
      uint32_t fixed = 0;   // bit s: parity of the next phase of v_fixed[s]
      auto k_ready = [&](int j) { return mbar_wait(&bars->k_full[j % C::K_STAGES], (uint32_t)(j / C::K_STAGES) & 1u, lim); };
      auto v_ready = [&](int j) {
        const int s = j % kStages;
        bool ok = !aborted(bars) && mbar_wait(&bars->v_full[s], (uint32_t)(j / kStages) & 1u, lim);
        if (ok && !F8 && !all_see(u, tile_pos(u, k0 + j))) {
          ok = mbar_wait(&bars->v_fixed[s], (fixed >> s) & 1u, lim);
          fixed ^= 1u << s;
        }
        return ok;
      };
      bool ok = n_tiles == 0 || mbar_wait(&bars->q_full, 0, lim);
      // the warpgroups are spelled out: with a running index the addresses of a product's sixteen steps are
      // computed between them (10 % of the kernel's time)
      auto p_ready = [&](int t, int use) { return !aborted(bars) && mbar_wait(&bars->p_full[t], (uint32_t)use & 1u, lim); };
      static_assert(kStages == 2, "V tile j's stage is j & 1");
      if (has_q1) {
        if (ok && n_tiles > 0) {
          ok = k_ready(0);
          tc_fence_after();
          if (ok) {
            qk(0, 0, 0);
            qk(1, 1, 0);
            umma_commit(&bars->k_empty[0]);
          }
        }
        for (int j = 0; ok && j < n_tiles; ++j) {
          const bool more = j + 1 < n_tiles;
          // K of the next key tile is awaited with V, while P0 is still being formed
          ok = v_ready(j) && (!more || k_ready(j + 1)) && p_ready(0, j);
          if (!ok) break;
          tc_fence_after();
          pv(0, j);
          if (more) qk(0, 0, j + 1);
          ok = p_ready(1, j);
          if (!ok) break;
          tc_fence_after();
          pv(1, j);
          umma_commit(&bars->v_empty[j & 1]);
          if (more) {
            qk(1, 1, j + 1);
            umma_commit(&bars->k_empty[(j + 1) % C::K_STAGES]);
          }
        }
      } else {
        // one query tile: warpgroup t has key tiles t, t + 2, ...
        for (int j = 0; ok && j < min(2, n_tiles); ++j) {
          ok = k_ready(j);
          if (!ok) break;
          tc_fence_after();
          qk(j, 0, j);
          umma_commit(&bars->k_empty[j]);
        }
        auto step = [&](int t, int j) {
          const bool more = j + 2 < n_tiles;
          if (!(v_ready(j) && (!more || k_ready(j + 2)) && p_ready(t, j >> 1))) return false;
          tc_fence_after();
          pv(t, j);
          umma_commit(&bars->v_empty[t]);
          if (more) {
            qk(t, 0, j + 2);
            umma_commit(&bars->k_empty[(j + 2) % C::K_STAGES]);
          }
          return true;
        };
        for (int j = 0; ok && j < n_tiles; j += 2) {
          ok = step(0, j);
          if (ok && j + 1 < n_tiles) ok = step(1, j + 1);
        }
      }
      if (!ok) set_abort(bars);
      umma_commit(&bars->fin);
      mbar_wait(&bars->fin, 0, lim);
    }
    __syncwarp();
    if (!another()) break;
    }
    if ((warp == 0 || warp == 2) && aborted(bars)) {
      // the CTA gave up: none of its copies may land after it has left.  They are the segment's last, of which no
      // stage has begun anew, and its queries.
      const int issued = min(bars->issued[warp == 0 ? 0 : 1], u.n_tiles);
      uint64_t* full = warp == 0 ? bars->k_full : F8 ? bars->raw_full : bars->v_full;
      const int log_stages = warp == 0 ? (C::K_STAGES == 4 ? 2 : 1) : F8 && u.i0 + a.tile_tokens >= u.n_new ? 2 : 1;
#pragma unroll 1
      for (int j = max(issued - (1 << log_stages), 0); j < issued; ++j)
        mbar_wait(&full[j & ((1 << log_stages) - 1)], (uint32_t)(j >> log_stages) & 1u, lim);
      if (warp == 0 && u.n_tiles > 0) mbar_wait(F8 ? &bars->q_raw : &bars->q_full, 0, lim);
    }
    if (warp == 1) tmem_dealloc(tmem, kTmemCols);
  } else if (warp < 12) {
    setmaxnreg_inc<C::REGS_SOFTMAX>();
    for (;;) {
        const int k0 = u.k0, n_tiles = u.n_tiles;
      const bool has_q1 = u.i0 + a.tile_tokens < u.n_new;   // else the warpgroups share the key tiles
      // ------------------------------------------------------------ softmax and result
      const int t = warp < 8 ? 0 : 1;
      const int qt = has_q1 ? t : 0;         // the query tile of this warpgroup
      const int every = has_q1 ? 1 : 2;      // its key tiles: t (or 0), and every so many on
      const int q4 = warp & 3;
      const int row = q4 * 32 + lane;
      const uint32_t tl = tmem + ((uint32_t)(q4 * 32) << 16);
      const uint32_t colS = t * BN, colO = 256 + t * 128;
      // the row's token and query head, and what it sees: below hi, and below sinks or from lo on
      const int tok = row / a.group, i = u.i0 + qt * a.tile_tokens + tok;
      const bool live = tok < a.tile_tokens && i < u.n_new;
      const int p = u.p0 + i;
      const int hi = !live ? 0 : a.causal ? min(u.hi, max(p + 1, 0)) : u.hi;
      const int lo = a.window > 0 ? max(p - a.window + 1, 0) : 0;
      const int sinks = a.window > 0 ? a.sinks : 0;
      float m_ref = -INFINITY, l = 0.f;
      // 8-bit pages: lane c < 8 has the K and V scale of columns 16c .. 16c + 15 of a key tile (one page), fetched
      // one tile ahead, and the page two tiles ahead, so that neither load is waited for
      const int j0 = has_q1 ? 0 : t;
      auto page_of = [&](int j) {
        return lane < BN / 16 && j < n_tiles ? page_at(a, u, (tile_pos(u, k0 + j) + 16 * lane) & -a.page_size) : a.n_pages;
      };
      auto scales_of = [&](int page) {
        float2 x = make_float2(1.f, 0.f);
        if (page < a.n_pages) {
          x.x = __ldg(a.k_scale + (int64_t)page * a.H + u.h);
          x.y = __ldg(a.v_scale + (int64_t)page * a.H + u.h);
        }
        return x;
      };
      float2 next = make_float2(1.f, 0.f);
      int next_page = 0;
      if constexpr (F8) {
        next = scales_of(page_of(j0));
        next_page = page_of(j0 + every);
      }
      float unit = a.scale_log2;   // what the row's S is multiplied by (and, with 8-bit pages, by their scales)
      if constexpr (F8) {
        // the row as two e4m3 pieces of row * 2^-ex; without a second tile both warpgroups have the row
        if (n_tiles > 0 && __any_sync(0xffffffffu, live)) {
          bool w = !aborted(bars) && mbar_wait(&bars->q_raw, 0, lim);
          if (!__all_sync(0xffffffffu, w)) set_abort(bars);
          const uint8_t* src = sV + qt * C::Q_BYTES + row * 128;
          auto eight = [&](int c) {   // channels 8 c .. 8 c + 7
            return live ? *reinterpret_cast<const uint4*>(src + (c / 8) * BM * 128 + ((c ^ row) & 7) * 16) : make_uint4(0, 0, 0, 0);
          };
          uint32_t top = 0;   // magnitudes order as their bits
#pragma unroll 4
          for (int c = 0; c < HD / 8; ++c) {
            const uint4 x = eight(c);
            top = max(top, max(max(x.x & 0x7fff0000u, (x.x << 16) & 0x7fff0000u), max(x.y & 0x7fff0000u, (x.y << 16) & 0x7fff0000u)));
            top = max(top, max(max(x.z & 0x7fff0000u, (x.z << 16) & 0x7fff0000u), max(x.w & 0x7fff0000u, (x.w << 16) & 0x7fff0000u)));
          }
          const int ex = scale_exponent(__uint_as_float(top));
          // a row that is not finite has no finite logit
          unit = top >= 0x7f800000u && hi > 0 ? __int_as_float(0x7fffffff) : unit * pow2f(ex);
          {
            const float down = pow2f(-ex);
            uint8_t* piece = sQ + qt * C::Q_BYTES;
            const int c0 = has_q1 ? 0 : t * (HD / 16), c1 = has_q1 ? HD / 8 : c0 + HD / 16;   // or half of the row each
#pragma unroll 2
            for (int c = c0; c < c1; ++c) {
              float x[8];
              unpack8(eight(c), x);
              uint32_t w1[2], w2[2];
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float y0 = x[2 * e] * down, y1 = x[2 * e + 1] * down;
                const uint32_t q1 = code2(y0, y1);
                const __half2 h(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)q1, __NV_E4M3));
                const uint32_t q2 = code2(y0 - __low2float(h), y1 - __high2float(h));
                w1[e >> 1] = e & 1 ? w1[e >> 1] | q1 << 16 : q1;
                w2[e >> 1] = e & 1 ? w2[e >> 1] | q2 << 16 : q2;
              }
              const int at = (HD == 128 ? row * 128 + (((c >> 1) ^ row) & 7) * 16 : row * 64 + (((c >> 1) ^ (row >> 1)) & 3) * 16) + (c & 1) * 8;
              *reinterpret_cast<uint2*>(piece + at) = make_uint2(w1[0], w1[1]);
              *reinterpret_cast<uint2*>(piece + BM * HD + at) = make_uint2(w2[0], w2[1]);
            }
            fence_proxy_async_smem();
          }
        }
        mbar_arrive(&bars->q_full);
      }
      // log2 of the largest V scale that the row has seen so far: its o is in units of 2^(e_ref - kLift).  It is
      // the row's own, since a page that the row does not see must not cost its values bits.
      float e_ref = -INFINITY;
      {
        uint32_t zero[32];
#pragma unroll
        for (int c = 0; c < 32; ++c) zero[c] = 0u;
#pragma unroll
        for (int c = 0; c < HD; c += 32) tmem_st_x32(tl + colO + c, zero);
      }
      auto scale_o = [&](float f) {
#pragma unroll 1
        for (int c = 0; c < HD; c += 32) {
          uint32_t x[32];
          tmem_ld_x32(tl + colO + c, x);
#pragma unroll
          for (int e = 0; e < 32; ++e) x[e] = __float_as_uint(__uint_as_float(x[e]) * f);
          tmem_st_x32(tl + colO + c, x);
        }
      };
      bool ok = true;
      uint32_t fixed = 0;
      const bool some_live = __any_sync(0xffffffffu, live);   // else this warp's rows are nobody's
      for (int j = j0; j < n_tiles; j += every) {
        if (!some_live) {
          const bool w = !aborted(bars) && mbar_wait(&bars->s_full[t], (uint32_t)(has_q1 ? j : j >> 1) & 1u, lim);
          if (!__all_sync(0xffffffffu, w)) { ok = false; break; }
          mbar_arrive(&bars->p_full[t]);
          continue;
        }
        float2 scale;
        if constexpr (F8) {
          scale = make_float2(next.x, log2f(next.y));
          next = scales_of(next_page);
          next_page = page_of(j + 2 * every);
        }
        bool w = !aborted(bars) && mbar_wait(&bars->s_full[t], (uint32_t)(has_q1 ? j : j >> 1) & 1u, lim);
        if (!__all_sync(0xffffffffu, w)) { ok = false; break; }
        tc_fence_after();
        const int pos = tile_pos(u, k0 + j);
        const bool whole = all_see(u, pos);
        if (!whole) {
          // S of columns that the row does not see (not below hi - pos, or below lo - pos and not below
          // sinks - pos) becomes -inf where it lies.  What few tiles need is kept in short loops: the
          // code that every tile runs has to stay in the instruction cache, for three kinds of warps.
          float e = -INFINITY;   // 8-bit pages: log2 of the largest V scale that the row (if it is one) sees
#pragma unroll 1
          for (int b = 0; b < BN; b += 32) {
            uint32_t x[32];
            tmem_ld_x32(tl + colS + b, x);
            auto below = [&](int c) {   // bits of columns b .. b + 31 that are below c
              const int k = c - b;
              return k <= 0 ? 0u : k >= 32 ? 0xffffffffu : (1u << k) - 1u;
            };
            const uint32_t see = below(hi - pos) & (~below(lo - pos) | below(sinks - pos));
#pragma unroll
            for (int c = 0; c < 32; ++c)
              if (!((see >> c) & 1u)) x[c] = __float_as_uint(-INFINITY);
            tmem_st_x32(tl + colS + b, x);
            if constexpr (F8) {
              const float e0 = __shfl_sync(0xffffffffu, scale.y, b / 16), e1 = __shfl_sync(0xffffffffu, scale.y, b / 16 + 1);
              e = fmaxf(e, fmaxf(!live || (see & 0xffffu) ? e0 : -INFINITY, !live || see >> 16 ? e1 : -INFINITY));
            }
          }
          if (F8 && __any_sync(0xffffffffu, e > e_ref)) {
            const float f = e > e_ref ? exp2_fast(e_ref - e) : 1.f;
            e_ref = fmaxf(e, e_ref);
            if (j > 0) scale_o(f);   // (o is 0 before the first tile)
          }
        }
        uint32_t sr[BN];
        tmem_ld_x64(tl + colS, sr);
        tmem_ld_x64(tl + colS + 64, sr + 64);
        float mx = -INFINITY;
        if constexpr (F8) {
#pragma unroll
          for (int c = 0; c < BN; c += 16) {
            auto x = [&](int e) { return __uint_as_float(sr[c + e]); };
            const float m0 = max3(max3(x(0), x(1), x(2)), x(3), x(4)), m1 = max3(max3(x(5), x(6), x(7)), x(8), x(9));
            const float m2 = max3(max3(x(10), x(11), x(12)), x(13), x(14));
            mx = fmaxf(mx, max3(m0, m1, fmaxf(m2, x(15))) * __shfl_sync(0xffffffffu, scale.x, c / 16));
          }
        } else {
          float m8[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) m8[e] = fmaxf(__uint_as_float(sr[2 * e]), __uint_as_float(sr[2 * e + 1]));
#pragma unroll
          for (int c = 16; c < BN; c += 16)
#pragma unroll
            for (int e = 0; e < 8; ++e)
              m8[e] = max3(m8[e], __uint_as_float(sr[c + 2 * e]), __uint_as_float(sr[c + 2 * e + 1]));
          mx = max3(max3(m8[0], m8[1], m8[2]), max3(m8[3], m8[4], m8[5]), fmaxf(m8[6], m8[7]));
        }
        mx *= unit;
        bool need = mx > m_ref + 8.f;
        float corr = 1.f;
        if (need) {
          corr = exp2_fast(m_ref - mx);   // 0 where the row has seen nothing yet
          m_ref = mx;
          l *= corr;
        }
        // a row that has seen nothing: 2^(-inf - 0) = 0
        const float ref = m_ref == -INFINITY ? 0.f : m_ref;
        if constexpr (F8) {
          float e = whole ? scale.y : -INFINITY;
#pragma unroll
          for (int o = 4; o; o >>= 1) e = fmaxf(e, __shfl_xor_sync(0xffffffffu, e, o, 8));
          e = __shfl_sync(0xffffffffu, e, 0);
          if (e > e_ref) {
            corr *= exp2_fast(e_ref - e);
            e_ref = e;
            need = true;
          }
          const float lift = kLift - ref;
#pragma unroll
          for (int c = 0; c < BN; c += 16) {
            // never 0: a hidden column's -inf has to stay -inf where a row of zeros (2^-123) meets a page of zero
            // keys (2^-120).  (A factor above 2^-102 is what it was; NaN, a query that is not finite, stays NaN.)
            const float by = fmaf(unit, __shfl_sync(0xffffffffu, scale.x, c / 16), 0x1p-126f);
            // log2 of the page's V scale in the row's units (a scale 2^60 below the largest adds nothing to o, and
            // everything to the sum; a page that the row does not see may have a larger one)
            const float in = fmaxf(fminf(__shfl_sync(0xffffffffu, scale.y, c / 16) - e_ref, 0.f), -60.f), add = in + lift;
            const float2 sc2 = make_float2(by, by), nm2 = make_float2(add, add);
            float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
            for (int k = 0; k < 16; k += 2) {
              const float2 x = __ffma2_rn(make_float2(__uint_as_float(sr[c + k]), __uint_as_float(sr[c + k + 1])), sc2, nm2);
              const float2 p2 = make_float2(exp2_fast(x.x), exp2_fast(x.y));
              sum[(k >> 1) & 1] = __fadd2_rn(sum[(k >> 1) & 1], p2);
              const __half2 h2 = __floats2half2_rn(p2.x, p2.y);
              sr[(c + k) / 2] = *reinterpret_cast<const uint32_t*>(&h2);
            }
            const float2 s2 = __fadd2_rn(sum[0], sum[1]);
            l = fmaf(s2.x + s2.y, exp2_fast(-in), l);   // 2^kLift times the sum
          }
          tmem_st_x64(tl + colS, sr);
        } else {
          const float2 sc2 = make_float2(unit, unit), nm2 = make_float2(-ref, -ref);
          float2 s4[4] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
          for (int c = 0; c < BN; c += 2) {
            const float2 x = __ffma2_rn(make_float2(__uint_as_float(sr[c]), __uint_as_float(sr[c + 1])), sc2, nm2);
            const float2 e = make_float2(exp2_fast(x.x), exp2_fast(x.y));
            s4[(c >> 1) & 3] = __fadd2_rn(s4[(c >> 1) & 3], e);
            const __nv_bfloat162 b2 = __floats2bfloat162_rn(e.x, e.y);
            sr[c / 2] = *reinterpret_cast<const uint32_t*>(&b2);
          }
          const float2 s2 = __fadd2_rn(__fadd2_rn(s4[0], s4[1]), __fadd2_rn(s4[2], s4[3]));
          l += s2.x + s2.y;
          tmem_st_x64(tl + colS, sr);
        }
        if (j > 0 && __any_sync(0xffffffffu, need)) scale_o(corr);
        if (!whole) {
          const int s = j % kStages;
          w = F8 ? mbar_wait(&bars->v_full[s], (uint32_t)(j / kStages) & 1u, lim)
                 : mbar_wait(&bars->v_fixed[s], (fixed >> s) & 1u, lim);
          fixed ^= 1u << s;
          if (!__all_sync(0xffffffffu, w)) { ok = false; break; }
          for (int b = 0; b < 4; ++b) {
            for (uint32_t bits = bars->apart[s][b]; bits; bits &= bits - 1) {
              // V row r holds a value that is not finite: its token by itself, where it is seen
              const int r = 32 * b + __ffs(bits) - 1, key = pos + r;
              const uint32_t pp = tmem_ld_1(tl + colS + r / 2);
              const float prob = F8 ? __half2float(__ushort_as_half((unsigned short)(r & 1 ? pp >> 16 : pp)))
                                    : __uint_as_float(r & 1 ? pp & 0xffff0000u : pp << 16);
              const bool see = key < hi && (key >= lo || key < sinks);
              const int page = __ldg(a.batch.page_table + (int64_t)u.b * a.batch.page_table_stride + (key >> a.page_shift));
              const int64_t at = ((int64_t)page * a.page_size + (key & (a.page_size - 1))) * a.row_stride + (int64_t)u.h * HD;
#pragma unroll 1
              for (int c = 0; c < HD; c += 32) {
                uint32_t orr[32];
                tmem_ld_x32(tl + colO + c, orr);
#pragma unroll
                for (int e = 0; e < 32; ++e) {
                  float x;
                  if (F8) {
                    const __half h(__nv_cvt_fp8_to_halfraw(__ldg(a.v + at + c + e), __NV_E4M3));
                    x = __half2float(h);
                  } else {
                    x = __uint_as_float((uint32_t)__ldg(reinterpret_cast<const uint16_t*>(a.v) + at + c + e) << 16);
                  }
                  if (see) orr[e] = __float_as_uint(__uint_as_float(orr[e]) + prob * x);
                }
                tmem_st_x32(tl + colO + c, orr);
              }
            }
          }
        }
        tc_fence_before();
        mbar_arrive(&bars->p_full[t]);
      }
      if (ok) {
        bool w = !aborted(bars) && mbar_wait(&bars->fin, 0, lim);
        ok = __all_sync(0xffffffffu, w);
      }
      if (!ok) set_abort(bars);
      tc_fence_after();
      const float o_unit = F8 ? exp2_fast(e_ref) * 0x1p-7f : 1.f;
      if (F8) l *= 0x1p-7f;
      float* other = reinterpret_cast<float*>(sV);   // [HD][128]: o of the second warpgroup (every product is done)
      const bool join = u.slot < 0 && !has_q1;
      if (join) {
        if (t == 1 && ok) {
#pragma unroll 1
          for (int half = 0; half < HD / 64; ++half) {
            uint32_t orr[64];
            tmem_ld_x64(tl + colO + half * 64, orr);
#pragma unroll
            for (int c = 0; c < 64; ++c) other[(half * 64 + c) * 128 + row] = __uint_as_float(orr[c]) * o_unit;
          }
          bars->ml[row] = make_float2(m_ref, l);
        }
        ok = !bar_sync_or(3, 256, !ok);
      }
      if (ok && u.slot < 0 && qt == t) {
        const int64_t out = (int64_t)(u.t0 + i) * a.H_q + u.h * a.group + (row - tok * a.group);
        float f0 = o_unit, f1 = 0.f;   // of this warpgroup's o, and of the second's
        if (join) {
          const float2 v = bars->ml[row];
          const float top = fmaxf(m_ref, v.x);
          f0 = m_ref == -INFINITY ? 0.f : exp2_fast(m_ref - top);
          f1 = v.x == -INFINITY ? 0.f : exp2_fast(v.x - top);
          l = f0 * l + f1 * v.y;
          m_ref = top;
          f0 *= o_unit;
        }
        const float inv = l == 0.f ? 0.f : (join ? 1.f : f0) / l;
#pragma unroll 1
        for (int half = 0; half < HD / 64; ++half) {
          uint32_t orr[64];
          tmem_ld_x64(tl + colO + half * 64, orr);
          float* v = reinterpret_cast<float*>(orr);
          if (join) {
#pragma unroll
            for (int c = 0; c < 64; ++c) v[c] = f0 * v[c] + f1 * other[(half * 64 + c) * 128 + row];
          }
          if (a.o_f32) {
            if (live) {
              float* dst = static_cast<float*>(a.o) + out * HD + half * 64;
#pragma unroll
              for (int c = 0; c < 64; c += 4)
                *reinterpret_cast<float4*>(dst + c) = make_float4(v[c] * inv, v[c + 1] * inv, v[c + 2] * inv, v[c + 3] * inv);
            }
          } else {
            // through the queries' place (every product is done), so that eight lanes write a row's 128 bytes
            uint8_t* stage = sQ + (warp - 4) * 4096;
#pragma unroll
            for (int c = 0; c < 64; c += 8) {
              float y[8];
#pragma unroll
              for (int e = 0; e < 8; ++e) y[e] = v[c + e] * inv;
              *reinterpret_cast<uint4*>(stage + lane * 128 + (((c / 8) ^ lane) & 7) * 16) = pack8(y);
            }
            __syncwarp();
            const uint32_t rows = __ballot_sync(0xffffffffu, live);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const int r = 4 * k + (lane >> 3);
              const int64_t to = __shfl_sync(0xffffffffu, out, r);
              const uint4 x = *reinterpret_cast<const uint4*>(stage + r * 128 + ((lane ^ r) & 7) * 16);
              if ((rows >> r) & 1u)
                *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.o) + to * HD + half * 64 + (lane & 7) * 8) = x;
            }
          }
          __syncwarp();
        }
        if (a.lse && live) a.lse[out] = l == 0.f ? -INFINITY : (m_ref + log2f(l)) * 0.69314718055994531f;
      } else if (ok && u.slot >= 0) {
        const int64_t slot = u.slot;
#pragma unroll 1
        for (int half = 0; half < HD / 64; ++half) {
          uint32_t orr[64];
          tmem_ld_x64(tl + colO + half * 64, orr);
          float* v = reinterpret_cast<float*>(orr);
          if (F8) {
#pragma unroll
            for (int c = 0; c < 64; ++c) v[c] *= o_unit;
          }
          if (live) {
#pragma unroll
            for (int c = 0; c < 64; c += 4)
              __stcg(a.part_o + (slot * (HD / 4) + half * 16 + c / 4) * 256 + t * 128 + row,
                     make_float4(v[c], v[c + 1], v[c + 2], v[c + 3]));
          }
          __syncwarp();
        }
        if (live) __stcg(a.part_ml + slot * 256 + t * 128 + row, make_float2(m_ref, l));
      }
      if (!another()) break;
    }
  } else if constexpr (F8) {
    // -------------------------------------------------------------- V codes to f16 tiles
    setmaxnreg_dec<C::REGS_DECODE>();
    const int tid = threadIdx.x - 384;
    constexpr int CH = HD / 16;   // 16-code chunks of a row, and of a thread
    const int quarter = lane & 3, second = (lane >> 2) & 1, w4 = warp & 3;
    auto row_of = [&](int i) {
      if (HD == 128) return ((i >> 1) * 4 + w4) * 8 + ((lane >> 3) ^ (second * 5));
      return (i * 4 + w4) * 8 + (lane >> 3) * 2 + second;
    };
    for (;;) {
    const int k0 = u.k0, n_tiles = u.n_tiles;
    const int log_stages = u.i0 + a.tile_tokens < u.n_new ? 1 : 2;
    // the queries lie in the V tiles' place until they are split
    bool ok = n_tiles == 0 || (!aborted(bars) && mbar_wait(&bars->q_full, 0, lim));
    ok = !bar_sync_or(2, 128, !ok);
    for (int j = 0; ok && j < n_tiles; ++j) {
      const int s = j % kStages, pos = tile_pos(u, k0 + j);
      const bool whole = all_see(u, pos);
      const int rs = j & ((1 << log_stages) - 1);   // of the codes
      const bool w = !aborted(bars) && mbar_wait(&bars->raw_full[rs], (uint32_t)(j >> log_stages) & 1u, lim) &&
                     mbar_wait(&bars->v_empty[s], ((uint32_t)(j / kStages) & 1u) ^ 1u, lim);
      // the four warps leave together: they meet at barriers below
      if (bar_sync_or(2, 128, !w)) { ok = false; break; }
      const uint8_t* src = raw_stage(rs);
      uint8_t* dst = sV + s * C::V_BYTES;
      if (!whole) {
        // rows that hold NaN, of a tile that the unit's rows do not all see alike (one row a thread)
        bool bad = false;
        if (some_see(u, pos + tid))
          for (int c = 0; c < CH; ++c) bad |= not_finite<true>(*reinterpret_cast<const uint4*>(src + tid * HD + c * 16));
        const uint32_t apart = __ballot_sync(0xffffffffu, bad);
        if (lane == 0) bars->apart[s][tid >> 5] = apart;
        asm volatile("bar.sync 2, 128;" ::: "memory");
      }
      // A thread has chunk `quarter` of 64 channels in CH rows; all its loads come first.  Eight lanes
      // have four chunks of two rows: of rows r and r ^ 5 the swizzled codes lie in eight bank groups, and
      // so do the f16 chunks they become (64-channel heads: rows r and r + 1 of unswizzled codes).
      uint4 codes[CH];
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const int r = row_of(i), box = HD == 128 ? i & 1 : 0;
        codes[i] = *reinterpret_cast<const uint4*>(src + r * HD + (HD == 128 ? ((box * 4 + quarter) ^ r) & 7 : quarter) * 16);
      }
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const int r = row_of(i), box = HD == 128 ? i & 1 : 0;
        uint4 o0, o1;
        half4(codes[i].x, o0.x, o0.y);
        half4(codes[i].y, o0.z, o0.w);
        half4(codes[i].z, o1.x, o1.y);
        half4(codes[i].w, o1.z, o1.w);
        if (!whole && (!some_see(u, pos + r) || ((bars->apart[s][r >> 5] >> (r & 31)) & 1u)))
          o0 = o1 = make_uint4(0, 0, 0, 0);
        uint8_t* base = dst + box * BN * 128 + r * 128;
        *reinterpret_cast<uint4*>(base + (((2 * quarter) ^ r) & 7) * 16) = o0;
        *reinterpret_cast<uint4*>(base + (((2 * quarter + 1) ^ r) & 7) * 16) = o1;
      }
      fence_proxy_async_smem();
      mbar_arrive(&bars->v_full[s]);
      mbar_arrive(&bars->raw_empty[rs]);
    }
    if (!ok) set_abort(bars);
    if (!another()) break;
    }
  }
}

// Joins the parts of the units that no CTA had whole: CTA (x, y, z) takes 32 rows (a lane each), and all
// channels or a quarter of them, of the unit that the share of CTA x + 1 begins inside of, if that is the
// first such share.  A warp has four channels and every so many of the parts, so that all of a CTA's loads
// are on their way together.  Bound: latency (measured: with eight parts loaded at once instead of summed one
// after the other 1000 rows of 6 heads over 9000 positions 41 -> 38 us in all).
constexpr int kMergeWarps = 16;
// SPREAD: units of few rows, of which four CTAs have a quarter of the channels each (then many CTAs had parts)
template <int HD, bool SPREAD>
__global__ void __launch_bounds__(kMergeWarps * 32) k_tiles_merge(const __grid_constant__ TilesKArgs a) {
  __shared__ float2 s_ml[kMergeWarps][32];
  __shared__ float4 s_o[kMergeWarps][32];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const Cut u = a.cuts[blockIdx.x + 1];
  if (u.c0 != (int)blockIdx.x) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, t = blockIdx.y >> 2;
  // the first CTA began the unit (its second place), the others began inside it (their first place); a
  // unit of one tile has two places of each row in a part
  const int c0 = u.c0;
  const bool pair = u.i0 + a.tile_tokens < u.n_new;
  const int n = (u.c1 - c0 + 1) * (pair ? 1 : 2);
  if (t == 1 && !pair) return;
  auto slot = [&](int p) {
    const int64_t c = c0 + (pair ? p : p >> 1);
    return 2 * c + (c == c0 ? 1 : 0);
  };
  const int row = (blockIdx.y & 3) * 32 + lane, tok = row / a.group, i = u.i0 + t * a.tile_tokens + tok;
  const bool in = tok < a.tile_tokens && i < u.n_new;
  if (!__any_sync(0xffffffffu, in)) return;   // the same rows in every warp
  auto place = [&](int p) { return pair ? t * 128 + row : row + (p & 1) * 128; };
  const int64_t out = (int64_t)(u.t0 + i) * a.H_q + u.h * a.group + (row - tok * a.group);
  auto store = [&](int c, const float4& v) {
    if (a.o_f32) *reinterpret_cast<float4*>(static_cast<float*>(a.o) + out * HD + c * 4) = v;
    else *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.o) + out * HD + c * 4) = make_uint2(pack2(v.x, v.y), pack2(v.z, v.w));
  };
  // Few parts: every warp has the maxima and sums of all of them, and all of a round's loads are on their way
  // at once: up to four parts of all of the warp's channels, or eight of four channels.
  auto few = [&](auto most, auto at_once) {
    constexpr int P = decltype(most)::value, Q = decltype(at_once)::value, COLUMNS = HD / 4 / kMergeWarps;
    float2 ml[P];
#pragma unroll
    for (int p = 0; p < P; ++p) ml[p] = p < n ? a.part_ml[slot(p) * 256 + place(p)] : make_float2(-INFINITY, 0.f);
#pragma unroll
    for (int k0 = 0; k0 < COLUMNS; k0 += Q) {
      float4 y[Q][P];
#pragma unroll
      for (int k = 0; k < Q; ++k)
#pragma unroll
        for (int p = 0; p < P; ++p)
          y[k][p] = p < n ? a.part_o[(slot(p) * (HD / 4) + warp + (k0 + k) * kMergeWarps) * 256 + place(p)]
                          : make_float4(0.f, 0.f, 0.f, 0.f);
      float top = -INFINITY, l = 0.f;
#pragma unroll
      for (int p = 0; p < P; ++p) top = fmaxf(top, ml[p].x);
      float4 acc[Q];
#pragma unroll
      for (int k = 0; k < Q; ++k) acc[k] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const float f = ml[p].x == -INFINITY ? 0.f : exp2_fast(ml[p].x - top);
        l += f * ml[p].y;
#pragma unroll
        for (int k = 0; k < Q; ++k) {
          acc[k].x += f * y[k][p].x; acc[k].y += f * y[k][p].y; acc[k].z += f * y[k][p].z; acc[k].w += f * y[k][p].w;
        }
      }
      const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
      for (int k = 0; k < Q; ++k)
        store(warp + (k0 + k) * kMergeWarps, make_float4(acc[k].x * inv, acc[k].y * inv, acc[k].z * inv, acc[k].w * inv));
      if (a.lse && warp == 0 && k0 == 0) a.lse[out] = l == 0.f ? -INFINITY : (top + log2f(l)) * 0.69314718055994531f;
    }
  };
  if constexpr (!SPREAD) if (n <= 8) {
    if (in && n <= 4) few(std::integral_constant<int, 4>{}, std::integral_constant<int, HD / 64>{});
    else if (in) few(std::integral_constant<int, 8>{}, std::integral_constant<int, 1>{});
    return;
  }
  // maximum and sum: each warp over some of the parts, then over the warps
  float top = -INFINITY, l = 0.f;
  if (in)
    for (int p = warp; p < n; p += kMergeWarps) {
      const float2 v = a.part_ml[slot(p) * 256 + place(p)];
      const float m = fmaxf(top, v.x);
      l = (top == -INFINITY ? 0.f : l * exp2_fast(top - m)) + (v.x == -INFINITY ? 0.f : v.y * exp2_fast(v.x - m));
      top = m;
    }
  s_ml[warp][lane] = make_float2(top, l);
  __syncthreads();
  for (int w = 0; w < kMergeWarps; ++w) top = fmaxf(top, s_ml[w][lane].x);
  l = 0.f;
  for (int w = 0; w < kMergeWarps; ++w) {
    const float2 v = s_ml[w][lane];
    l += v.x == -INFINITY ? 0.f : v.y * exp2_fast(v.x - top);
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  // columns of four channels: `columns` of them at a time, each by `sharers` warps
  constexpr int mine = HD / 4 / (SPREAD ? 4 : 1), columns = mine < kMergeWarps ? mine : kMergeWarps, sharers = kMergeWarps / columns;
  for (int k = 0; k < mine; k += columns) {
    const int c = blockIdx.z * mine + k + warp % columns;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    if (in)
#pragma unroll 8
      for (int p = warp / columns; p < n; p += sharers) {
        const float m = a.part_ml[slot(p) * 256 + place(p)].x;
        const float4 y = a.part_o[(slot(p) * (HD / 4) + c) * 256 + place(p)];
        const float f = m == -INFINITY ? 0.f : exp2_fast(m - top);
        acc.x += f * y.x; acc.y += f * y.y; acc.z += f * y.z; acc.w += f * y.w;
      }
    if (sharers > 1) {   // (one round)
      s_o[warp][lane] = acc;
      __syncthreads();
      if (warp >= columns) return;
      for (int w = warp + columns; w < kMergeWarps; w += columns) {
        const float4 y = s_o[w][lane];
        acc.x += y.x; acc.y += y.y; acc.z += y.z; acc.w += y.w;
      }
    }
    if (!in) continue;
    store(c, make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
  }
  if (a.lse && in && warp == 0 && blockIdx.z == 0) a.lse[out] = l == 0.f ? -INFINITY : (top + log2f(l)) * 0.69314718055994531f;
}

// ---------------------------------------------------------------- host side
bool encode(CUtensorMap* m, int elt, CUtensorMapSwizzle swizzle, const void* base, const cuuint64_t (&dims)[3],
            const cuuint64_t (&strides)[2], const cuuint32_t (&box)[3]) {
  EncodeTiledFn fn = tensor_map_encoder();
  const cuuint32_t es[3] = {1, 1, 1};
  return fn && fn(m, elt == 1 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base),
                  dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int HD, bool F8>
cast_status launch(const cast_cache_attn_args& a, const TilesKArgs& k, const TilesPlan& p, cudaStream_t st) {
  using C = Cfg<HD, F8>;
  const cast_kv_cache& c = a.cache;
  CUtensorMap mq, mk, mv;
  constexpr int elt = F8 ? 1 : 2;
  const cuuint64_t kd[3] = {(cuuint64_t)c.H * HD, (cuuint64_t)c.page_size, (cuuint64_t)c.n_pages};
  const cuuint64_t ks[2] = {(cuuint64_t)c.row_stride * elt, (cuuint64_t)c.row_stride * elt * c.page_size};
  const cuuint32_t kb[3] = {F8 ? HD : 64, (cuuint32_t)c.page_size, 1};
  // operand tiles are swizzled by their rows' 128 (or 64) bytes; V codes pass through registers
  const CUtensorMapSwizzle operand = F8 && HD == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B;
  const cuuint64_t qd[3] = {HD, (cuuint64_t)a.H_q, (cuuint64_t)a.batch.T}, qs[2] = {HD * 2, (cuuint64_t)a.q_row_stride * 2};
  const cuuint32_t qb[3] = {64, (cuuint32_t)k.group, (cuuint32_t)k.tile_tokens};
  const bool ok = encode(&mk, elt, operand, c.k, kd, ks, kb) &&
                  encode(&mv, elt, F8 && HD == 64 ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B, c.v, kd, ks, kb) &&
                  encode(&mq, 2, CU_TENSOR_MAP_SWIZZLE_128B, a.q, qd, qs, qb);
  if (!ok) return fail(CAST_ERR_CUDA, "cache attention: cuTensorMapEncodeTiled failed");
  static std::atomic<uint64_t> attr_done{0};
  cast_status setup = CAST_OK;
  if (!once_per_device(attr_done, [&] {
        cudaFuncAttributes fa{};
        if (cudaFuncGetAttributes(&fa, k_cache_tiles<HD, F8>) != cudaSuccess) return false;
        if (fa.numRegs != C::LAUNCH) {
          // the register hand-over counts on exactly this many
          setup = fail(CAST_ERR_UNSUPPORTED, "cache attention kernel built with %d registers per thread, expected %d", fa.numRegs,
                       C::LAUNCH);
          return false;
        }
        return cudaFuncSetAttribute(k_cache_tiles<HD, F8>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM) == cudaSuccess;
      }))
    return setup != CAST_OK ? setup : check_launch("cache attention kernel attributes");
  k_cache_tiles<HD, F8><<<(unsigned)p.grid, C::THREADS, C::SMEM, st>>>(mq, mk, mv, k);
  cast_status s = check_launch("cache attention");
  if (s || p.whole || p.grid == 1) return s;
  cudaLaunchConfig_t cfg{};
  // 32 rows of a unit a CTA, as many as a unit may have
  const int most = a.batch.max_new < a.batch.T ? a.batch.max_new : a.batch.T;
  const int rows = most > k.tile_tokens ? 8 : (most * k.group + 31) / 32;
  const bool spread = rows <= 2;
  cfg.gridDim = dim3((unsigned)(p.grid - 1), rows, spread ? 4 : 1);
  cfg.blockDim = dim3(kMergeWarps * 32, 1, 1);
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, spread ? k_tiles_merge<HD, true> : k_tiles_merge<HD, false>, k) != cudaSuccess) return check_launch("cache attention merge");
  return check_launch("cache attention merge");
}

}  // namespace

TilesPlan tiles_plan(const cast_cache_attn_args& a) {
  TilesPlan p{};
  const int group = a.H_q / a.cache.H, d = a.cache.d;
  p.tile_tokens = BM / group;
  const int per = 2 * p.tile_tokens;
  const int64_t T = a.batch.T, B = a.batch.B;
  // exactly, without cu_new; with it at most one ragged pair a sequence more than the whole ones
  const int64_t max_new = a.batch.max_new < T ? a.batch.max_new : T;
  int64_t pairs = a.batch.cu_new ? T / per + B : B * ((T / B + per - 1) / per);
  const int64_t bound = B * ((max_new + per - 1) / per);
  if (pairs > bound) pairs = bound;
  p.pairs = (int)(pairs > 0x7fffff ? 0x7fffff : pairs);
  const int64_t units = (int64_t)p.pairs * a.cache.H;
  const int64_t room = (int64_t)a.batch.max_pages * a.cache.page_size;
  int64_t seen = room;
  if (a.window > 0 && a.window + per + (int64_t)a.sinks + 3 * BN < room) seen = a.window + per + (int64_t)a.sinks + 3 * BN;
  const int64_t tiles = (seen + BN - 1) / BN;
  int dev = 0, nsm = 152;
  if (cudaGetDevice(&dev) == cudaSuccess) cudaDeviceGetAttribute(&nsm, cudaDevAttrMultiProcessorCount, dev);
  if (nsm < 1) nsm = 1;
  // Measured, shares / whole units, us: 6 prompts of up to 1201 with a window of 500 33 / 21.5, 16 chunks of 700 of
  // 1000 positions 46 / 37, 4 of 256 19.6 / 19.1; but of 3000 positions (24 tiles) 2 chunks of 512 23 / 41, 6 of up to
  // 1201 38 / 41, 16 of 700 88 / 80.
  p.whole = tiles <= 8;
  p.grid = p.whole ? units : nsm;
  if (!p.whole) {
    p.part_o_bytes = align_up((size_t)2 * p.grid * 256 * d * sizeof(float));
    p.part_ml_bytes = align_up((size_t)2 * p.grid * 256 * sizeof(float2));
    p.total_bytes = p.part_o_bytes + p.part_ml_bytes + align_up((size_t)p.grid * sizeof(Cut));
  }
  return p;
}

cast_status launch_tiles(const cast_cache_attn_args& a, const TilesPlan& p, void* ws, cudaStream_t st) {
  const cast_kv_cache& c = a.cache;
  if ((int64_t)p.pairs * c.H > 0x7fffffff)
    return fail(CAST_ERR_UNSUPPORTED, "cast_cache_attention: too many units");
  TilesKArgs k{};
  k.batch = a.batch;
  k.n_pages = c.n_pages;
  k.page_size = c.page_size;
  while ((1 << k.page_shift) < c.page_size) ++k.page_shift;
  k.H = c.H;
  k.H_q = a.H_q;
  k.group = a.H_q / c.H;
  k.tile_tokens = p.tile_tokens;
  k.causal = a.causal ? 1 : 0;
  k.window = a.window < (int64_t)a.batch.max_pages * c.page_size ? a.window : 0;
  k.sinks = k.window > 0 ? a.sinks : 0;
  k.o_f32 = a.o_dtype == CAST_F32;
  k.row_stride = c.row_stride;
  k.v = static_cast<const uint8_t*>(c.v);
  k.k_scale = c.k_scale;
  k.v_scale = c.v_scale;
  k.o = a.o;
  k.lse = a.lse;
  k.scale_log2 = (a.scale > 0.f ? a.scale : 1.f / sqrtf((float)c.d)) * 1.4426950408889634f;
  k.pairs = p.pairs;
  k.most_pairs = (int)(((a.batch.max_new < a.batch.T ? a.batch.max_new : a.batch.T) + 2 * p.tile_tokens - 1) / (2 * p.tile_tokens));
  k.whole = p.whole;
  k.least = 12;   // three key tiles of two query tiles, six of one: fewer are not worth a part
  k.part_o = static_cast<float4*>(ws);
  k.part_ml = reinterpret_cast<float2*>(static_cast<char*>(ws) + p.part_o_bytes);
  k.cuts = reinterpret_cast<Cut*>(static_cast<char*>(ws) + p.part_o_bytes + p.part_ml_bytes);
  k.wait_ns = 2000000000ull;
  if (c.dtype == CAST_F8E4M3) return c.d == 128 ? launch<128, true>(a, k, p, st) : launch<64, true>(a, k, p, st);
  return c.d == 128 ? launch<128, false>(a, k, p, st) : launch<64, false>(a, k, p, st);
}

unsigned int cache_tiles_error_word(cudaStream_t st, bool clear) { return read_left_out(st, clear); }

unsigned int tiles_error_word(cudaStream_t st, bool clear) {
  unsigned int v = 0;
  cudaMemcpyFromSymbolAsync(&v, g_tiles_error, sizeof(v), 0, cudaMemcpyDeviceToHost, st);
  cudaStreamSynchronize(st);
  if (clear && v) {
    const unsigned int z = 0;
    cudaMemcpyToSymbolAsync(g_tiles_error, &z, sizeof(z), 0, cudaMemcpyHostToDevice, st);
    cudaStreamSynchronize(st);
  }
  return v;
}

}  // namespace cast
