// The paged KV cache's writers: rotary positions (cast_rotary) and the append of new tokens to the
// pages with the rotation and the 8-bit quantisation on the way (cast_cache_append).
//
// Both are bound by memory: every channel is read and written once, a pair costs six flops.  What
// is not free is the angle: 64 sines and cosines a token for heads of 128, shared by all heads, so
// a CTA computes them once for its tokens and several heads.  A call of a few tokens takes what its
// launch takes.
#include <cmath>

#include "cache.cuh"
#include "ptx.cuh"

namespace cast {
namespace {

// ------------------------------------------------------------------ cast_rotary
struct RotaryKArgs {
  const void* x;
  void* out;
  int64_t x_stride, out_stride;
  int T, H, d, n_axes, tokens;   // tokens: of one CTA
  const int* positions;
  float sign;
};

// Runs of 8 channels at p
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float* v) {
  unpack8(__ldcs(reinterpret_cast<const uint4*>(p)), v);
}
__device__ __forceinline__ void load8(const float* p, float* v) {
  const float4 a = __ldcs(reinterpret_cast<const float4*>(p));
  const float4 b = __ldcs(reinterpret_cast<const float4*>(p) + 1);
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
  v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float* v) {
  *reinterpret_cast<uint4*>(p) = pack8(v);
}
__device__ __forceinline__ void store8(float* p, const float* v) {
  reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}

// blockDim = (units in parallel, tokens in parallel): about one unit a thread, whose channels are on
// their way while the CTA computes its tokens' angles (shared memory, pair 8u + i at 8-unit stride, so
// that the threads of a row read without bank conflicts).  Measured, GB300: 1560 tokens of 12 heads of 128 in
// bf16 (9.6 MB) 4.6 us; 9973 tokens of 7 heads of 64 in f32 (36 MB) 9.4 us, 3.8 TB/s, most of the rest the launch.
template <class T>
__global__ void __launch_bounds__(256) k_rotary(const __grid_constant__ RotaryKArgs a,
                                                const __grid_constant__ cast_rotary_table tab) {
  extern __shared__ float2 cs[];   // [tokens][8][pairs / 8]
  const int pairs = tab.rot_dim / 2, turned = tab.rot_dim / 16, per_head = a.d / 16, units = a.H * per_head;
  const int t0 = blockIdx.x * a.tokens, n = min(a.tokens, a.T - t0);
  const int tid = threadIdx.y * blockDim.x + threadIdx.x, threads = blockDim.x * blockDim.y;
  const T* x = static_cast<const T*>(a.x) + (int64_t)t0 * a.x_stride;
  T* out = static_cast<T*>(a.out) + (int64_t)t0 * a.out_stride;
  float v[16];
  int c0 = 0, c1 = 0;
  auto load = [&](int u, int t) {
    const int h = u / per_head, c = u - h * per_head;
    unit_channels(c, tab.layout, tab.rot_dim, c0, c1);
    c0 += h * a.d;
    c1 += h * a.d;
    load8(x + t * a.x_stride + c0, v);
    load8(x + t * a.x_stride + c1, v + 8);
  };
  if (threadIdx.x < units && threadIdx.y < n) load(threadIdx.x, threadIdx.y);
  for (int i = tid; i < n * pairs; i += threads) {
    const int t = i / pairs, p = i - t * pairs;
    float2 c = rotary_cs(tab, p, __ldg(a.positions + (int64_t)(t0 + t) * a.n_axes + tab.axis[p]));
    c.y *= a.sign;
    cs[t * pairs + (p & 7) * turned + (p >> 3)] = c;
  }
  __syncthreads();
  for (int u = threadIdx.x; u < units; u += blockDim.x)
    for (int t = threadIdx.y; t < n; t += blockDim.y) {
      if (u != threadIdx.x || t != threadIdx.y) load(u, t);
      const int c = u % per_head;
      if (c < turned) {
        float2 w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = cs[t * pairs + i * turned + c];
        rotate_unit(v, w, tab.layout);
      }
      store8(out + t * a.out_stride + c0, v);
      store8(out + t * a.out_stride + c1, v + 8);
    }
}

// ------------------------------------------------------------------ cast_cache_append
struct AppendKArgs {
  cast_cache_batch batch;
  int n_pages, page_size, d, H, H_q, n_axes, turned;   // turned: a rotary table is given
  int64_t row_stride, k_stride, v_stride, q_stride, q_out_stride;
  const __nv_bfloat16 *k, *v, *q;
  __nv_bfloat16* q_out;
  void *ck, *cv;
  float *k_scale, *v_scale;
  const int* positions;
  int runs;               // page runs of a sequence that the grid has room for
  int group;              // heads of one CTA
  int jobs_kv, jobs_q;    // head groups of K (and of V), of the queries
};

// One CTA: the new tokens of one sequence in one page (a run of rows lo .. hi-1), for a group of
// heads of K, V or the queries.  A thread has one unit (row, 16 channels) of every head: it computes its
// eight angles once, and a page's maximum is known before the values leave the registers.  The next three
// heads' values are fetched while this one's are turned, reduced and stored: 1024 threads an SM have one
// head's 32 KB on their way otherwise, which is what the copy rate times the memory's latency takes.
// Bound: memory (every channel read and written once).  Measured, GB300: 14080 tokens, 24 KV and 24 query
// heads of 128, 8-bit pages (433 MB) 78 us, 5.5 TB/s, with three heads ahead (two 80, one 90 us) and
// groups of 12 heads (24 79, 8 84, 4 104 us: what the angles cost).
constexpr int kAhead = 4;
template <bool F8>
__global__ void __launch_bounds__(1024) k_append(const __grid_constant__ AppendKArgs a,
                                                 const __grid_constant__ cast_rotary_table tab) {
  __shared__ uint32_t s_max[2][32];
  extern __shared__ uint4 s_in[];   // [kAhead][2][threads]: what a thread has fetched ahead
  const int b = blockIdx.x / a.runs, run = blockIdx.x - b * a.runs;
  const Sequence s = sequence_of(a.batch, b);
  const int p0 = s.len - s.n_new;                       // place of the first new token
  const int first = max(p0, 0);
  const int g = first / a.page_size + run;              // page of the sequence
  if (run == 0 && s.n_new > a.batch.max_new && threadIdx.x == 0) left_out();
  const int end = p0 + min(s.n_new, a.batch.max_new);   // behind the last token that is stored
  if ((int64_t)g * a.page_size >= end) return;
  const int base = g * a.page_size;
  const int lo = max(first - base, 0), hi = min(end - base, a.page_size);
  if (lo >= hi) return;
  int job = blockIdx.y;
  const int kind = job < a.jobs_kv ? 0 : job < 2 * a.jobs_kv ? 1 : 2;   // K, V, queries
  job -= kind == 0 ? 0 : kind == 1 ? a.jobs_kv : 2 * a.jobs_kv;
  const int h0 = job * a.group, h1 = min(h0 + a.group, kind == 2 ? a.H_q : a.H);
  int page = 0;
  if (kind != 2) {
    page = g < a.batch.max_pages ? __ldg(a.batch.page_table + (int64_t)b * a.batch.page_table_stride + g) : -1;
    if (page < 0 || page >= a.n_pages) {
      if (threadIdx.x == 0) left_out();
      return;
    }
  }
  const int64_t token0 = (int64_t)s.t0 + base - p0;   // the call's row of the page's row 0 (may lie before the run)
  // the thread's unit: a row and its channels
  const int per_row = a.d / 16, row = threadIdx.x / per_row, col = threadIdx.x - row * per_row;
  const bool in = row >= lo && row < hi;
  const bool turned = a.turned && kind != 1 && col < tab.rot_dim / 16;
  int c0, c1;
  unit_channels(col, turned ? tab.layout : CAST_ROTARY_INTERLEAVED, tab.rot_dim, c0, c1);
  float2 cs[8];
  if (turned && in) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int p = 8 * col + i;
      cs[i] = rotary_cs(tab, p, a.positions ? __ldg(a.positions + (token0 + row) * a.n_axes + tab.axis[p]) : base + row);
    }
  }
  const __nv_bfloat16* src = (kind == 0 ? a.k : kind == 1 ? a.v : a.q) +
                             (token0 + row) * (kind == 0 ? a.k_stride : kind == 1 ? a.v_stride : a.q_stride);
  const int64_t to = kind == 2 ? (token0 + row) * a.q_out_stride : ((int64_t)page * a.page_size + row) * a.row_stride;
  const bool codes = F8 && kind != 2;
  auto fetch = [&](int h) {
    if (in && h < h1) {
      uint4* to = s_in + (h - h0) % kAhead * 2 * blockDim.x + threadIdx.x;
      copy16(smem_u32(to), src + (int64_t)h * a.d + c0);
      copy16(smem_u32(to + blockDim.x), src + (int64_t)h * a.d + c1);
    }
    copy_commit();
  };
#pragma unroll
  for (int i = 0; i < kAhead - 1; ++i) fetch(h0 + i);
  for (int h = h0; h < h1; ++h) {
    float v[16];
    copy_wait<kAhead - 2>();
    const uint4* from = s_in + (h - h0) % kAhead * 2 * blockDim.x + threadIdx.x;
    unpack8(in ? from[0] : make_uint4(0, 0, 0, 0), v);
    unpack8(in ? from[blockDim.x] : make_uint4(0, 0, 0, 0), v + 8);
    fetch(h + kAhead - 1);
    if (turned && in) rotate_unit(v, cs, tab.layout);
    const int64_t at = to + (int64_t)h * a.d;
    if (!codes) {
      if (in) {
        __nv_bfloat16* dst = kind == 2 ? a.q_out : static_cast<__nv_bfloat16*>(kind == 0 ? a.ck : a.cv);
        store8(dst + at + c0, v);
        store8(dst + at + c1, v + 8);
      }
      continue;
    }
    if constexpr (F8) {
      // the page's scale for this head: the largest magnitude of the tile (magnitudes order as their
      // bits; NaN is passed over), or, if that is infinite, the largest finite one
      float mine = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) mine = fmaxf(mine, fabsf(v[i]));
      uint32_t top = __reduce_max_sync(0xffffffffu, in ? __float_as_uint(mine) : 0u);
      if ((threadIdx.x & 31) == 0) s_max[h & 1][threadIdx.x >> 5] = top;
      float* scale = (kind == 0 ? a.k_scale : a.v_scale) + (int64_t)page * a.H + h;
      const float old = lo > 0 ? *scale : 0.f;
      __syncthreads();
      const int warps = blockDim.x / 32;
      top = __reduce_max_sync(0xffffffffu, (threadIdx.x & 31) < warps ? s_max[h & 1][threadIdx.x & 31] : 0u);
      if (top >= 0x7f800000u) {   // every thread alike
        mine = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          if (isinf(v[i])) v[i] = __int_as_float(0x7fffffff);   // the format has no infinity
          mine = fmaxf(mine, fabsf(v[i]));
        }
        top = __reduce_max_sync(0xffffffffu, in ? __float_as_uint(mine) : 0u);
        __syncthreads();
        if ((threadIdx.x & 31) == 0) s_max[h & 1][threadIdx.x >> 5] = top;
        __syncthreads();
        top = __reduce_max_sync(0xffffffffu, (threadIdx.x & 31) < warps ? s_max[h & 1][threadIdx.x & 31] : 0u);
      }
      const float now = fmaxf(pow2f(scale_exponent(__uint_as_float(top))), old);
      const float inv = 1.f / now;   // exact: a power of two within 2^-120 .. 2^120
      uint8_t* cache = static_cast<uint8_t*>(kind == 0 ? a.ck : a.cv);
      if (in) {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] *= inv;
        const uint2 w0 = encode8(v), w1 = encode8(v + 8);
        if (c1 == c0 + 8) {
          *reinterpret_cast<uint4*>(cache + at + c0) = make_uint4(w0.x, w0.y, w1.x, w1.y);
        } else {
          *reinterpret_cast<uint2*>(cache + at + c0) = w0;
          *reinterpret_cast<uint2*>(cache + at + c1) = w1;
        }
      }
      if (lo > 0 && now > old && row < lo) {
        // rows that were there before, rounded again at the larger scale
        uint4* p = reinterpret_cast<uint4*>(cache + at + 16 * col);
        const uint4 w = *p;
        const uint32_t in4[4] = {w.x, w.y, w.z, w.w};
        const float f = old * inv;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t two = in4[e >> 1] >> (16 * (e & 1));
          const __half2 y(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(two & 0xffffu), __NV_E4M3));
          v[2 * e] = __low2float(y) * f;
          v[2 * e + 1] = __high2float(y) * f;
        }
        const uint2 w0 = encode8(v), w1 = encode8(v + 8);
        *p = make_uint4(w0.x, w0.y, w1.x, w1.y);
      }
      // every thread has read `scale` before the barrier above
      if (threadIdx.x == 0) *scale = now;
    }
  }
}

// ------------------------------------------------------------------ host side
cast_status check_table(const cast_rotary_table* t, int d, const char* who) {
  if (t->rot_dim < 16 || t->rot_dim > 2 * CAST_MAX_ROTARY_PAIRS || t->rot_dim % 16 || t->n_axes < 1 ||
      t->n_axes > CAST_MAX_AXES || (t->layout != CAST_ROTARY_HALF && t->layout != CAST_ROTARY_INTERLEAVED) ||
      !std::isfinite(t->amplitude))
    return fail(CAST_ERR_INVALID_ARG, "%s: rotary table not made by cast_rotary_table_init", who);
  for (int i = 0; i < t->rot_dim / 2; ++i)
    if (t->axis[i] >= t->n_axes)
      return fail(CAST_ERR_INVALID_ARG, "%s: rotary table not made by cast_rotary_table_init", who);
  if (t->rot_dim > d)
    return fail(CAST_ERR_INVALID_ARG, "%s: %d rotated channels in heads of %d", who, t->rot_dim, d);
  return CAST_OK;
}

cast_status check_rows(const void* p, int64_t stride, int64_t least, const char* name, const char* who) {
  if (!p || !aligned16(p)) return fail(CAST_ERR_INVALID_ARG, "%s: %s is NULL or not 16-byte aligned", who, name);
  if (stride < least || stride % 8)
    return fail(CAST_ERR_INVALID_ARG, "%s: %s row stride %lld must be >= H*d = %lld and a multiple of 8", who, name,
                (long long)stride, (long long)least);
  return CAST_OK;
}

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

}  // namespace

cast_status validate_cache(const cast_kv_cache& c, const char* who) {
  if (c.dtype != CAST_BF16 && c.dtype != CAST_F8E4M3)
    return fail(CAST_ERR_INVALID_ARG, "%s: cache dtype %d", who, c.dtype);
  if (c.d != 64 && c.d != 128) return fail(CAST_ERR_UNSUPPORTED, "%s: head dim %d (64 or 128)", who, c.d);
  if (c.page_size != 16 && c.page_size != 32 && c.page_size != 64 && c.page_size != 128)
    return fail(CAST_ERR_UNSUPPORTED, "%s: page_size %d (16, 32, 64 or 128)", who, c.page_size);
  if (c.n_pages < 1 || c.H < 1)
    return fail(CAST_ERR_INVALID_ARG, "%s: n_pages %d and H %d must be positive", who, c.n_pages, c.H);
  if (!c.k || !c.v || !aligned16(c.k) || !aligned16(c.v))
    return fail(CAST_ERR_INVALID_ARG, "%s: cache k / v NULL or not 16-byte aligned", who);
  if (c.row_stride < (int64_t)c.H * c.d || c.row_stride % 16)
    return fail(CAST_ERR_INVALID_ARG, "%s: cache row stride %lld must be >= H*d and a multiple of 16", who,
                (long long)c.row_stride);
  if (c.dtype == CAST_F8E4M3 && (!c.k_scale || !c.v_scale || !aligned4(c.k_scale) || !aligned4(c.v_scale)))
    return fail(CAST_ERR_INVALID_ARG, "%s: 8-bit pages need k_scale and v_scale", who);
  return CAST_OK;
}

cast_status validate_batch(const cast_cache_batch& b, const char* who) {
  if (b.B < 1 || b.T < 0 || b.max_pages < 0 || b.max_new < (b.T > 0 ? 1 : 0))
    return fail(CAST_ERR_INVALID_ARG, "%s: bad batch (B %d, T %d, max_pages %d, max_new %d)", who, b.B, b.T,
                b.max_pages, b.max_new);
  if (!b.page_table || !b.kv_len || !aligned4(b.page_table) || !aligned4(b.kv_len) || !aligned4(b.cu_new))
    return fail(CAST_ERR_INVALID_ARG, "%s: page_table / kv_len NULL or misaligned", who);
  if (b.page_table_stride < b.max_pages && b.page_table_stride != 0)
    return fail(CAST_ERR_INVALID_ARG, "%s: page_table stride %lld below max_pages %d (and not 0)", who,
                (long long)b.page_table_stride, b.max_pages);
  if (!b.cu_new && (b.T % b.B || b.T / b.B > b.max_new))
    return fail(CAST_ERR_INVALID_ARG, "%s: without cu_new every sequence has T / B = %d / %d <= max_new = %d tokens", who,
                b.T, b.B, b.max_new);
  return CAST_OK;
}

unsigned int cache_error_word(cudaStream_t st, bool clear) { return read_left_out(st, clear); }

}  // namespace cast

using namespace cast;

extern "C" {

cast_status cast_rotary_table_init(const cast_rotary_params* p, cast_rotary_table* t) {
  clear_error_detail();
  const char* who = "cast_rotary_table_init";
  if (!p || !t) return fail(CAST_ERR_INVALID_ARG, "%s: params or table is NULL", who);
  if (p->rot_dim < 2 || p->rot_dim % 2) return fail(CAST_ERR_INVALID_ARG, "%s: rot_dim %d", who, p->rot_dim);
  if (p->rot_dim % 16 || p->rot_dim > 2 * CAST_MAX_ROTARY_PAIRS)
    return fail(CAST_ERR_UNSUPPORTED, "%s: rot_dim %d (a multiple of 16 up to %d)", who, p->rot_dim,
                2 * CAST_MAX_ROTARY_PAIRS);
  if (p->layout != CAST_ROTARY_HALF && p->layout != CAST_ROTARY_INTERLEAVED)
    return fail(CAST_ERR_INVALID_ARG, "%s: layout %d", who, p->layout);
  if (p->n_axes < 1 || p->n_axes > CAST_MAX_AXES) return fail(CAST_ERR_INVALID_ARG, "%s: n_axes %d", who, p->n_axes);
  if (p->scaling < CAST_ROTARY_PLAIN || p->scaling > CAST_ROTARY_PARTS)
    return fail(CAST_ERR_INVALID_ARG, "%s: scaling %d", who, p->scaling);
  if (!(p->base > 1.0) || !std::isfinite(p->base)) return fail(CAST_ERR_INVALID_ARG, "%s: base must be above 1", who);
  const bool scaled = p->scaling != CAST_ROTARY_PLAIN;
  if (scaled && (!(p->factor >= 1.0) || !std::isfinite(p->factor)))
    return fail(CAST_ERR_INVALID_ARG, "%s: factor must be >= 1", who);
  if (p->scaling == CAST_ROTARY_PARTS && p->original_length < 1)
    return fail(CAST_ERR_INVALID_ARG, "%s: original_length %d", who, p->original_length);
  int64_t sum = 0;
  for (int a = 0; a < p->n_axes; ++a) {
    if (p->pairs[a] < 1) return fail(CAST_ERR_INVALID_ARG, "%s: axis %d has %d pairs", who, a, p->pairs[a]);
    if (p->scaling == CAST_ROTARY_STRETCH && p->pairs[a] < 2)
      return fail(CAST_ERR_INVALID_ARG, "%s: a stretched base needs two pairs an axis", who);
    sum += p->pairs[a];
  }
  if (sum != p->rot_dim / 2)
    return fail(CAST_ERR_INVALID_ARG, "%s: the axes have %lld pairs, rot_dim %d has %d", who, (long long)sum, p->rot_dim,
                p->rot_dim / 2);
  constexpr double kTwoPi = 6.283185307179586476925;
  *t = cast_rotary_table{};
  t->rot_dim = p->rot_dim;
  t->layout = p->layout;
  t->n_axes = p->n_axes;
  t->amplitude = p->scaling == CAST_ROTARY_PARTS ? (float)(1.0 + 0.1 * std::log(p->factor)) : 1.f;
  int i = 0;
  for (int a = 0; a < p->n_axes; ++a) {
    const double n = p->pairs[a];
    const double base =
        p->scaling == CAST_ROTARY_STRETCH ? p->base * std::pow(p->factor, n / (n - 1.0)) : p->base;
    for (int k = 0; k < p->pairs[a]; ++k, ++i) {
      double f = std::pow(base, -k / n);
      if (p->scaling == CAST_ROTARY_LINEAR) f /= p->factor;
      if (p->scaling == CAST_ROTARY_PARTS) {
        double g = (p->original_length * f / kTwoPi - 1.0) / 31.0;
        g = g < 0.0 ? 0.0 : g > 1.0 ? 1.0 : g;
        f *= g + (1.0 - g) / p->factor;
      }
      t->turn[i] = (uint64_t)(f / kTwoPi * 0x1p64);   // f <= 1: below 2^62
      t->axis[i] = (uint8_t)a;
    }
  }
  return CAST_OK;
}

cast_status cast_rotary(const cast_rotary_args* a, void* stream) {
  clear_error_detail();
  const char* who = "cast_rotary";
  if (!a) return fail(CAST_ERR_INVALID_ARG, "%s: args is NULL", who);
  if (a->dtype != CAST_BF16 && a->dtype != CAST_F32) return fail(CAST_ERR_INVALID_ARG, "%s: dtype %d", who, a->dtype);
  if (a->T < 0 || a->H < 1 || a->d < 1)
    return fail(CAST_ERR_INVALID_ARG, "%s: bad shape T %d, H %d, d %d", who, a->T, a->H, a->d);
  if (a->d % 16 || a->d > 256) return fail(CAST_ERR_UNSUPPORTED, "%s: head dim %d (a multiple of 16 up to 256)", who, a->d);
  if ((int64_t)a->H * a->d > (1 << 24)) return fail(CAST_ERR_UNSUPPORTED, "%s: %d heads of %d", who, a->H, a->d);
  if (!a->table) return fail(CAST_ERR_INVALID_ARG, "%s: table is NULL", who);
  cast_status s = check_table(a->table, a->d, who);
  if (s) return s;
  if (a->T == 0) return CAST_OK;
  if ((s = check_rows(a->x, a->x_row_stride, (int64_t)a->H * a->d, "x", who))) return s;
  if ((s = check_rows(a->out, a->out_row_stride, (int64_t)a->H * a->d, "out", who))) return s;
  if (!a->positions || !aligned4(a->positions))
    return fail(CAST_ERR_INVALID_ARG, "%s: positions NULL or misaligned", who);
  RotaryKArgs k{};
  k.x = a->x;
  k.out = a->out;
  k.x_stride = a->x_row_stride;
  k.out_stride = a->out_row_stride;
  k.T = a->T;
  k.H = a->H;
  k.d = a->d;
  k.n_axes = a->table->n_axes;
  k.positions = a->positions;
  k.sign = a->inverse ? -1.f : 1.f;
  const int units = a->H * (a->d / 16);
  int tx = 1;
  while (tx < units && tx < 256) tx *= 2;
  const dim3 block(tx, 256 / tx);
  // about one unit a thread, and fewer tokens a CTA where the SMs would not be filled twice; never more
  // than 48 KB of angles
  int tokens = (256 + units - 1) / units;
  if (tokens > (a->T + 303) / 304) tokens = (a->T + 303) / 304;
  const int cap = 48 * 1024 / (a->table->rot_dim / 2 * 8);
  if (tokens > cap) tokens = cap;
  k.tokens = tokens;
  const size_t smem = (size_t)tokens * (a->table->rot_dim / 2) * sizeof(float2);
  const unsigned grid = (unsigned)((a->T + (int64_t)tokens - 1) / tokens);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (a->dtype == CAST_BF16)
    k_rotary<__nv_bfloat16><<<grid, block, smem, st>>>(k, *a->table);
  else
    k_rotary<float><<<grid, block, smem, st>>>(k, *a->table);
  return check_launch(who);
}

cast_status cast_cache_append(const cast_append_args* a, void* stream) {
  clear_error_detail();
  const char* who = "cast_cache_append";
  if (!a) return fail(CAST_ERR_INVALID_ARG, "%s: args is NULL", who);
  cast_status s = validate_cache(a->cache, who);
  if (s) return s;
  if ((s = validate_batch(a->batch, who))) return s;
  const cast_kv_cache& c = a->cache;
  if (a->rotary) {
    if ((s = check_table(a->rotary, c.d, who))) return s;
    if (!a->positions && a->rotary->n_axes != 1)
      return fail(CAST_ERR_INVALID_ARG, "%s: a table of %d axes needs positions", who, a->rotary->n_axes);
    if (!aligned4(a->positions)) return fail(CAST_ERR_INVALID_ARG, "%s: positions misaligned", who);
  }
  if (a->batch.T == 0) return CAST_OK;
  if ((s = check_rows(a->k, a->k_row_stride, (int64_t)c.H * c.d, "k", who))) return s;
  if ((s = check_rows(a->v, a->v_row_stride, (int64_t)c.H * c.d, "v", who))) return s;
  if (a->q) {
    if (a->H_q < 1) return fail(CAST_ERR_INVALID_ARG, "%s: H_q %d", who, a->H_q);
    if (!a->rotary) return fail(CAST_ERR_INVALID_ARG, "%s: q given without a rotary table", who);
    if ((s = check_rows(a->q, a->q_row_stride, (int64_t)a->H_q * c.d, "q", who))) return s;
    if ((s = check_rows(a->q_out, a->q_out_row_stride, (int64_t)a->H_q * c.d, "q_out", who))) return s;
  }
  AppendKArgs k{};
  k.batch = a->batch;
  k.n_pages = c.n_pages;
  k.page_size = c.page_size;
  k.d = c.d;
  k.H = c.H;
  k.H_q = a->q ? a->H_q : 0;
  k.n_axes = a->rotary ? a->rotary->n_axes : 1;
  k.turned = a->rotary ? 1 : 0;
  k.row_stride = c.row_stride;
  k.k_stride = a->k_row_stride;
  k.v_stride = a->v_row_stride;
  k.q_stride = a->q_row_stride;
  k.q_out_stride = a->q_out_row_stride;
  k.k = static_cast<const __nv_bfloat16*>(a->k);
  k.v = static_cast<const __nv_bfloat16*>(a->v);
  k.q = static_cast<const __nv_bfloat16*>(a->q);
  k.q_out = static_cast<__nv_bfloat16*>(a->q_out);
  k.ck = c.k;
  k.cv = c.v;
  k.k_scale = c.k_scale;
  k.v_scale = c.v_scale;
  k.positions = a->positions;
  // a sequence's new tokens touch at most this many pages
  const int max_new = a->batch.max_new < a->batch.T ? a->batch.max_new : a->batch.T;
  k.runs = (max_new + c.page_size - 2) / c.page_size + 1;
  const int64_t gx = (int64_t)k.runs * a->batch.B;
  if (gx > 0x7fffffff) return fail(CAST_ERR_UNSUPPORTED, "%s: %lld page runs", who, (long long)gx);
  const int threads = c.page_size * c.d / 16;
  // heads of one CTA: twelve share the angles' cost, fewer where the grid would not fill the SMs (1024 threads
  // each) three times
  int group = 12;
  while (group > 1 &&
         gx * (2 * ((c.H + group - 1) / group) + (k.H_q + group - 1) / group) * threads < (int64_t)3 * 152 * 1024)
    group /= 2;
  k.group = group;
  k.jobs_kv = (c.H + group - 1) / group;
  k.jobs_q = (k.H_q + group - 1) / group;
  if (2 * (int64_t)k.jobs_kv + k.jobs_q > 65535) return fail(CAST_ERR_UNSUPPORTED, "%s: too many heads", who);
  const int bytes = kAhead * 2 * 16 * threads;
  static std::atomic<uint64_t> attr_done{0};
  if (!once_per_device(attr_done, [&] {
        return cudaFuncSetAttribute(k_append<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kAhead * 32 * 1024) == cudaSuccess &&
               cudaFuncSetAttribute(k_append<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kAhead * 32 * 1024) == cudaSuccess;
      }))
    return check_launch("cache append kernel attributes");
  const dim3 grid((unsigned)gx, 2 * k.jobs_kv + k.jobs_q);
  const cast_rotary_table none{};
  const cast_rotary_table& tab = a->rotary ? *a->rotary : none;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (c.dtype == CAST_F8E4M3)
    k_append<true><<<grid, threads, bytes, st>>>(k, tab);
  else
    k_append<false><<<grid, threads, bytes, st>>>(k, tab);
  return check_launch(who);
}

}  // extern "C"
