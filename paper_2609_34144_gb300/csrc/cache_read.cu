// The reading back of the paged KV cache (cast_cache_read): rows of tokens in their sequence's order, in bf16 or
// f32, from pages of any type.  What routing and anchor attention take as history blocks, and what a program looks
// at; attention over the cache itself reads the pages.
//
// Bound: memory (4-bit pages: 0.56 bytes a channel in, 2 out).  A thread has 8 channels of a row at a time, so that
// eight lanes write 128 bytes of a bf16 row side by side, and up to eight heads' loads are on their way together (with
// four 40 us where it is 35).  Measured, GB300, 24960 tokens of 12 heads of 128 to bf16: from 4 bits (196 MB) 33 us, 5.9 TB/s;
// from 8 bits 40 us; from bf16 (307 MB) 50 us, 6.1 TB/s.
#include "cache.cuh"

namespace cast {
namespace {

struct ReadKArgs {
  cast_cache_batch batch;
  int n_pages, page_size, d, H;
  int64_t row_stride, k_stride, v_stride;
  const uint8_t *ck, *cv;
  const uint8_t *k_scale, *v_scale;
  void *k, *v;
  int runs;        // page runs of a sequence that the grid has room for
  int chunks;      // CTAs that share a page's rows
  int group;       // heads of one CTA
  int jobs;        // head groups of K (and of V)
};

constexpr int kAtOnce = 8;

// Eight channels, as floats
template <int KIND>
struct Eight;
template <>
struct Eight<CAST_BF16> {
  uint4 w;
  __device__ __forceinline__ void values(float* v) const { unpack8(w, v); }
};
template <>
struct Eight<CAST_F8E4M3> {
  uint2 w;
  float scale;
  __device__ __forceinline__ void values(float* v) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t two = (e < 2 ? w.x : w.y) >> (16 * (e & 1));
      const __half2 y(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(two & 0xffffu), __NV_E4M3));
      v[2 * e] = __low2float(y) * scale;
      v[2 * e + 1] = __high2float(y) * scale;
    }
  }
};
template <>
struct Eight<CAST_F4E2M1> {
  uint32_t w, scale;
  __device__ __forceinline__ void values(float* v) const {
    uint32_t h[4];
    half8(w, h);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t t = times2(h[e], scale4_pair(scale));
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&t));
      v[2 * e] = f.x;
      v[2 * e + 1] = f.y;
    }
  }
};

// One CTA: some rows of a page of a sequence, for a group of heads of K or V.  blockDim = (runs of 8 channels of a row,
// rows).
template <int KIND, class OUT>
__global__ void __launch_bounds__(256) k_read(const __grid_constant__ ReadKArgs a) {
  const int chunk = blockIdx.x % a.chunks, b = blockIdx.x / a.chunks / a.runs, run = blockIdx.x / a.chunks - b * a.runs;
  const Sequence s = sequence_of(a.batch, b);
  const int kept = min(s.n_new, a.batch.max_new);
  const int p0 = s.len - s.n_new, first = max(p0, 0), end = p0 + kept;
  const bool is_k = (int)blockIdx.y < a.jobs;
  const int h0 = (blockIdx.y - (is_k ? 0 : a.jobs)) * a.group, heads = min(a.group, a.H - h0);
  OUT* out = static_cast<OUT*>(is_k ? a.k : a.v) + (int64_t)s.t0 * (is_k ? a.k_stride : a.v_stride) + threadIdx.x * 8;
  const int64_t out_stride = is_k ? a.k_stride : a.v_stride;
  const bool one = threadIdx.x == 0 && threadIdx.y == 0 && chunk == 0;
  const float none[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  auto store = [&](OUT* to, const float* v) {
    if constexpr (sizeof(OUT) == 2) {
      *reinterpret_cast<uint4*>(to) = pack8(v);
    } else {
      reinterpret_cast<float4*>(to)[0] = make_float4(v[0], v[1], v[2], v[3]);
      reinterpret_cast<float4*>(to)[1] = make_float4(v[4], v[5], v[6], v[7]);
    }
  };
  if (run == 0 && chunk == 0) {
    if (s.n_new > a.batch.max_new && one) left_out();
    // positions below 0
    for (int i = threadIdx.y; i < min(-p0, kept); i += blockDim.y)
      for (int h = h0; h < h0 + heads; ++h) store(out + (int64_t)i * out_stride + (int64_t)h * a.d, none);
  }
  const int g = first / a.page_size + run;   // page of the sequence
  if ((int64_t)g * a.page_size >= end) return;
  const int base = g * a.page_size;
  const int lo = max(first - base, 0), hi = min(end - base, a.page_size);
  if (lo >= hi) return;
  int page = g < a.batch.max_pages ? __ldg(a.batch.page_table + (int64_t)b * a.batch.page_table_stride + g) : -1;
  if (page < 0 || page >= a.n_pages) {
    if (one) left_out();
    page = -1;
  }
  const uint8_t* cache = is_k ? a.ck : a.cv;
  const uint8_t* scales = is_k ? a.k_scale : a.v_scale;
  const int row = chunk * blockDim.y + threadIdx.y;
  if (row < lo || row >= hi) return;
  OUT* to = out + (int64_t)(base + row - p0) * out_stride + (int64_t)h0 * a.d;
  if (page < 0) {
    for (int h = 0; h < heads; ++h) store(to + h * a.d, none);
    return;
  }
  // the row of head h0: codes, and the steps to the next head's
  const int64_t in_page = (int64_t)h0 * a.page_size + row;
  const uint8_t* from;
  const uint8_t* scale;
  int64_t step, scale_step;
  if constexpr (KIND == CAST_F4E2M1) {
    from = cache + (int64_t)page * a.page_size * a.row_stride / 2 + in_page * (a.d / 2) + threadIdx.x * 4;
    scale = scales + ((int64_t)page * a.H * a.page_size + in_page) * (a.d / 16) + threadIdx.x / 2;
    step = a.page_size * (a.d / 2);
    scale_step = a.page_size * (a.d / 16);
  } else {
    const int elt = KIND == CAST_BF16 ? 2 : 1;
    from = cache + (((int64_t)page * a.page_size + row) * a.row_stride + h0 * a.d + threadIdx.x * 8) * elt;
    scale = scales + ((int64_t)page * a.H + h0) * 4;
    step = a.d * elt;
    scale_step = 4;
  }
  for (int h = 0; h < heads; h += kAtOnce) {
    Eight<KIND> x[kAtOnce];
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {
      if (h + j >= heads) break;
      if constexpr (KIND == CAST_F4E2M1) {
        x[j].w = __ldg(reinterpret_cast<const uint32_t*>(from + (h + j) * step));
        x[j].scale = __ldg(scale + (h + j) * scale_step);
      } else if constexpr (KIND == CAST_F8E4M3) {
        x[j].w = __ldg(reinterpret_cast<const uint2*>(from + (h + j) * step));
        x[j].scale = __ldg(reinterpret_cast<const float*>(scale + (h + j) * scale_step));
      } else {
        x[j].w = __ldg(reinterpret_cast<const uint4*>(from + (h + j) * step));
      }
    }
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {
      if (h + j >= heads) break;
      float v[8];
      x[j].values(v);
      store(to + (h + j) * a.d, v);
    }
  }
}

template <int KIND>
void launch(const ReadKArgs& k, dim3 grid, dim3 block, bool f32, cudaStream_t st) {
  if (f32) k_read<KIND, float><<<grid, block, 0, st>>>(k);
  else k_read<KIND, __nv_bfloat16><<<grid, block, 0, st>>>(k);
}

}  // namespace

unsigned int cache_read_error_word(cudaStream_t st, bool clear) { return read_left_out(st, clear); }

}  // namespace cast

using namespace cast;

extern "C" cast_status cast_cache_read(const cast_cache_read_args* a, void* stream) {
  clear_error_detail();
  const char* who = "cast_cache_read";
  if (!a) return fail(CAST_ERR_INVALID_ARG, "%s: args is NULL", who);
  cast_status s = validate_cache(a->cache, who);
  if (s) return s;
  if ((s = validate_batch(a->batch, who))) return s;
  const cast_kv_cache& c = a->cache;
  if (a->out_dtype != CAST_BF16 && a->out_dtype != CAST_F32)
    return fail(CAST_ERR_INVALID_ARG, "%s: out_dtype %d", who, a->out_dtype);
  if (a->batch.T == 0) return CAST_OK;
  if (!a->k_out && !a->v_out) return fail(CAST_ERR_INVALID_ARG, "%s: neither k_out nor v_out", who);
  if (a->k_out && (s = check_rows(a->k_out, a->k_row_stride, (int64_t)c.H * c.d, "k_out", who))) return s;
  if (a->v_out && (s = check_rows(a->v_out, a->v_row_stride, (int64_t)c.H * c.d, "v_out", who))) return s;
  ReadKArgs k{};
  k.batch = a->batch;
  k.n_pages = c.n_pages;
  k.page_size = c.page_size;
  k.d = c.d;
  k.H = c.H;
  k.row_stride = c.row_stride;
  // K only, V only, or both: the grid's first jobs are K's
  const bool both = a->k_out && a->v_out;
  k.ck = static_cast<const uint8_t*>(a->k_out ? c.k : c.v);
  k.cv = static_cast<const uint8_t*>(c.v);
  k.k_scale = static_cast<const uint8_t*>((a->k_out ? c.k_scale : c.v_scale).bytes);
  k.v_scale = static_cast<const uint8_t*>(c.v_scale.bytes);
  k.k = a->k_out ? a->k_out : a->v_out;
  k.v = a->v_out;
  k.k_stride = a->k_out ? a->k_row_stride : a->v_row_stride;
  k.v_stride = a->v_row_stride;
  const int max_new = a->batch.max_new < a->batch.T ? a->batch.max_new : a->batch.T;
  k.runs = (int)(((int64_t)max_new + c.page_size - 2) / c.page_size + 1);
  const int lanes = c.d / 8, rows = 256 / lanes < c.page_size ? 256 / lanes : c.page_size;
  k.chunks = c.page_size / rows;
  const int64_t gx = (int64_t)k.runs * k.chunks * a->batch.B;
  if (gx > 0x7fffffff) return fail(CAST_ERR_UNSUPPORTED, "%s: %lld page runs", who, (long long)gx);
  // heads of one CTA: fewer where the grid would not fill the SMs
  int group = 16;
  while (group > 1 && gx * (both ? 2 : 1) * ((c.H + group - 1) / group) < 4 * 152 * 4) group /= 2;
  if ((int64_t)((c.H + group - 1) / group) * 2 > 65535) group = (c.H + 32766) / 32767;
  k.group = group;
  k.jobs = (c.H + group - 1) / group;
  const dim3 grid((unsigned)gx, (both ? 2 : 1) * k.jobs), block(lanes, rows);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool f32 = a->out_dtype == CAST_F32;
  if (c.dtype == CAST_F4E2M1) launch<CAST_F4E2M1>(k, grid, block, f32, st);
  else if (c.dtype == CAST_F8E4M3) launch<CAST_F8E4M3>(k, grid, block, f32, st);
  else launch<CAST_BF16>(k, grid, block, f32, st);
  return check_launch(who);
}
