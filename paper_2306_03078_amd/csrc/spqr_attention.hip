// Softmax attention of a step's rows over a paged cache (spqr_tree_attention).
#include "spqr_serve.h"

#include <cmath>

namespace spqr_srv {

struct Attend {
  const void *q, *k, *v;
  void* out;
  int64_t q_stride, out_stride;
  const int32_t *cached, *table, *q_start;
  const uint64_t* mask;
  int requests, tokens, heads, group, kv_heads, page, pages, max_pages, words;
  float scale;
};

__device__ __forceinline__ float all_lanes_sum(float v) {
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
  return v;
}

// A workgroup a (row, head), a wavefront every fourth key: running maximum and sum, joined at the end.
template <typename T, int D>
__global__ void __launch_bounds__(256) row_kernel(Attend a) {
  constexpr int E = (D + 63) / 64;
  __shared__ float part[4][D + 2];
  const int t = blockIdx.x, h = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int r = 0, end = a.requests;               // the last request that starts at or before t
  while (end - r > 1) {
    const int mid = (r + end) / 2;
    if (a.q_start[mid] <= t) r = mid; else end = mid;
  }
  const int start = max(0, a.q_start[r]), rows = min(min(a.q_start[r + 1], a.tokens) - start, SPQR_MAX_FRESH);
  if (t < start || t - start >= rows) return;
  const int64_t cached = max(0, a.cached[r]), keys = cached + rows;
  const int kv = h / a.group, log_page = __ffs(a.page) - 1;
  const T* q = static_cast<const T*>(a.q) + t * a.q_stride + h * D;
  float x[E], o[E], m = -INFINITY, l = 0.f;
  for (int e = 0; e < E; ++e) { x[e] = lane + 64 * e < D ? (float)q[lane + 64 * e] * a.scale : 0.f; o[e] = 0.f; }
  for (int64_t j = wave; j < keys; j += 4) {
    const int64_t n = j - cached;
    if (n >= 0 && (a.words == 0 ? n > t - start : n >= 64 * a.words || !(a.mask[(int64_t)t * a.words + (n >> 6)] >> (n & 63) & 1))) continue;
    const int64_t at = j >> log_page;
    const int id = at < a.max_pages ? a.table[(int64_t)r * a.max_pages + at] : -1;
    if (id < 0 || id >= a.pages) continue;
    const int64_t row = (((int64_t)id * a.kv_heads + kv) * a.page + (j & (a.page - 1))) * D;
    const T *k = static_cast<const T*>(a.k) + row, *v = static_cast<const T*>(a.v) + row;
    float s = 0.f;
    for (int e = 0; e < E; ++e) if (lane + 64 * e < D) s = fmaf(x[e], (float)k[lane + 64 * e], s);
    s = all_lanes_sum(s);
    const float top = fmaxf(m, s), old = m == -INFINITY ? 0.f : __expf(m - top), p = top == -INFINITY ? 0.f : __expf(s - top);
    l = l * old + p;
    for (int e = 0; e < E; ++e) o[e] = o[e] * old + (lane + 64 * e < D ? p * (float)v[lane + 64 * e] : 0.f);
    m = top;
  }
  if (lane == 0) { part[wave][D] = m; part[wave][D + 1] = l; }
  for (int e = 0; e < E; ++e) if (lane + 64 * e < D) part[wave][lane + 64 * e] = o[e];
  __syncthreads();
  if (threadIdx.x >= D) return;
  float top = -INFINITY, sum = 0.f, y = 0.f;
  for (int w = 0; w < 4; ++w) top = fmaxf(top, part[w][D]);
  for (int w = 0; w < 4; ++w) {
    const float c = part[w][D] == -INFINITY ? 0.f : __expf(part[w][D] - top);
    sum = fmaf(c, part[w][D + 1], sum);
    y = fmaf(c, part[w][threadIdx.x], y);
  }
  static_cast<T*>(a.out)[t * a.out_stride + h * D + threadIdx.x] = (T)(sum == 0.f ? 0.f : y / sum);
}

template <typename T>
static void launch_rows(int D, const Attend& a, hipStream_t st) {
  const dim3 grid(a.tokens, a.heads), block(256);
  switch (D) {
    case 64: hipLaunchKernelGGL((row_kernel<T, 64>), grid, block, 0, st, a); break;
    case 96: hipLaunchKernelGGL((row_kernel<T, 96>), grid, block, 0, st, a); break;
    case 128: hipLaunchKernelGGL((row_kernel<T, 128>), grid, block, 0, st, a); break;
    default: hipLaunchKernelGGL((row_kernel<T, 256>), grid, block, 0, st, a);
  }
}

}  // namespace spqr_srv

using namespace spqr_srv;

extern "C" int64_t spqr_tree_attention_workspace_bytes(const spqr_step_t* s) {
  const int rc = check_cache(s);
  return rc ? rc : 0;
}

extern "C" int spqr_tree_attention(const spqr_step_t* s, int32_t layer, const void* q, int64_t q_stride, void* out, int64_t out_stride,
                                   void* stream) {
  const int rc = check_cache(s);
  if (rc) return rc;
  if (layer < 0 || layer >= s->layers) return SPQR_ERR_PARAM;
  if (!q || !out || !s->cached || !s->table || !s->q_start || (s->mask_words > 0 && !s->mask)) return SPQR_ERR_NULL;
  if (!std::isfinite(s->scale)) return SPQR_ERR_PARAM;
  const int64_t row = (int64_t)s->heads * s->head_dim;
  if (q_stride < row || out_stride < row) return SPQR_ERR_SHAPE;
  if (!aligned(q, 16) || !aligned(out, 16) || q_stride % 8 != 0 || out_stride % 8 != 0 || !aligned(s->cached, 4) || !aligned(s->table, 4) ||
      !aligned(s->q_start, 4) || !aligned(s->mask, 8))
    return SPQR_ERR_ALIGN;
  const int64_t layer_bytes = (int64_t)s->pages * s->kv_heads * s->page * s->head_dim * 2;
  Attend a;
  a.q = q; a.out = out; a.q_stride = q_stride; a.out_stride = out_stride;
  a.k = static_cast<const char*>(s->k) + layer * layer_bytes;
  a.v = static_cast<const char*>(s->v) + layer * layer_bytes;
  a.cached = s->cached; a.table = s->table; a.q_start = s->q_start; a.mask = s->mask;
  a.requests = s->requests; a.tokens = s->tokens; a.heads = s->heads; a.kv_heads = s->kv_heads; a.group = s->heads / s->kv_heads;
  a.page = s->page; a.pages = s->pages; a.max_pages = s->max_pages; a.words = s->mask_words; a.scale = s->scale;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if (s->dtype == SPQR_F16) launch_rows<_Float16>(s->head_dim, a, st);
  else launch_rows<__bf16>(s->head_dim, a, st);
  return launched();
}
