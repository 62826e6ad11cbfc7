// Norms before and after a block with its gate and the residual sum (spqr_residual_norm).
#include "spqr_block.h"

namespace spqr_blk {

// Sum over the `lanes` threads of a row (a power of two; whole wavefronts above 64), in every one of them.  part: one float a
// wavefront; all threads of the workgroup take part.
__device__ __forceinline__ float row_sum(float v, int lanes, float* part) {
  for (int d = min(lanes, 64) >> 1; d > 0; d >>= 1) v += __shfl_xor(v, d);
  if (lanes > 64) {
    const int wave = threadIdx.x >> 6, waves = lanes >> 6, first = wave & ~(waves - 1);
    __syncthreads();                             // everyone has read the last sum
    if ((threadIdx.x & 63) == 0) part[wave] = v;
    __syncthreads();
    v = 0.f;
    for (int w = 0; w < waves; ++w) v += part[first + w];
  }
  return v;
}

template <int CH>
__device__ __forceinline__ void norm(int kind, float (&v)[CH][8], const int (&at)[CH], int n, float eps, int weight_dtype, float offset,
                                     const void* weight, const void* bias, int lanes, float* part) {
  if (kind == SPQR_NORM_NONE) return;
  float mean = 0.f;
  if (kind == SPQR_NORM_LAYER) {
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += v[c][e];
    mean = row_sum(sum, lanes, part) / (float)n;
  }
  float squares = 0.f;
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[c][e] = at[c] + e < n ? v[c][e] - mean : 0.f;
      squares = fmaf(v[c][e], v[c][e], squares);
    }
  const float r = 1.f / sqrtf(row_sum(squares, lanes, part) / (float)n + eps);
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    float w[8], b[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) { w[e] = 1.f; b[e] = 0.f; }
    if (weight && at[c] < n) {
      load_row8_as(weight_dtype, weight, 0, at[c], n, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] += offset;
    }
    if (bias && at[c] < n) load_row8_as(weight_dtype, bias, 0, at[c], n, b);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[c][e] = fmaf(v[c][e] * r, w[e], b[e]);
  }
}

__device__ __forceinline__ float activated(int act, float g) {
  if (act == SPQR_ACT_TANH) return tanhf(g);
  const float s = 1.f / (1.f + __expf(-g));
  return act == SPQR_ACT_SIGMOID ? s : g * s;
}

// `lanes` threads a row, CH runs of eight elements each, which stay in registers from the loads to the stores.
template <int CH>
__global__ void __launch_bounds__(1024) residual_norm_kernel(spqr_residual_norm_t p, int lanes) {
  __shared__ float part[16];
  const int n = p.width, in_row = threadIdx.x & (lanes - 1);
  const int64_t row = (int64_t)blockIdx.x * (blockDim.x / lanes) + threadIdx.x / lanes;
  const bool live = row < p.rows;
  const int64_t t = live ? row : p.rows - 1;               // (takes part in the sums, stores nothing)
  int at[CH];
  float v[CH][8];
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    at[c] = 8 * (in_row + lanes * c);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[c][e] = 0.f;
    if (p.y && at[c] < n) load_row8_as(p.y_dtype, p.y, t * p.y_stride, at[c], n, v[c]);
  }
  if (p.y) {
    norm<CH>(p.norm_y, v, at, n, p.eps, p.weight_dtype, p.weight_offset, p.y_weight, p.y_bias, lanes, part);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float g[8];
      if (p.gate && at[c] < n) {
        load_row8_as(p.gate_dtype, p.gate, t * p.gate_stride, at[c], n, g);
        if (p.act != SPQR_ACT_NONE)
#pragma unroll
          for (int e = 0; e < 8; ++e) g[e] = activated(p.act, g[e]);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[c][e] *= g[e];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) v[c][e] *= p.scale;
    }
  }
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    float x[8];
    if (p.x && at[c] < n) {
      load_row8_as(p.x_dtype, p.x, t * p.x_stride, at[c], n, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[c][e] = fmaf(p.skip, x[e], v[c][e]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[c][e] = at[c] + e < n ? v[c][e] : 0.f;
    if (p.sum && live && at[c] < n) store_row8_as(p.x_dtype, p.sum, t * p.sum_stride, at[c], n, v[c]);
  }
  if (!p.out) return;
  norm<CH>(p.norm_x, v, at, n, p.eps, p.weight_dtype, p.weight_offset, p.x_weight, p.x_bias, lanes, part);
#pragma unroll
  for (int c = 0; c < CH; ++c)
    if (live && at[c] < n) store_row8_as(p.out_dtype, p.out, t * p.out_stride, at[c], n, v[c]);
}

static int check_vectors(const spqr_residual_norm_t* p) {
  const void* vectors[4] = {p->y_weight, p->y_bias, p->x_weight, p->x_bias};
  for (const void* v : vectors) {
    if (v && !known(p->weight_dtype)) return SPQR_ERR_DTYPE;
    if (!aligned(v, v ? size_of(p->weight_dtype) : 1)) return SPQR_ERR_ALIGN;
  }
  return SPQR_OK;
}

// A tensor of rows: its type, the distance of its rows, its address.
static int check_rows(const spqr_residual_norm_t* p, const void* v, int dtype, int64_t stride) {
  if (!v) return SPQR_OK;
  if (!known(dtype)) return SPQR_ERR_DTYPE;
  if (stride < p->width || stride > INT64_MAX / 8 / (p->rows > 0 ? p->rows : 1)) return SPQR_ERR_SHAPE;
  return aligned(v, size_of(dtype)) ? SPQR_OK : SPQR_ERR_ALIGN;
}

}  // namespace spqr_blk

using namespace spqr_blk;

extern "C" int spqr_residual_norm(const spqr_residual_norm_t* p, void* stream) {
  if (!p) return SPQR_ERR_NULL;
  if (p->rows < 0 || p->width < 1 || p->width > SPQR_MAX_WIDTH) return SPQR_ERR_SHAPE;
  if (p->norm_y < SPQR_NORM_NONE || p->norm_y > SPQR_NORM_LAYER || p->norm_x < SPQR_NORM_NONE || p->norm_x > SPQR_NORM_LAYER ||
      p->act < SPQR_ACT_NONE || p->act > SPQR_ACT_TANH)
    return SPQR_ERR_PARAM;
  if (!(p->eps > 0.f) || !isfinite(p->eps) || !isfinite(p->weight_offset) || !isfinite(p->skip) || !isfinite(p->scale)) return SPQR_ERR_PARAM;
  if (p->rows == 0) return SPQR_OK;
  if ((!p->x && !p->y) || (!p->sum && !p->out)) return SPQR_ERR_NULL;
  int rc = check_rows(p, p->x, p->x_dtype, p->x_stride);
  if (!rc) rc = check_rows(p, p->y, p->y_dtype, p->y_stride);
  if (!rc) rc = check_rows(p, p->sum, p->x_dtype, p->sum_stride);
  if (!rc) rc = check_rows(p, p->out, p->out_dtype, p->out_stride);
  if (!rc) rc = check_rows(p, p->gate, p->gate_dtype, p->gate_stride == 0 ? p->width : p->gate_stride);
  if (!rc) rc = check_vectors(p);
  if (rc) return rc;
  const int runs = (p->width + 7) / 8;
  int lanes = 8;
  while (lanes < runs && lanes < 1024) lanes *= 2;
  const int threads = lanes > 256 ? lanes : 256, per = threads / lanes;
  const int64_t grid = ((int64_t)p->rows + per - 1) / per;
  const dim3 g((unsigned)grid), b(threads);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const int ch = (runs + lanes - 1) / lanes;
  if (ch <= 1) hipLaunchKernelGGL(residual_norm_kernel<1>, g, b, 0, st, *p, lanes);
  else if (ch <= 2) hipLaunchKernelGGL(residual_norm_kernel<2>, g, b, 0, st, *p, lanes);
  else if (ch <= 4) hipLaunchKernelGGL(residual_norm_kernel<4>, g, b, 0, st, *p, lanes);
  else hipLaunchKernelGGL(residual_norm_kernel<8>, g, b, 0, st, *p, lanes);
  return launched();
}
