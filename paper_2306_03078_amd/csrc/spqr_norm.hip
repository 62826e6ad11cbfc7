// Norms before and after a block with its gate and the residual sum (spqr_residual_norm).
#include "spqr_block.h"

namespace spqr_blk {

// Adds what a data-parallel move brings (0 where it brings nothing).
template <int CTRL, int ROWS>
__device__ __forceinline__ float plus(float v) {
  return v + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, ROWS, 0xF, false));
}
// Sum over 16 lanes, in the last of them; over the wavefront, the same in all of its lanes.
__device__ __forceinline__ float sum16(float v) {
  v = plus<0x111, 0xF>(v);                       // row_shr:1, 2, 4, 8
  v = plus<0x112, 0xF>(v);
  v = plus<0x114, 0xF>(v);
  return plus<0x118, 0xF>(v);
}
__device__ __forceinline__ float lane_of(float v, int lane) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), lane)); }
__device__ __forceinline__ float sum64(float v) {
  v = plus<0x142, 0xA>(sum16(v));                // row_bcast:15, then :31: a row's sum to the next one, the first half's to the second
  return lane_of(plus<0x143, 0xC>(v), 63);
}

// Sum over the `lanes` threads of a row (a power of two; whole wavefronts above 64), in every one of them.  part: two buffers of one float a
// wavefront, taken in turn, so that one barrier a sum is enough (the next sum's stands between its readers and the next writers).
struct RowSum {
  float (*part)[16];
  int lanes, turn;
  __device__ __forceinline__ float operator()(float v) {
    if (lanes < 64) {
      for (int d = lanes >> 1; d > 0; d >>= 1) v += __shfl_xor(v, d);
      return v;
    }
    v = sum64(v);
    if (lanes > 64) {
      const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = lanes >> 6;
      if (lane == 0) part[turn][wave] = v;
      __syncthreads();
      // 16 lanes take the row's wavefronts
      v = lane_of(sum16((lane & 15) < waves ? part[turn][(wave & ~(waves - 1)) + (lane & 15)] : 0.f), 15);
      turn ^= 1;
    }
    return v;
  }
};

__device__ __forceinline__ float activated(int act, float g) {
  if (act == SPQR_ACT_TANH) return tanhf(g);
  const float s = __builtin_amdgcn_rcpf(1.f + __expf(-g));
  return act == SPQR_ACT_SIGMOID ? s : g * s;
}

// ---------------------------------------------------------------------------------------------------------------------
// Rows of up to 8192 elements: eight of them a thread.
// ---------------------------------------------------------------------------------------------------------------------
// Eight elements as they were loaded, of any type: they are worked out where they are needed, so that the loads of all terms are on their
// way at once.
struct Raw { u32x4 a, b; };
typedef u32x4 u32x4_at2 __attribute__((aligned(2)));

__device__ __forceinline__ void load(Raw& r, int dtype, const void* p, int64_t element) {
  const char* at = static_cast<const char*>(p) + element * (dtype == SPQR_F32 ? 4 : 2);
  r.a = *reinterpret_cast<const u32x4_at2*>(at);
  if (dtype == SPQR_F32) r.b = *reinterpret_cast<const u32x4_at2*>(at + 16);
}
__device__ __forceinline__ void floats(const Raw& r, int dtype, float (&v)[8]) {
  if (dtype == SPQR_F32) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(e < 4 ? r.a[e] : r.b[e - 4]);
  } else if (dtype == SPQR_F16) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = spqr::h2f((uint16_t)(r.a[e / 2] >> 16 * (e & 1)));
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(e & 1 ? r.a[e / 2] & 0xFFFF0000u : r.a[e / 2] << 16);
  }
}

// Where a thread's eight elements lie in a row: it reads those from `from` on, whatever it has; `shift` of them are another thread's where the row
// ends inside its eight, `count` (0 .. 8) are there.  ODD: rows whose length is no multiple of 8; else a thread has all eight or none.
struct Place { int col, from, shift, count; };

template <bool ODD>
__device__ __forceinline__ void floats_at(const Raw& r, int dtype, const Place& at, float (&v)[8]) {
  floats(r, dtype, v);
  if (!ODD) return;
#pragma unroll
  for (int d = 4; d > 0; d >>= 1)
#pragma unroll
    for (int e = 0; e + d < 8; ++e) v[e] = at.shift & d ? v[e + d] : v[e];
}
// What is no element counts nothing.
template <bool ODD>
__device__ __forceinline__ float sum_of(const float (&v)[8], const Place& at) {
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) s += !ODD || e < at.count ? v[e] : 0.f;
  return ODD || at.count > 0 ? s : 0.f;
}
template <bool ODD>
__device__ __forceinline__ float squares_of(const float (&v)[8], const Place& at) {
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float x = !ODD || e < at.count ? v[e] : 0.f;
    s = fmaf(x, x, s);
  }
  return ODD || at.count > 0 ? s : 0.f;
}

template <bool ODD>
__device__ __forceinline__ void norm_rows(int kind, float (&v)[8], const Place& at, const spqr_residual_norm_t& p, const void* weight, const void* bias, const Raw& w,
                                          const Raw& b, RowSum& sum) {
  if (kind == SPQR_NORM_NONE) return;
  const float inverse = 1.f / (float)p.width;
  if (kind == SPQR_NORM_LAYER) {
    const float mean = sum(sum_of<ODD>(v, at)) * inverse;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] -= mean;
  }
  const float r = __builtin_amdgcn_rsqf(fmaf(sum(squares_of<ODD>(v, at)), inverse, p.eps));
  float x[8];
  if (weight) {
    floats_at<ODD>(w, p.weight_dtype, at, x);
    if (p.weight_offset != 0.f)
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] += p.weight_offset;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= r * x[e];
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= r;
  }
  if (bias) {
    floats_at<ODD>(b, p.weight_dtype, at, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += x[e];
  }
}

template <typename T> struct TypeOf { static constexpr int value = SPQR_F32; };
template <> struct TypeOf<_Float16> { static constexpr int value = SPQR_F16; };
template <> struct TypeOf<__bf16> { static constexpr int value = SPQR_BF16; };

// `lanes` threads a row.  MANY: rows in turn; the next row's terms are on their way while one is worked out (4096 gated rows of 6656: 119 us with a
// workgroup a row).
template <typename X, typename Y, bool ODD, bool MANY>
__global__ void __launch_bounds__(1024) norm_rows_kernel(spqr_residual_norm_t p, int lanes) {
  __shared__ __align__(16) float part[2][16];
  constexpr int XT = TypeOf<X>::value, YT = TypeOf<Y>::value;
  const int n = p.width, in_row = threadIdx.x & (lanes - 1), per = blockDim.x / lanes, mine = threadIdx.x / lanes;
  const bool has_x = p.x != nullptr, has_y = p.y != nullptr, has_gate = p.gate != nullptr;
  Place at;
  at.col = 8 * in_row;
  at.count = min(max(n - at.col, 0), 8);
  at.from = min(at.col, n - 8);
  at.shift = at.count > 0 ? at.col - at.from : 0;
  RowSum sum{part, lanes, 0};
  int64_t first = (int64_t)blockIdx.x * per, t = min(first + mine, (int64_t)p.rows - 1);
  Raw y, x, g;
  auto load_row = [&](int64_t t, bool gate) {
    if (has_y) load(y, YT, p.y, t * p.y_stride + at.from);
    if (has_x) load(x, XT, p.x, t * p.x_stride + at.from);
    if (gate) load(g, p.gate_dtype, p.gate, t * p.gate_stride + at.from);
  };
  auto load_vectors = [&](Raw& w, Raw& b, const void* weight, const void* bias) {
    if (weight) load(w, p.weight_dtype, weight, at.from);
    if (bias) load(b, p.weight_dtype, bias, at.from);
  };
  load_row(t, has_gate);
  for (; first < p.rows; first += (int64_t)gridDim.x * per) {
    const bool live = first + mine < p.rows;     // (other threads take part in the sums, and store nothing)
    const int64_t here = t;
    float v[8], xs[8], f[8];
    Raw w, b;
    load_vectors(w, b, p.y_weight, p.y_bias);
    if (has_y) floats_at<ODD>(y, YT, at, v);
    if (has_x) floats_at<ODD>(x, XT, at, xs);
    if (has_gate) floats_at<ODD>(g, p.gate_dtype, at, f);
    const int64_t next = first + (int64_t)gridDim.x * per;
    if (MANY && next < p.rows) {
      t = min(next + mine, (int64_t)p.rows - 1);
      load_row(t, has_gate && p.gate_stride != 0);         // (one gate for all rows stays in its registers)
    }
    if (has_y) {
      norm_rows<ODD>(p.norm_y, v, at, p, p.y_weight, p.y_bias, w, b, sum);
      if (has_gate) {
        if (p.act == SPQR_ACT_SIGMOID) {
#pragma unroll
          for (int e = 0; e < 8; ++e) f[e] = activated(SPQR_ACT_SIGMOID, f[e]);
        } else if (p.act != SPQR_ACT_NONE) {
#pragma unroll
          for (int e = 0; e < 8; ++e) f[e] = activated(p.act, f[e]);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= f[e];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] *= p.scale;
    }
    load_vectors(w, b, p.x_weight, p.x_bias);
    if (has_x)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = has_y ? fmaf(p.skip, xs[e], v[e]) : p.skip * xs[e];
    if (p.sum && live && at.count > 0) store_row8_as(XT, p.sum, here * p.sum_stride, at.col, n, v);
    if (p.out) {
      norm_rows<ODD>(p.norm_x, v, at, p, p.x_weight, p.x_bias, w, b, sum);
      if (live && at.count > 0) store_row8_as(p.out_dtype, p.out, here * p.out_stride, at.col, n, v);
    }
    if (!MANY) return;
  }
}

// Threads that run at once: of the kernel with a row a workgroup (59 to 67 registers), of the one with rows in turn (97 to 126; as many as of the
// other are two sets of workgroups, the second without a row on its way: 4096 rows of 6656 83 us in place of 81, 1030 of 8192 25 in place of 23.6).
constexpr int64_t kThreads = 512 * 1024, kThreadsInTurn = 256 * 1024;

template <typename X, typename Y, bool ODD>
static void launch_rows(const spqr_residual_norm_t& p, int lanes, int threads, int64_t groups, hipStream_t st) {
  if (groups <= kThreads / threads) hipLaunchKernelGGL((norm_rows_kernel<X, Y, ODD, false>), dim3((unsigned)groups), dim3(threads), 0, st, p, lanes);
  else hipLaunchKernelGGL((norm_rows_kernel<X, Y, ODD, true>), dim3((unsigned)(kThreadsInTurn / threads)), dim3(threads), 0, st, p, lanes);
}

template <typename X, bool ODD>
static void launch_rows_of(const spqr_residual_norm_t& p, int lanes, int threads, int64_t groups, hipStream_t st) {
  if (!p.y || p.y_dtype == SPQR_F32) launch_rows<X, float, ODD>(p, lanes, threads, groups, st);
  else if (p.y_dtype == SPQR_F16) launch_rows<X, _Float16, ODD>(p, lanes, threads, groups, st);
  else launch_rows<X, __bf16, ODD>(p, lanes, threads, groups, st);
}

template <typename X>
static void launch_rows_any(const spqr_residual_norm_t& p, int lanes, int threads, int64_t groups, hipStream_t st) {
  if (p.width % 8 == 0) launch_rows_of<X, false>(p, lanes, threads, groups, st);
  else launch_rows_of<X, true>(p, lanes, threads, groups, st);
}

// ---------------------------------------------------------------------------------------------------------------------
// Longer rows, rows of fewer than eight elements, and an eps below 2^-126.
// ---------------------------------------------------------------------------------------------------------------------
template <int CH>
__device__ __forceinline__ void norm(int kind, float (&v)[CH][8], const int (&at)[CH], int n, float eps, int weight_dtype, float offset,
                                     const void* weight, const void* bias, RowSum& row_sum) {
  if (kind == SPQR_NORM_NONE) return;
  float mean = 0.f;
  if (kind == SPQR_NORM_LAYER) {
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += v[c][e];
    mean = row_sum(sum) / (float)n;
  }
  float squares = 0.f;
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[c][e] = at[c] + e < n ? v[c][e] - mean : 0.f;
      squares = fmaf(v[c][e], v[c][e], squares);
    }
  const float r = 1.f / sqrtf(row_sum(squares) / (float)n + eps);
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
    if (CH > 2) __builtin_amdgcn_sched_barrier(0);         // (registers)
  }
}

// `lanes` threads a row, CH runs of eight elements each, kept from the loads to the stores: in registers up to four runs (32768 elements), a good
// part of eight in memory (760 bytes a lane).  first: of the launch's workgroups.
template <int CH>
__global__ void __launch_bounds__(1024) residual_norm_kernel(spqr_residual_norm_t p, int lanes, int64_t first) {
  __shared__ __align__(16) float part[2][16];
  RowSum row_sum{part, lanes, 0};
  const int n = p.width, in_row = threadIdx.x & (lanes - 1);
  const int64_t row = (first + blockIdx.x) * (blockDim.x / lanes) + threadIdx.x / lanes;
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
    norm<CH>(p.norm_y, v, at, n, p.eps, p.weight_dtype, p.weight_offset, p.y_weight, p.y_bias, row_sum);
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
      if (CH > 2) __builtin_amdgcn_sched_barrier(0);
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
    if (CH > 2) __builtin_amdgcn_sched_barrier(0);
  }
  if (!p.out) return;
  norm<CH>(p.norm_x, v, at, n, p.eps, p.weight_dtype, p.weight_offset, p.x_weight, p.x_bias, row_sum);
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
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const int ch = (runs + lanes - 1) / lanes;
  // (The card's inverse root takes subnormal numbers for 0: with an eps that keeps nothing from being one, the other kernel's division and root.  A
  // case of it beside the inverse root cost 4096 gated rows 1 to 3 us.)
  if (ch <= 1 && p->width >= 8 && p->eps >= 0x1p-126f) {
    if ((!p->x && !p->sum) || p->x_dtype == SPQR_F32) launch_rows_any<float>(*p, lanes, threads, grid, st);
    else if (p->x_dtype == SPQR_F16) launch_rows_any<_Float16>(*p, lanes, threads, grid, st);
    else launch_rows_any<__bf16>(*p, lanes, threads, grid, st);
    return launched();
  }
  // 2^31 threads a launch (a grid of 2^32 threads in one direction loses what is beyond them, without an error)
  for (int64_t first = 0; first < grid; first += 1 << 21) {
    const dim3 g((unsigned)(grid - first < 1 << 21 ? grid - first : 1 << 21)), b(threads);
    if (ch <= 1) hipLaunchKernelGGL(residual_norm_kernel<1>, g, b, 0, st, *p, lanes, first);
    else if (ch <= 2) hipLaunchKernelGGL(residual_norm_kernel<2>, g, b, 0, st, *p, lanes, first);
    else if (ch <= 4) hipLaunchKernelGGL(residual_norm_kernel<4>, g, b, 0, st, *p, lanes, first);
    else hipLaunchKernelGGL(residual_norm_kernel<8>, g, b, 0, st, *p, lanes, first);
  }
  return launched();
}
