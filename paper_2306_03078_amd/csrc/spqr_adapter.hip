// Low-rank adapters of many requests beside the projections that share an input: a step's rows by adapter (spqr_adapter_plan),
// B (A x) added to the projections' rows (spqr_adapters).
#include "spqr_block.h"

namespace spqr_blk {

constexpr int kTile = SPQR_ADAPTER_TILE;

// ---------------------------------------------------------------------------------------------------------------------
// A step's rows by adapter.
// ---------------------------------------------------------------------------------------------------------------------
// Bounds that are no ascending ones may name a row more than once: then there are more rows than the arrays have room for (2^30 at
// most), and what is behind their end is left out.
//
// A workgroup a slot (the last one: rows of no adapter).  Each counts the rows of all slots for itself, which gives the tiles before
// its own, then walks through the requests in order and writes its rows.
__global__ void __launch_bounds__(256) adapter_plan_kernel(spqr_adapter_plan_t p) {
  __shared__ int rows_of[SPQR_MAX_SLOTS + 1];
  __shared__ int part[4][3];
  __shared__ int wave_rows[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, slot = blockIdx.x, S = p.slots;
  auto slot_of = [&](int i) { const int a = p.adapter[i]; return a >= 0 && a < S ? a : S; };
  auto rows_at = [&](int i, int* first) {
    if (!p.q_start) { *first = i; return i < p.rows ? 1 : 0; }
    const int lo = min(max(p.q_start[i], 0), p.rows), hi = min(max(p.q_start[i + 1], 0), p.rows);
    *first = lo;
    return max(0, hi - lo);
  };
  for (int s = tid; s <= S; s += 256) rows_of[s] = 0;
  __syncthreads();
  for (int i = tid; i < p.requests; i += 256) {
    int first;
    const int rows = rows_at(i, &first);
    if (rows > 0) atomicAdd(&rows_of[slot_of(i)], rows);
  }
  __syncthreads();
  int before = 0, all = 0;
  for (int s = tid; s <= S; s += 256) {
    const int tiles = (rows_of[s] + kTile - 1) / kTile;
    all += tiles;
    if (s < slot) before += tiles;
  }
  for (int d = 32; d > 0; d >>= 1) { before += __shfl_xor(before, d); all += __shfl_xor(all, d); }
  if (lane == 0) { part[wave][0] = before; part[wave][1] = all; }
  __syncthreads();
  before = part[0][0] + part[1][0] + part[2][0] + part[3][0];
  all = min(part[0][1] + part[1][1] + part[2][1] + part[3][1], p.max_tiles);
  const int rows = rows_of[slot], tiles = (rows + kTile - 1) / kTile;
  if (slot == 0 && tid == 0) p.count[0] = all;
  // behind the last tile: shared out
  for (int64_t t = all + slot; t < p.max_tiles; t += S + 1) {
    if (tid < 2) p.tile[2 * t + tid] = tid == 0 ? -1 : 0;
    if (tid < kTile) p.row[t * kTile + tid] = -1;
  }
  for (int t = tid; t < tiles; t += 256)
    if (before + t < p.max_tiles) {
      p.tile[2 * (before + t)] = slot < S ? slot : -1;
      p.tile[2 * (before + t) + 1] = min(kTile, rows - kTile * t);
    }
  if (rows == 0) return;
  const int64_t base = (int64_t)before * kTile, room = (int64_t)p.max_tiles * kTile;
  if (rows % kTile != 0 && tid < kTile && tid >= rows % kTile && base + (int64_t)(tiles - 1) * kTile + tid < room)
    p.row[base + (int64_t)(tiles - 1) * kTile + tid] = -1;
  int64_t done = base;
  for (int i0 = 0; i0 < p.requests; i0 += 256) {
    const int i = i0 + tid;
    int first = 0, mine = 0;
    if (i < p.requests && slot_of(i) == slot) mine = rows_at(i, &first);
    int sum = mine;                              // of the lanes up to this one
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(sum, d);
      if (lane >= d) sum += o;
    }
    if (lane == 63) wave_rows[wave] = sum;
    __syncthreads();
    int64_t to = done + sum - mine;
    for (int w = 0; w < wave; ++w) to += wave_rows[w];
    const int fit = (int)min((int64_t)mine, room - to);
    for (int k = 0; k < fit; ++k) p.row[to + k] = first + k;
    done += wave_rows[0] + wave_rows[1] + wave_rows[2] + wave_rows[3];
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------------------------------------------------
// The adapters.
// ---------------------------------------------------------------------------------------------------------------------
__device__ __forceinline__ int tile_of(const spqr_adapter_plan_t& plan, const spqr_adapters_t& a, int t, int* rows) {
  const int slot = plan.tile[2 * t];
  *rows = min(max(plan.tile[2 * t + 1], 0), kTile);
  return slot >= 0 && slot < a.slots ? slot : -1;
}
__device__ __forceinline__ int rank_of(const spqr_adapters_t& a, int p, int slot) {
  return a.rank[p] ? min(max(a.rank[p][slot], 0), a.max_rank[p]) : a.max_rank[p];
}

typedef float f32x4 __attribute__((ext_vector_type(4)));
template <typename T> struct __attribute__((packed, aligned(sizeof(T)))) Run4 { T e[4]; };
template <typename T> using x8 = T __attribute__((ext_vector_type(8)));

__device__ __forceinline__ f32x4 mfma(x8<_Float16> a, x8<_Float16> b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mfma(x8<__bf16> a, x8<__bf16> b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// Eight neighbouring elements of a row of n from k on, zeros behind its end.
template <typename T>
__device__ __forceinline__ x8<T> operand(const T* row, int k) {
  const Run8<T> r = *reinterpret_cast<const Run8<T>*>(row + k);
  return __builtin_bit_cast(x8<T>, r);
}
template <typename T>
__device__ __forceinline__ x8<T> operand_to(const T* row, int k, int n) {
  if (k + 8 <= n) return operand(row, k);
  x8<T> v;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = k + e < n ? row[k + e] : (T)0.f;
  return v;
}

constexpr int kGroup = 64;                       // ranks that a workgroup takes at once
constexpr int kUnit = 64;                        // elements of a row of x that a wavefront takes at once: two products, 128 bytes of a row
constexpr int kMostSplits = 16;
constexpr int kShrinkGroups = 512;               // workgroups that A x is split into where tiles are few

// How a call is cut: into how many parts the sum over the elements of x, for the tiles that there are (no fewer than the step's rows may
// have, which the workspace is made for).
struct Cut {
  int groups;                                    // of up to 64 ranks, of all projections
  int units;                                     // of the elements of x
  int total;                                     // floats of a row of A x: ranks rounded up to 16
  __host__ __device__ int splits(int there, int rows) const {
    const int full = (rows + kTile - 1) / kTile, tiles = there > full ? there : full;
    const int by_work = kShrinkGroups / (tiles * groups > 0 ? tiles * groups : 1), by_units = (units + 3) / 4;
    const int s = by_work < by_units ? by_work : by_units;
    return s < 1 ? 1 : s < kMostSplits ? s : kMostSplits;
  }
};
__host__ __device__ inline int padded(int rank) { return (rank + 15) / 16 * 16; }

// v[split][row][offset of p + k] = the split's part of A_p[slot][k] . x[row], NR * 16 ranks of up to NS * 16 rows: 16 ranks x 32 elements
// times 32 elements x 16 rows a product, operands straight from memory.  The workgroup's wavefronts take units in turn and add up in LDS.
template <typename T, int NR, int NS>
__device__ __forceinline__ void shrink_tile(const T* A, int64_t a_stride, int ranks, const T* x, int64_t x_stride, int n, const int32_t* row, int rows,
                                            int u0, int u1, float* v, int total, f32x4* red) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, g = lane >> 4;
  const T *ap[NR], *xp[NS];
  int64_t at[NS];
#pragma unroll
  for (int r = 0; r < NR; ++r) ap[r] = A + min(16 * r + l16, ranks - 1) * a_stride;
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    at[s] = row[min(16 * s + l16, rows - 1)];
    xp[s] = x + at[s] * x_stride;
  }
  f32x4 acc[NR][NS];
#pragma unroll
  for (int r = 0; r < NR; ++r)
#pragma unroll
    for (int s = 0; s < NS; ++s) acc[r][s] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto add = [&](auto load, int u) {
    x8<T> a[2][NR], b[2][NS];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int k = kUnit * u + 32 * h + 8 * g;
#pragma unroll
      for (int r = 0; r < NR; ++r) a[h][r] = load(ap[r], k);
#pragma unroll
      for (int s = 0; s < NS; ++s) b[h][s] = load(xp[s], k);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int s = 0; s < NS; ++s) acc[r][s] = mfma(a[h][r], b[h][s], acc[r][s]);
  };
  int u = u0 + wave;
  for (; u < u1 && kUnit * (u + 1) <= n; u += 4) add([](const T* p, int k) { return operand(p, k); }, u);
  for (; u < u1; u += 4) add([&](const T* p, int k) { return operand_to(p, k, n); }, u);
#pragma unroll
  for (int r = 0; r < NR; ++r)
#pragma unroll
    for (int s = 0; s < NS; ++s) red[(wave * NR * NS + r * NS + s) * 64 + lane] = acc[r][s];
  __syncthreads();
  for (int i = wave; i < NR * NS; i += 4) {
    const int r = i / NS, s = i % NS;
    f32x4 sum = red[i * 64 + lane];
    for (int w = 1; w < 4; ++w) sum += red[(w * NR * NS + i) * 64 + lane];
    const int token = 16 * s + l16;
    if (token < rows && 16 * r < ranks) *reinterpret_cast<f32x4*>(v + (int64_t)row[token] * total + 16 * r + 4 * g) = sum;
  }
  __syncthreads();
}

template <typename T, int NR>
__device__ __forceinline__ void shrink_rows(const T* A, int64_t a_stride, int ranks, const T* x, int64_t x_stride, int n, const int32_t* row, int rows,
                                            int u0, int u1, float* v, int total, f32x4* red) {
  if (rows <= 16) shrink_tile<T, NR, 1>(A, a_stride, ranks, x, x_stride, n, row, rows, u0, u1, v, total, red);
  else if (rows <= 32) shrink_tile<T, NR, 2>(A, a_stride, ranks, x, x_stride, n, row, rows, u0, u1, v, total, red);
  else shrink_tile<T, NR, 4>(A, a_stride, ranks, x, x_stride, n, row, rows, u0, u1, v, total, red);
}

// The tile's rows into LDS; entries that are no rows of the step end it.
__device__ __forceinline__ int rows_of_tile(const spqr_adapter_plan_t& plan, int t, int rows, int32_t* row) {
  if (threadIdx.x < kTile) row[threadIdx.x] = plan.row[(int64_t)t * kTile + threadIdx.x];
  __syncthreads();
  const int bad = threadIdx.x < rows && (row[threadIdx.x & (kTile - 1)] < 0 || row[threadIdx.x & (kTile - 1)] >= plan.rows);
  return __syncthreads_or(bad) ? 0 : rows;
}

template <typename T>
__global__ void __launch_bounds__(256) shrink_kernel(spqr_adapters_t a, spqr_adapter_plan_t plan, Cut cut, float* v) {
  __shared__ f32x4 red[4 * 16 * 64];
  __shared__ int32_t row[kTile];
  const int tiles = min(plan.count[0], plan.max_tiles), splits = cut.splits(tiles, plan.rows);
  const int64_t items = (int64_t)tiles * cut.groups * splits;
  for (int64_t i = blockIdx.x; i < items; i += gridDim.x) {
    const int group = (int)(i % cut.groups), t = (int)(i / cut.groups % tiles), split = (int)(i / cut.groups / tiles);
    int rows, p = 0, g = group, at = 0;
    const int slot = tile_of(plan, a, t, &rows);
    for (; g >= (a.max_rank[p] + kGroup - 1) / kGroup; ++p) { g -= (a.max_rank[p] + kGroup - 1) / kGroup; at += padded(a.max_rank[p]); }
    const int ranks = slot < 0 ? 0 : min(rank_of(a, p, slot) - kGroup * g, kGroup);
    if (ranks <= 0) continue;
    rows = rows_of_tile(plan, t, rows, row);
    if (rows == 0) continue;
    const T* A = static_cast<const T*>(a.A[p]) + ((int64_t)slot * a.max_rank[p] + kGroup * g) * a.width;
    const T* x = static_cast<const T*>(a.x);
    float* to = v + (int64_t)split * plan.rows * cut.total + at + kGroup * g;
    const int u0 = (int)((int64_t)cut.units * split / splits), u1 = (int)((int64_t)cut.units * (split + 1) / splits);
    if (ranks <= 16) shrink_rows<T, 1>(A, a.width, ranks, x, a.x_stride, a.width, row, rows, u0, u1, to, cut.total, red);
    else if (ranks <= 32) shrink_rows<T, 2>(A, a.width, ranks, x, a.x_stride, a.width, row, rows, u0, u1, to, cut.total, red);
    else shrink_rows<T, 4>(A, a.width, ranks, x, a.x_stride, a.width, row, rows, u0, u1, to, cut.total, red);
  }
}

// A x as it meets B: v = the sum of PARTS values of 16 bits.  Binary16 holds 22 bits in two, with the row's largest element brought to 2^13
// .. 2^14, so that what is 2^-27 of it still has its bits and none overflows; bfloat16 24 bits in three, at any size.
template <typename T> struct Parts;
template <> struct Parts<_Float16> { static constexpr int N = 2; };
template <> struct Parts<__bf16> { static constexpr int N = 3; };

constexpr int kOutTile = 256;                    // elements of the outputs' rows that a workgroup takes

// out[row][m] = y[row][m] + factor[row] * sum_k B[m][k] v[row][k] for 64 m of each wavefront, up to NS * 16 rows; 64 ranks at a time.
template <typename T, typename Y, int NS>
__device__ __forceinline__ void expand_tile(const T* B, int b_stride, int rank, float scale, int m0, int M, const Y* y, int64_t y_stride, Y* out,
                                            int64_t out_stride, const int32_t* row, int rows, const float* v, int total, int64_t v_split, int splits,
                                            x8<T>* vs, float* factor) {
  constexpr int N = Parts<T>::N, MT = 4, PER = 16 / NS;    // threads a row
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15, g = lane >> 4;
  const int m_wave = m0 + 64 * wave;
  f32x4 acc[MT][NS];
#pragma unroll
  for (int j = 0; j < MT; ++j)
#pragma unroll
    for (int s = 0; s < NS; ++s) acc[j][s] = f32x4{0.f, 0.f, 0.f, 0.f};
  // thread: row tid / PER of the tile, ranks 4 * NS * (tid % PER) .. of a group
  const int token = tid / PER, mine = 4 * NS * (tid % PER);
  const bool there = token < rows;
  const float* vr = v + (there ? (int64_t)row[token] * total : 0);
  auto sums = [&](int k0, f32x4 (&x)[NS]) {
#pragma unroll
    for (int i = 0; i < NS; ++i) x[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (!there) return;
#pragma unroll 4
    for (int s = 0; s < splits; ++s)
#pragma unroll
      for (int i = 0; i < NS; ++i)
        if (k0 + mine + 4 * i < rank) x[i] += *reinterpret_cast<const f32x4*>(vr + s * v_split + k0 + mine + 4 * i);
#pragma unroll
    for (int i = 0; i < NS; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (k0 + mine + 4 * i + e >= rank) x[i][e] = 0.f;
  };
  float up = 1.f;                                // what the row is multiplied with
  if (N == 2) {
    float top = 0.f;
    for (int k0 = 0; k0 < rank; k0 += kGroup) {
      f32x4 x[NS];
      sums(k0, x);
#pragma unroll
      for (int i = 0; i < NS; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) top = fmaxf(top, fabsf(x[i][e]));
    }
#pragma unroll
    for (int d = 1; d < PER; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
    const int e = (int)(__float_as_uint(top) >> 23) - 127;                                 // of its leading bit
    if (e < 128) up = __uint_as_float((uint32_t)(127 + 13 - max(e, -100)) << 23);
  }
  if (tid % PER == 0) factor[token] = scale / up;
  for (int k0 = 0; k0 < rank; k0 += kGroup) {
    x8<T> w[2][MT];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int k = k0 + 32 * h + 8 * g;
      const T* b = B + k;
#pragma unroll
      for (int j = 0; j < MT; ++j) {
        w[h][j] = x8<T>{};
        const int64_t m = min(m_wave + 16 * j + l16, M - 1);
        if (k < rank) w[h][j] = operand_to(b + m * b_stride, 0, rank - k);
      }
    }
    f32x4 x[NS];
    sums(k0, x);
    if (k0 > 0) __syncthreads();                 // everyone is done with the last ranks
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      const int k = mine + 4 * i;
      T* to = reinterpret_cast<T*>(vs + ((k >> 5) * NS + (token >> 4)) * 64 + (k >> 3 & 3) * 16 + (token & 15)) + (k & 7);
      f32x4 rest = x[i] * up;
#pragma unroll
      for (int part = 0; part < N; ++part) {
        Run4<T> piece;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          piece.e[e] = (T)rest[e];
          rest[e] -= (float)piece.e[e];
        }
        *reinterpret_cast<Run4<T>*>(to + part * 2 * NS * 64 * 8) = piece;
      }
    }
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (k0 + 32 * h < rank)
#pragma unroll
        for (int part = 0; part < N; ++part)
#pragma unroll
          for (int s = 0; s < NS; ++s) {
            const x8<T> b = vs[((part * 2 + h) * NS + s) * 64 + lane];
#pragma unroll
            for (int j = 0; j < MT; ++j) acc[j][s] = mfma(w[h][j], b, acc[j][s]);
          }
  }
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    const int token = 16 * s + l16;
    if (token >= rows) continue;
    const int64_t t = row[token];
    const float f = factor[token];
#pragma unroll
    for (int j = 0; j < MT; ++j) {
      const int m = m_wave + 16 * j + 4 * g;
      if (m + 4 <= M) {
        Run4<Y> o;
        if (y) o = *reinterpret_cast<const Run4<Y>*>(y + t * y_stride + m);
#pragma unroll
        for (int e = 0; e < 4; ++e) o.e[e] = (Y)fmaf(f, acc[j][s][e], y ? (float)o.e[e] : 0.f);
        *reinterpret_cast<Run4<Y>*>(out + t * out_stride + m) = o;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (m + e < M) out[t * out_stride + m + e] = (Y)fmaf(f, acc[j][s][e], y ? (float)y[t * y_stride + m + e] : 0.f);
      }
    }
  }
}

// Rows that no adapter changes.
template <typename Y>
__device__ __forceinline__ void copy_tile(int m0, int M, const Y* y, int64_t y_stride, Y* out, int64_t out_stride, const int32_t* row, int rows) {
  if (y == out && y_stride == out_stride) return;
  const int m = m0 + threadIdx.x;
  if (m >= M) return;
  for (int i = 0; i < rows; ++i) out[row[i] * out_stride + m] = y ? y[row[i] * y_stride + m] : (Y)0.f;
}

template <typename T, typename Y>
__global__ void __launch_bounds__(256) expand_kernel(spqr_adapters_t a, spqr_adapter_plan_t plan, Cut cut, const float* v, int out_tiles) {
  __shared__ x8<T> vs[Parts<T>::N * 2 * 4 * 64];
  __shared__ float factor[kTile];
  __shared__ int32_t row[kTile];
  const int tiles = min(plan.count[0], plan.max_tiles), splits = cut.splits(tiles, plan.rows);
  for (int64_t i = blockIdx.x; i < (int64_t)tiles * out_tiles; i += gridDim.x) {
    const int t = (int)(i / out_tiles);
    int rows, p = 0, c = (int)(i % out_tiles), at = 0;
    const int slot = tile_of(plan, a, t, &rows);
    for (; c >= (a.m[p] + kOutTile - 1) / kOutTile; ++p) { c -= (a.m[p] + kOutTile - 1) / kOutTile; at += padded(a.max_rank[p]); }
    const int rank = slot < 0 ? 0 : rank_of(a, p, slot), M = a.m[p];
    __syncthreads();                             // everyone is done with the last tile
    rows = rows_of_tile(plan, t, rows, row);
    const Y* y = static_cast<const Y*>(a.y[p]);
    Y* out = static_cast<Y*>(a.out[p]);
    if (rank <= 0) {
      copy_tile(kOutTile * c, M, y, a.y_stride[p], out, a.out_stride[p], row, rows);
      continue;
    }
    const T* B = static_cast<const T*>(a.B[p]) + (int64_t)slot * M * a.max_rank[p];
    const float scale = a.scale[p] ? a.scale[p][slot] : 1.f;
    const int64_t v_split = (int64_t)plan.rows * cut.total;
#define SPQR_EXPAND(NS) expand_tile<T, Y, NS>(B, a.max_rank[p], rank, scale, kOutTile * c, M, y, a.y_stride[p], out, a.out_stride[p], row, rows, v + at, cut.total, v_split, splits, vs, factor)
    if (rows <= 16) SPQR_EXPAND(1);
    else if (rows <= 32) SPQR_EXPAND(2);
    else SPQR_EXPAND(4);
#undef SPQR_EXPAND
  }
}

static int check_bank(const spqr_adapters_t* a) {
  if (!a) return SPQR_ERR_NULL;
  if (a->count < 1 || a->count > SPQR_MAX_FUSED) return SPQR_ERR_PARAM;
  if (a->width < 1 || a->width > SPQR_MAX_WIDTH) return SPQR_ERR_SHAPE;
  for (int p = 0; p < a->count; ++p)
    if (a->max_rank[p] < 1 || a->max_rank[p] > SPQR_MAX_RANK) return SPQR_ERR_PARAM;
  return SPQR_OK;
}

static Cut cut_of(const spqr_adapters_t* a) {
  Cut c{0, (a->width + kUnit - 1) / kUnit, 0};
  for (int p = 0; p < a->count; ++p) {
    c.groups += (a->max_rank[p] + kGroup - 1) / kGroup;
    c.total += padded(a->max_rank[p]);
  }
  return c;
}

template <typename T, typename Y>
static int launch_adapters(const spqr_adapters_t& a, const spqr_adapter_plan_t& plan, int tiles, hipStream_t st) {
  float* v = static_cast<float*>(a.workspace);
  const Cut cut = cut_of(&a);
  int out_tiles = 0;
  for (int p = 0; p < a.count; ++p) out_tiles += (a.m[p] + kOutTile - 1) / kOutTile;
  // As many workgroups as the most tiles there can be give work; those that are too many end at once.
  const int64_t shrink = (int64_t)tiles * cut.groups, expand = (int64_t)tiles * out_tiles;
  const int shrink_grid = (int)(shrink < kShrinkGroups ? shrink * kMostSplits < kShrinkGroups ? shrink * kMostSplits : kShrinkGroups : shrink < 65536 ? shrink : 65536);
  hipLaunchKernelGGL((shrink_kernel<T>), dim3(shrink_grid), dim3(256), 0, st, a, plan, cut, v);
  hipLaunchKernelGGL((expand_kernel<T, Y>), dim3((unsigned)(expand < 65536 ? expand : 65536)), dim3(256), 0, st, a, plan, cut, v, out_tiles);
  return launched();
}

template <typename T>
static int launch_for(const spqr_adapters_t& a, const spqr_adapter_plan_t& plan, int tiles, hipStream_t st) {
  if (a.y_dtype == SPQR_F32) return launch_adapters<T, float>(a, plan, tiles, st);
  if (a.y_dtype == SPQR_F16) return launch_adapters<T, _Float16>(a, plan, tiles, st);
  return launch_adapters<T, __bf16>(a, plan, tiles, st);
}

}  // namespace spqr_blk

using namespace spqr_blk;

extern "C" int32_t spqr_adapter_tiles(int32_t rows, int32_t slots) {
  if (rows < 0 || rows > SPQR_MAX_ROWS || slots < 1 || slots > SPQR_MAX_SLOTS) return SPQR_ERR_SHAPE;
  const int32_t most = rows / kTile + slots + 1;
  return rows < most ? rows : most;
}

// The sizes and arrays that both calls look at.
static int check_plan(const spqr_adapter_plan_t* p) {
  if (!p) return SPQR_ERR_NULL;
  const int32_t tiles = spqr_adapter_tiles(p->rows, p->slots);
  if (tiles < 0) return tiles;
  if (p->rows == 0) return SPQR_OK;
  if (p->max_tiles < tiles) return SPQR_ERR_SIZE;
  if (!p->count || !p->tile || !p->row) return SPQR_ERR_NULL;
  return aligned(p->count, 4) && aligned(p->tile, 4) && aligned(p->row, 4) ? SPQR_OK : SPQR_ERR_ALIGN;
}

extern "C" int spqr_adapter_plan(const spqr_adapter_plan_t* p, void* stream) {
  const int rc = check_plan(p);
  if (rc) return rc;
  if (p->q_start ? p->requests < 0 || p->requests > SPQR_MAX_REQUESTS : p->requests != p->rows) return SPQR_ERR_SHAPE;
  if (p->rows == 0) return SPQR_OK;
  if (!p->adapter) return SPQR_ERR_NULL;
  if (!aligned(p->adapter, 4) || !aligned(p->q_start, 4)) return SPQR_ERR_ALIGN;
  hipLaunchKernelGGL(adapter_plan_kernel, dim3(p->slots + 1), dim3(256), 0, static_cast<hipStream_t>(stream), *p);
  return launched();
}

extern "C" int64_t spqr_adapters_workspace_bytes(const spqr_adapters_t* a, int32_t rows) {
  const int rc = check_bank(a);
  if (rc) return rc;
  if (rows < 0 || rows > SPQR_MAX_ROWS) return SPQR_ERR_SHAPE;
  // as many parts of the sums as steps of up to so many rows are cut into
  const Cut cut = cut_of(a);
  int64_t most = 0;
  for (int64_t n = rows; n > 0; n = (n + kTile - 1) / kTile - 1 > 0 ? ((n + kTile - 1) / kTile - 1) * kTile : 0) {
    const int64_t floats = n * cut.splits(1, (int)n);
    most = floats > most ? floats : most;
  }
  return (most * cut.total * 4 + 255) / 256 * 256;
}

extern "C" int spqr_adapters(const spqr_adapters_t* a, const spqr_adapter_plan_t* plan, void* stream) {
  int rc = check_bank(a);
  if (!rc) rc = check_plan(plan);
  if (rc) return rc;
  if (a->slots != plan->slots) return SPQR_ERR_PARAM;
  if ((a->dtype != SPQR_F16 && a->dtype != SPQR_BF16) || !known(a->y_dtype)) return SPQR_ERR_DTYPE;
  const int rows = plan->rows;
  const int64_t most = INT64_MAX / 8 / (rows > 0 ? rows : 1);
  if (a->x_stride < a->width || a->x_stride > most) return SPQR_ERR_SHAPE;
  for (int p = 0; p < a->count; ++p)
    if (a->m[p] < 1 || a->m[p] > SPQR_MAX_WIDTH || (a->y[p] && (a->y_stride[p] < a->m[p] || a->y_stride[p] > most)) || a->out_stride[p] < a->m[p] ||
        a->out_stride[p] > most)
      return SPQR_ERR_SHAPE;
  if (rows == 0) return SPQR_OK;
  if (!a->x || !a->workspace) return SPQR_ERR_NULL;
  if (!aligned(a->x, 2) || !aligned(a->workspace, 256)) return SPQR_ERR_ALIGN;
  for (int p = 0; p < a->count; ++p) {
    if (!a->A[p] || !a->B[p] || !a->out[p]) return SPQR_ERR_NULL;
    if (!aligned(a->A[p], 2) || !aligned(a->B[p], 2) || !aligned(a->rank[p], 4) || !aligned(a->scale[p], 4) ||
        !aligned(a->y[p], size_of(a->y_dtype)) || !aligned(a->out[p], size_of(a->y_dtype)))
      return SPQR_ERR_ALIGN;
  }
  if (a->workspace_bytes < spqr_adapters_workspace_bytes(a, rows)) return SPQR_ERR_WORKSPACE;
  const int tiles = spqr_adapter_tiles(rows, plan->slots);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return a->dtype == SPQR_F16 ? launch_for<_Float16>(*a, *plan, tiles, st) : launch_for<__bf16>(*a, *plan, tiles, st);
}
