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

// v[p][row][k] = A_p[slot][k] . x[row]: a wavefront a (row, k).
template <typename T>
__global__ void __launch_bounds__(256) shrink_kernel(spqr_adapters_t a, spqr_adapter_plan_t plan, float* v, int total) {
  const int t = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (t >= min(plan.count[0], plan.max_tiles)) return;
  int rows;
  const int slot = tile_of(plan, a, t, &rows);
  if (slot < 0) return;
  int at = 0;
  for (int p = 0; p < a.count; at += a.max_rank[p], ++p) {
    const int rank = rank_of(a, p, slot);
    for (int i = wave; i < rows * rank; i += 4) {
      const int row = plan.row[(int64_t)t * kTile + i / rank], k = i % rank;
      if (row < 0 || row >= plan.rows) continue;
      const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
      const T* w = static_cast<const T*>(a.A[p]) + ((int64_t)slot * a.max_rank[p] + k) * a.width;
      float sum = 0.f;
      for (int c = 8 * lane; c < a.width; c += 512) {
        float xs[8], ws[8];
        load_row8(x, c, a.width, xs);
        load_row8(w, c, a.width, ws);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = fmaf(xs[e], ws[e], sum);
      }
      for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
      if (lane == 0) v[(int64_t)row * total + at + k] = sum;
    }
  }
}

template <typename T, typename Y>
__global__ void __launch_bounds__(256) expand_kernel(spqr_adapters_t a, spqr_adapter_plan_t plan, const float* v, int total) {
  const int t = blockIdx.x;
  if (t >= min(plan.count[0], plan.max_tiles)) return;
  int rows;
  const int slot = tile_of(plan, a, t, &rows);
  int at = 0;
  for (int p = 0; p < a.count; at += a.max_rank[p], ++p) {
    const int rank = slot < 0 ? 0 : rank_of(a, p, slot);
    const float scale = slot >= 0 && a.scale[p] ? a.scale[p][slot] : 1.f;
    for (int i = 0; i < rows; ++i) {
      const int row = plan.row[(int64_t)t * kTile + i];
      if (row < 0 || row >= plan.rows) continue;
      for (int m = blockIdx.y * 256 + threadIdx.x; m < a.m[p]; m += gridDim.y * 256) {
        const T* w = static_cast<const T*>(a.B[p]) + ((int64_t)max(slot, 0) * a.m[p] + m) * a.max_rank[p];
        const float* x = v + (int64_t)row * total + at;
        float sum = 0.f;
        for (int k = 0; k < rank; ++k) sum = fmaf(x[k], (float)w[k], sum);
        const float y = a.y[p] ? (float)(static_cast<const Y*>(a.y[p])[row * a.y_stride[p] + m]) : 0.f;
        static_cast<Y*>(a.out[p])[row * a.out_stride[p] + m] = (Y)(rank > 0 ? fmaf(scale, sum, y) : y);
      }
    }
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

static int total_rank(const spqr_adapters_t* a) {
  int total = 0;
  for (int p = 0; p < a->count; ++p) total += a->max_rank[p];
  return total;
}

template <typename T, typename Y>
static int launch_adapters(const spqr_adapters_t& a, const spqr_adapter_plan_t& plan, int tiles, hipStream_t st) {
  float* v = static_cast<float*>(a.workspace);
  const int total = total_rank(&a);
  hipLaunchKernelGGL((shrink_kernel<T>), dim3(tiles), dim3(256), 0, st, a, plan, v, total);
  hipLaunchKernelGGL((expand_kernel<T, Y>), dim3(tiles, 16), dim3(256), 0, st, a, plan, v, total);
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
  return ((int64_t)rows * total_rank(a) * 4 + 255) / 256 * 256;
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
