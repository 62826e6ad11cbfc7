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
// its own; a wavefront has an equal part of the requests, in order, counts those of the slot, and writes their rows behind those of the wavefronts
// before it.  Trips to memory and to LDS one after the other bound it: 4096 rows of 200 slots 6.0 us (256 threads, a barrier for every 256
// requests: 15.7), 64 requests of 48 slots 4.6 us; with many rows of many slots what every workgroup reads: 65536 rows of 4096 slots 316 us, 2^20 rows
// of 200 slots 650 us, of 4096 slots 6.4 ms.
constexpr int kPlanAhead = 4;

template <bool BY_ROW, int WAVES>
__global__ void __launch_bounds__(64 * WAVES) adapter_plan_kernel(spqr_adapter_plan_t p) {
  __shared__ int rows_of[SPQR_MAX_SLOTS + 1];
  __shared__ int part[WAVES][3];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, slot = blockIdx.x, S = p.slots, threads = 64 * WAVES;
  const int each = (p.requests + threads - 1) / threads * 64, i0 = min(wave * each, p.requests), i1 = min(i0 + each, p.requests);
  // a request's slot (S: none) and rows
  struct Request { int slot, first, rows; };
  auto request = [&](int i) {
    Request r{S, i, 0};
    if (i >= i1) return r;
    const int a = p.adapter[i];
    r.slot = a >= 0 && a < S ? a : S;
    if (BY_ROW) {
      r.rows = 1;
    } else {
      r.first = min(max(p.q_start[i], 0), p.rows);
      r.rows = max(0, min(max(p.q_start[i + 1], 0), p.rows) - r.first);
    }
    return r;
  };
  for (int s = tid; s <= S; s += threads) rows_of[s] = 0;
  __syncthreads();
  int own = 0;                                   // rows of the slot among the wavefront's
  for (int i = i0 + lane; i - lane < i1; i += 64 * kPlanAhead) {
    Request r[kPlanAhead];
#pragma unroll
    for (int k = 0; k < kPlanAhead; ++k) r[k] = request(i + 64 * k);
#pragma unroll
    for (int k = 0; k < kPlanAhead; ++k) {
      if (r[k].slot == slot) own += r[k].rows;
      // (rows of one slot side by side: one addition)
      const int first = __builtin_amdgcn_readfirstlane(r[k].slot);
      if (BY_ROW && __all(r[k].slot == first && r[k].rows == 1)) {
        if (lane == 0) atomicAdd(&rows_of[first], 64);
      } else if (r[k].rows > 0) {
        atomicAdd(&rows_of[r[k].slot], r[k].rows);
      }
    }
  }
  for (int d = 32; d > 0; d >>= 1) own += __shfl_xor(own, d);
  if (lane == 0) part[wave][2] = own;
  __syncthreads();
  int before = 0, all = 0;
  for (int s = tid; s <= S; s += threads) {
    const int tiles = (rows_of[s] + kTile - 1) / kTile;
    all += tiles;
    if (s < slot) before += tiles;
  }
  for (int d = 32; d > 0; d >>= 1) { before += __shfl_xor(before, d); all += __shfl_xor(all, d); }
  if (lane == 0) { part[wave][0] = before; part[wave][1] = all; }
  __syncthreads();
  before = all = 0;
  int done = 0;                                  // rows of the slot before the wavefront's
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    before += part[w][0];
    all += part[w][1];
    if (w < wave) done += part[w][2];
  }
  all = min(all, p.max_tiles);
  const int rows = rows_of[slot], tiles = (rows + kTile - 1) / kTile;
  if (slot == 0 && tid == 0) p.count[0] = all;
  // behind the last tile: shared out
  for (int64_t t = all + slot + (int64_t)wave * (S + 1); t < p.max_tiles; t += (int64_t)(S + 1) * WAVES) {
    if (lane < 2) p.tile[2 * t + lane] = lane == 0 ? -1 : 0;
    p.row[t * kTile + lane] = -1;
  }
  for (int t = tid; t < tiles; t += threads)
    if (before + t < p.max_tiles) {
      p.tile[2 * (before + t)] = slot < S ? slot : -1;
      p.tile[2 * (before + t) + 1] = min(kTile, rows - kTile * t);
    }
  const int64_t base = (int64_t)before * kTile, room = (int64_t)p.max_tiles * kTile;
  if (rows % kTile != 0 && tid < kTile && tid >= rows % kTile && base + (int64_t)(tiles - 1) * kTile + tid < room)
    p.row[base + (int64_t)(tiles - 1) * kTile + tid] = -1;
  if (own == 0) return;
  int64_t at = base + done;
  for (int i = i0 + lane; i - lane < i1; i += 64 * kPlanAhead) {
    Request r[kPlanAhead];
#pragma unroll
    for (int k = 0; k < kPlanAhead; ++k) r[k] = request(i + 64 * k);
#pragma unroll
    for (int k = 0; k < kPlanAhead; ++k) {
      const int mine = r[k].slot == slot ? r[k].rows : 0;
      if (BY_ROW) {
        const uint64_t of = __ballot(mine > 0);
        const int64_t to = at + __popcll(of & ((1ull << lane) - 1));
        if (mine > 0 && to < room) p.row[to] = r[k].first;
        at += __popcll(of);
      } else if (__any(mine > 0)) {
        int sum = mine;                          // of the lanes up to this one
        for (int d = 1; d < 64; d <<= 1) {
          const int o = __shfl_up(sum, d);
          if (lane >= d) sum += o;
        }
        // a request's rows, by all lanes
        for (uint64_t left = __ballot(mine > 0); left != 0; left &= left - 1) {
          const int l = __ffsll((unsigned long long)left) - 1, n = __shfl(mine, l), first = __shfl(r[k].first, l);
          const int64_t to = at + __shfl(sum, l) - n;
          for (int64_t m = lane; m < n && to + m < room; m += 64) p.row[to + m] = first + (int)m;
        }
        at += __shfl(sum, 63);
      }
    }
  }
}

// ---------------------------------------------------------------------------------------------------------------------
// The adapters.
// ---------------------------------------------------------------------------------------------------------------------
// Both products run on 16 x 16 x 32 matrix instructions.  An operand's lane l holds 8 values of line l & 15, so neighbouring lanes hold different
// lines, and loads of rows as they lie take a trip through the address unit for each lane (64 a load in place of 16: A x and B (A x) of 5000 rows
// were bound by it, 60 and 230 us).  A bank's weights are therefore packed, once, as operands: 64 lanes x 16 bytes one after the other, zeros
// where there is no weight.
typedef float f32x4 __attribute__((ext_vector_type(4)));
template <typename T> struct __attribute__((packed, aligned(sizeof(T)))) Run4 { T e[4]; };
template <typename T> using x8 = T __attribute__((ext_vector_type(8)));

__device__ __forceinline__ f32x4 mfma(x8<_Float16> a, x8<_Float16> b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mfma(x8<__bf16> a, x8<__bf16> b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// What is the same for all threads, by way of the scalar cache: such loads wait for nothing but each other.
template <typename V>
__device__ __forceinline__ V uniform(const V* p) {
  return *(const __attribute__((address_space(4))) V*)(uintptr_t)p;
}

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

// A projection's bank: the slots' ranks (rounded up to 256 bytes), then slot after slot
//   A: [tile of 16 ranks][step of 32 elements of x]: lane l has rank 16 * tile + (l & 15), elements 32 * step + 8 * (l >> 4) ..
//   B: [32 ranks][64 m][4: j]: lane l has m = 64 * block + 4 * (l & 15) + j, ranks 32 * h + 8 * (l >> 4) .. -- of the four results of a lane, those of j
//      0 .. 3 are neighbours, and neighbouring lanes' too.  Up to 16 ranks: [64 m][2]: lanes below 32 are the first half of j = 2 i, the others of
//      j = 2 i + 1.
struct Bank {
  int tiles, steps;                              // of 16 ranks; of 32 elements of x, a multiple of 4
  int halves, blocks;                            // of 32 ranks, 0: up to 16 ranks; of 64 m
  __host__ __device__ Bank(int width, int m, int max_rank)
      : tiles((max_rank + 15) / 16), steps((width + 127) / 128 * 4), halves(max_rank <= 16 ? 0 : (max_rank + 31) / 32), blocks((m + 63) / 64) {}
  __host__ __device__ int64_t a_operands() const { return (int64_t)tiles * steps; }
  __host__ __device__ int64_t operands() const { return a_operands() + (int64_t)blocks * (halves == 0 ? 2 : 4 * halves); }
};
__host__ __device__ inline int64_t header_bytes(int slots) { return ((int64_t)slots * 4 + 255) / 256 * 256; }

struct Pack {
  const uint16_t *A, *B;
  const int32_t* rank;
  uint8_t* bank;
  int width, m, max_rank, slots, first;
};

// A thread a lane of an operand.
__global__ void __launch_bounds__(256) pack_kernel(Pack a) {
  const Bank bank(a.width, a.m, a.max_rank);
  const int slot = blockIdx.y;                   // of those that are given
  const int rank = a.rank ? min(max(a.rank[slot], 0), a.max_rank) : a.max_rank;
  if (blockIdx.x == 0 && threadIdx.x == 0) reinterpret_cast<int32_t*>(a.bank)[a.first + slot] = rank;
  u32x4* to = reinterpret_cast<u32x4*>(a.bank + header_bytes(a.slots)) + (a.first + slot) * bank.operands() * 64;
  const uint16_t *A = a.A + (int64_t)slot * a.max_rank * a.width, *B = a.B + (int64_t)slot * a.m * a.max_rank;
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < bank.operands() * 64; i += gridDim.x * 256ll) {
    const int64_t which = i / 64;
    const int lane = (int)(i % 64), l16 = lane & 15, g = lane >> 4;
    uint16_t v[8];
    if (which < bank.a_operands()) {
      const int k = (int)(which / bank.steps) * 16 + l16, at = (int)(which % bank.steps) * 32 + 8 * g;
      for (int e = 0; e < 8; ++e) v[e] = k < rank && at + e < a.width ? A[(int64_t)k * a.width + at + e] : 0;
    } else {
      const int64_t w = which - bank.a_operands();
      int m, k;
      if (bank.halves == 0) {
        m = (int)(w / 2) * 64 + 4 * l16 + 2 * (int)(w % 2) + (g >> 1);
        k = 8 * (g & 1);
      } else {
        m = (int)(w / 4 % bank.blocks) * 64 + 4 * l16 + (int)(w % 4);
        k = (int)(w / 4 / bank.blocks) * 32 + 8 * g;
      }
      for (int e = 0; e < 8; ++e) v[e] = m < a.m && k + e < rank ? B[(int64_t)m * a.max_rank + k + e] : 0;
    }
    u32x4 x;
    for (int e = 0; e < 4; ++e) x[e] = v[2 * e] | (uint32_t)v[2 * e + 1] << 16;
    to[i] = x;
  }
}

constexpr int kStage = 128;                      // elements of x at a time
constexpr int kMostSplits = 8;
constexpr int kShrinkGroups = 512;               // workgroups that A x is split into where tiles are few
constexpr int kWaveTiles = 4;                    // tiles of 16 ranks that a wavefront takes at once

// How a call is cut: into how many parts the sum over the elements of x, for the tiles that there are (no fewer than the step's rows may
// have, which the workspace is made for).
struct Cut {
  int rank_tiles;                                // of 16 ranks, of all projections
  int rank_halves;                               // of 32 ranks, of all projections: blocks of A x
  int stages;                                    // of the elements of x
  __host__ __device__ int splits(int there, int rows) const {
    const int full = (rows + kTile - 1) / kTile, tiles = there > full ? there : full;
    const int groups = (rank_tiles + 4 * kWaveTiles - 1) / (4 * kWaveTiles);
    const int by_work = kShrinkGroups / (tiles * groups > 0 ? tiles * groups : 1), by_stages = (stages + 3) / 4;
    const int s = by_work < by_stages ? by_work : by_stages;
    return s < 1 ? 1 : s < kMostSplits ? s : kMostSplits;
  }
};

// A call as the kernels take it: what a workgroup needs of a projection lies together.
struct Projection {
  const uint8_t* bank;
  const float* scale;
  const void* y;
  void* out;
  int64_t y_stride, out_stride;
  int m, max_rank;
  int at;                                        // its first block of 32 ranks of A x
};
struct Call {
  Projection p[SPQR_MAX_FUSED];
  const void* x;
  int64_t x_stride;
  const int32_t *count, *tile, *row;
  float* v;                                      // A x: [splits][tiles][blocks of 32 ranks][16 rows: 4][lane][8], as the operands of the next product
  Cut cut;
  int width, slots, rows, max_tiles, v_tiles;
  int pieces;                                    // of 256 elements, of a row of all outputs
};
__device__ __forceinline__ float* v_of(const Call& c, int split, int tile, int half, int sub) {
  return c.v + (((int64_t)split * c.v_tiles + tile) * c.cut.rank_halves + half) * (4 * 512) + sub * 512;
}

// A tile as the kernels take it: slot -1 where no adapter (or none that the bank has) is used; rows, 0 behind the last tile; row: a lane's
// of them, -1 where there is none; count: of all tiles.
struct Tile { int slot, rows, count, row; };

__device__ __forceinline__ Tile tile_at(const Call& c, int t) {
  const int in_tile = threadIdx.x & (kTile - 1), row = c.row[(int64_t)t * kTile + in_tile];
  const int count = min(uniform(c.count), c.max_tiles), slot = uniform(c.tile + 2 * t), rows = uniform(c.tile + 2 * t + 1);
  Tile v;
  v.count = count;
  v.slot = slot >= 0 && slot < c.slots ? slot : -1;
  v.rows = t < count ? min(max(rows, 0), kTile) : 0;
  v.row = in_tile < v.rows && row >= 0 && row < c.rows ? row : -1;
  return v;
}
__device__ __forceinline__ int rank_of(const Projection& p, int slot) {
  return slot < 0 ? 0 : min(max(uniform(reinterpret_cast<const int32_t*>(p.bank) + slot), 0), p.max_rank);
}
template <typename T>
__device__ __forceinline__ const x8<T>* slot_of(const Call& c, const Projection& p, int slot) {
  return reinterpret_cast<const x8<T>*>(p.bank + header_bytes(c.slots)) + slot * Bank(c.width, p.m, p.max_rank).operands() * 64;
}

// 16 ranks of 16 rows to where the next product finds them: lane (row, 4 * g ..) of tile `tile` of the projection.
__device__ __forceinline__ void put(const Call& c, const Projection& p, int split, int t, int tile, int sub, int lane, f32x4 sum) {
  const int k = 16 * (tile & 1) + 4 * (lane >> 4);         // of the 32 ranks
  *reinterpret_cast<f32x4*>(v_of(c, split, t, p.at + tile / 2, sub) + ((k >> 3) * 16 + (lane & 15)) * 8 + (k & 7)) = sum;
}

// Up to 16 rows: NR tiles of 16 ranks of one projection, the workgroup's wavefronts take stages of 128 elements in turn and add up in LDS.  x comes
// straight from memory: few rows are few addresses.
template <typename T, int NR>
__device__ __forceinline__ void shrink_few(const Call& c, const Tile& t, const Projection& p, int tile0, int tiles, int split, int s0, int s1, f32x4* red) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, g = lane >> 4, n = c.width;
  const int steps = (n + 127) / 128 * 4;
  const x8<T>* A = slot_of<T>(c, p, t.slot) + (int64_t)tile0 * steps * 64 + lane;
  const T* x = static_cast<const T*>(c.x) + max(__shfl(t.row, min(l16, t.rows - 1)), 0) * c.x_stride;
  f32x4 acc[NR];
#pragma unroll
  for (int r = 0; r < NR; ++r) acc[r] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto add = [&](auto load, int s) {
    x8<T> a[4][NR], b[4];
#pragma unroll
    for (int h = 0; h < 4; ++h) {
#pragma unroll
      for (int r = 0; r < NR; ++r) a[h][r] = A[((int64_t)min(r, tiles - 1) * steps + 4 * s + h) * 64];
      b[h] = load(kStage * s + 32 * h + 8 * g);
    }
#pragma unroll
    for (int h = 0; h < 4; ++h)
#pragma unroll
      for (int r = 0; r < NR; ++r) acc[r] = mfma(a[h][r], b[h], acc[r]);
  };
  const int last = min(s1, n / kStage);
  int s = s0 + wave;
  for (; s < last; s += 4) add([&](int k) { return operand(x, k); }, s);
  if (s < s1) add([&](int k) { return operand_to(x, k, n); }, s);
#pragma unroll
  for (int r = 0; r < NR; ++r) red[(wave * NR + r) * 64 + lane] = acc[r];
  __syncthreads();
  for (int r = wave; r < tiles && r < NR; r += 4) {
    f32x4 sum = red[r * 64 + lane];
    for (int w = 1; w < 4; ++w) sum += red[(w * NR + r) * 64 + lane];
    put(c, p, split, blockIdx.y, tile0 + r, 0, lane, sum);
  }
}

// More rows: NS * 16 of them through LDS, a stage at a time (rows of 256 bytes, 16-byte pieces turned by the row so that 16 rows' are in all banks);
// each wavefront has NR tiles of 16 ranks of its own, of any projections, of those that the slot's ranks fill
// (all that the bank has room for, in four where three would do: 39 us in place of 35 for 5000 rows of three projections, ranks of 8 to 64).
template <typename T, int NR, int NS>
__device__ __forceinline__ void shrink_many(const Call& c, const Tile& t, const int (&tiles_of)[SPQR_MAX_FUSED], int first, int end, int split, int s0, int s1, x8<T>* xs) {
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, g = lane >> 4, n = c.width;
  const int steps = (n + 127) / 128 * 4;
  // a thread's piece of NS rows
  const int piece = tid & 15, row0 = tid >> 4;
  const T* x[NS];
#pragma unroll
  for (int i = 0; i < NS; ++i) x[i] = static_cast<const T*>(c.x) + max(__shfl(t.row, 16 * i + row0), 0) * c.x_stride + 8 * piece;
  // a wavefront's tiles; one that is none reads those of the first
  const x8<T>* A[NR];
  int of[NR], tile[NR];
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    const int i = first + wave + 4 * r;
    of[r] = 0;
    tile[r] = i < end ? i : first;
#pragma unroll
    for (int p = 0; p < SPQR_MAX_FUSED - 1; ++p)
      if (of[r] == p && tile[r] >= tiles_of[p]) { tile[r] -= tiles_of[p]; ++of[r]; }
    A[r] = slot_of<T>(c, c.p[of[r]], t.slot) + (int64_t)tile[r] * steps * 64 + lane;
  }
  f32x4 acc[NR][NS];
#pragma unroll
  for (int r = 0; r < NR; ++r)
#pragma unroll
    for (int i = 0; i < NS; ++i) acc[r][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  x8<T> next[NS];
  auto load_x = [&](int s) {
    if (kStage * (s + 1) <= n) {
#pragma unroll
      for (int i = 0; i < NS; ++i) next[i] = operand(x[i], kStage * s);
    } else {
#pragma unroll
      for (int i = 0; i < NS; ++i) next[i] = operand_to(x[i], kStage * s, n - 8 * piece);
    }
  };
  load_x(s0);
  for (int s = s0; s < s1; ++s) {
    x8<T> a[4][NR];
#pragma unroll
    for (int h = 0; h < 4; ++h)
#pragma unroll
      for (int r = 0; r < NR; ++r) a[h][r] = A[r][(4 * s + h) * 64];
    x8<T>* buffer = xs + ((s - s0) & 1) * (NS * 256);
#pragma unroll
    for (int i = 0; i < NS; ++i) buffer[(16 * i + row0) * 16 + (piece ^ row0)] = next[i];
    if (s + 1 < s1) load_x(s + 1);
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      x8<T> b[NS];
#pragma unroll
      for (int i = 0; i < NS; ++i) b[i] = buffer[(16 * i + l16) * 16 + ((4 * h + g) ^ l16)];
#pragma unroll
      for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int i = 0; i < NS; ++i) acc[r][i] = mfma(a[h][r], b[i], acc[r][i]);
    }
  }
#pragma unroll
  for (int r = 0; r < NR; ++r)
    if (first + wave + 4 * r < end) {
#pragma unroll
      for (int i = 0; i < NS; ++i) put(c, c.p[of[r]], split, blockIdx.y, tile[r], i, lane, acc[r][i]);
    }
}

template <typename T>
__global__ void __launch_bounds__(256) shrink_kernel(Call c) {
  __shared__ x8<T> shared[2 * 4 * 256];          // two stages of 64 rows; or the wavefronts' sums
  const Tile t = tile_at(c, blockIdx.y);
  const int split = (int)blockIdx.x, splits = c.cut.splits(t.count, c.rows);
  if (t.rows == 0 || t.slot < 0 || split >= splits) return;
  const int s0 = c.cut.stages * split / splits, s1 = c.cut.stages * (split + 1) / splits;
  if (t.rows <= 16) {
    // a workgroup a projection's next tiles: blockIdx.z counts tiles by four, projection by projection
    int p = 0, z = (int)blockIdx.z;
    for (; p < SPQR_MAX_FUSED && z >= (c.p[p].max_rank + 16 * kWaveTiles - 1) / (16 * kWaveTiles); ++p) z -= (c.p[p].max_rank + 16 * kWaveTiles - 1) / (16 * kWaveTiles);
    if (p == SPQR_MAX_FUSED) return;
    const int tiles = (rank_of(c.p[p], t.slot) + 15) / 16 - kWaveTiles * z;
    f32x4* red = reinterpret_cast<f32x4*>(shared);
    if (tiles <= 0) return;
    if (tiles == 1) shrink_few<T, 1>(c, t, c.p[p], kWaveTiles * z, tiles, split, s0, s1, red);
    else if (tiles == 2) shrink_few<T, 2>(c, t, c.p[p], kWaveTiles * z, tiles, split, s0, s1, red);
    else shrink_few<T, 4>(c, t, c.p[p], kWaveTiles * z, tiles, split, s0, s1, red);
    return;
  }
  int tiles_of[SPQR_MAX_FUSED], end = 0;
#pragma unroll
  for (int p = 0; p < SPQR_MAX_FUSED; ++p) {
    tiles_of[p] = (rank_of(c.p[p], t.slot) + 15) / 16;
    end += tiles_of[p];
  }
  const int first = 4 * kWaveTiles * (int)blockIdx.z, left = end - first;
  if (left <= 0) return;
#define SPQR_SHRINK(NR) do { if (t.rows <= 32) shrink_many<T, NR, 2>(c, t, tiles_of, first, end, split, s0, s1, shared); else shrink_many<T, NR, 4>(c, t, tiles_of, first, end, split, s0, s1, shared); } while (0)
  if (left <= 4) SPQR_SHRINK(1);
  else if (left <= 8) SPQR_SHRINK(2);
  else if (left <= 12) SPQR_SHRINK(3);
  else SPQR_SHRINK(4);
#undef SPQR_SHRINK
}

// A x as it meets B: v = the sum of N values of 16 bits.  Binary16 holds 22 bits in two, with the row's largest element brought to 2^13 .. 2^14,
// so that what is 2^-27 of it still has its bits and none overflows; bfloat16 24 bits in three, at any size.
template <typename T> struct Parts;
template <> struct Parts<_Float16> { static constexpr int N = 2; };
template <> struct Parts<__bf16> { static constexpr int N = 3; };

// out[row][m] = y[row][m] + factor[row] * sum_k B[m][k] v[row][k] for the m of [m0, m1) and up to 64 rows, 32 * H ranks (H = 0: 16).  The parts of v
// lie in LDS as operands, NS * 16 rows of them.  A wavefront takes 64 m at a time, four products side by side, whose results are 4 neighbouring m
// of 4 rows in every lane; the workgroup's four are neighbours, so that a row is read and written 1 KB at a time (wavefronts with rows of
// their own and 256 bytes of each: 168 us in place of 150 for 5000 rows of 8192 + 1024 + 1024 m, 64 ranks, binary32, before the split below).  The next weights and elements of y are on their way meanwhile.
// Ranks that a bank does not have (three times 32 of four) read its last ones and meet zeros.
template <typename T, typename Y, int H, int NS>
__device__ __forceinline__ void expand_rows(const Call& c, const Projection& p, const Tile& t, int tile, int sub0, int rank, int m0, int m1, f32x4* sums,
                                            x8<T>* vs, float* factors) {
  constexpr int N = Parts<T>::N, HV = H == 0 ? 1 : H, HL = H == 0 ? 2 : H;                 // operands of a row's ranks
  constexpr int CH = H <= 2 ? HV : 2, CHUNKS = HV / CH, F = H == 0 ? 2 : 4 * CH;           // weights are taken CH * 32 ranks at a time
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, g = lane >> 4;
  const Bank bank(c.width, p.m, p.max_rank);
  const x8<T>* B = slot_of<T>(c, p, t.slot) + bank.a_operands() * 64 + lane;
  const bool has_y = p.y != nullptr;
  const Y* const y = has_y ? static_cast<const Y*>(p.y) + 4 * l16 : reinterpret_cast<const Y*>(c.v);
  Y* const out = static_cast<Y*>(p.out) + 4 * l16;
  const int64_t y_stride = has_y ? p.y_stride : 0, out_stride = p.out_stride;
  int row[NS][4];
#pragma unroll
  for (int s = 0; s < NS; ++s)
#pragma unroll
    for (int i = 0; i < 4; ++i) row[s][i] = __shfl(t.row, 16 * (sub0 + s) + 4 * g + i);
  auto load_w = [&](x8<T> (&w)[F], int m, int chunk) {
    const int block = m / 64;
    if (H == 0) {
#pragma unroll
      for (int f = 0; f < F; ++f) w[f] = B[(int64_t)(2 * block + f) * 64];
    } else {
#pragma unroll
      for (int h = 0; h < CH; ++h)
#pragma unroll
        for (int j = 0; j < 4; ++j) w[4 * h + j] = B[((int64_t)min(CH * chunk + h, bank.halves - 1) * bank.blocks + block) * 256 + 64 * j];
    }
  };
  // (A row's address is worked out where it is needed: kept for all rows they would take half of the registers.)
  auto fresh = [](int row) {
    asm volatile("" : "+v"(row));
    return row;
  };
  auto load_y = [&](Run4<Y> (&before)[4], int s, int m) {
#pragma unroll
    for (int i = 0; i < 4; ++i) before[i] = *reinterpret_cast<const Run4<Y>*>(y + max(fresh(row[s][i]), 0) * y_stride + (has_y ? m : 0));
  };
  // Whole steps, then what is left.  Rows of 2^k bytes begin in the same channel of the L2, and workgroups that walk along them in step would all
  // want one: each begins somewhere else in its range.
  const int first = m0 + 64 * wave, steps = first < m1 ? (m1 - 64 - first + 256) / 256 : 0;
  const int begin = steps > 0 ? (int)(blockIdx.x * 3) % steps : 0;
  auto m_of = [&](int i) {       // begin <= i; what is behind the last step is the last one again
    const int k = min(i, begin + steps - 1);
    return first + 256 * (k < steps ? k : k - steps);
  };
  x8<T> w[F], next_w[F];
  Run4<Y> before[NS == 1 ? 2 : NS][4];           // of a step's rows (of this step's and the next's 16)
  if (steps > 0) {
    if (NS < 4) load_w(w, m_of(begin), 0);
#pragma unroll
    for (int s = 0; s < NS; ++s) load_y(before[s], s, m_of(begin));
  }
  {
    // The parts of v: 16 rows a wavefront, or of the same 16 a quarter of the sums' parts each.
    constexpr bool ALL = NS == 1;
    const int sub = ALL ? 0 : wave;
    const int splits = c.cut.splits(t.count, c.rows), left = rank - 8 * (H == 0 ? g & 1 : g), halves = (p.max_rank + 31) / 32;
    const float* v = v_of(c, 0, tile, p.at, sub0 + sub) + (H == 0 ? (g & 1) * 16 + l16 : lane) * 8;
    const int64_t v_split = (int64_t)c.v_tiles * c.cut.rank_halves * (4 * 512);
    const bool live = 16 * (sub0 + sub) + l16 < t.rows;
    f32x4 x[HV][2];
#pragma unroll
    for (int h = 0; h < HV; ++h) x[h][0] = x[h][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4 / HV
    for (int s = ALL ? wave : sub < NS ? 0 : splits; s < splits; s += ALL ? 4 : 1)
#pragma unroll
      for (int h = 0; h < HV; ++h) {
        const f32x4* from = reinterpret_cast<const f32x4*>(v + s * v_split + min(h, halves - 1) * (4 * 512));
        x[h][0] += from[0];
        x[h][1] += from[1];
      }
    if (ALL) {
#pragma unroll
      for (int h0 = 0; h0 < HV; h0 += 2) {       // 64 ranks at a time
        if (h0 > 0) __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (h0 + i / 2 < HV) sums[(4 * wave + i) * 64 + lane] = x[(h0 + i / 2) % HV][i % 2];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (h0 + i / 2 < HV) {
            f32x4 sum = sums[i * 64 + lane];
#pragma unroll
            for (int k = 1; k < 4; ++k) sum += sums[(4 * k + i) * 64 + lane];
            x[(h0 + i / 2) % HV][i % 2] = sum;
          }
      }
    }
    float top = 0.f, up = 1.f, factor = p.scale ? uniform(p.scale + t.slot) : 1.f;         // up: what the row is multiplied with
#pragma unroll
    for (int h = 0; h < HV; ++h)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (32 * h + e >= left || !live) x[h][e / 4][e % 4] = 0.f;
        top = fmaxf(top, fabsf(x[h][e / 4][e % 4]));
      }
    if (N == 2) {
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const int e = (int)(__float_as_uint(top) >> 23) - 127;                               // of its leading bit
      if (e < 128) up = __uint_as_float((uint32_t)(127 + 13 - max(e, -100)) << 23);
      factor /= up;
    }
    if (ALL ? wave == 0 : sub < NS) {
      if (lane < 16) factors[16 * sub + lane] = factor;
      x8<T>* const to = vs + sub * (N * HL * 64) + lane;
#pragma unroll
      for (int h = 0; h < HV; ++h) {
        x8<T> piece[N];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float rest = x[h][e / 4][e % 4] * up;
#pragma unroll
          for (int part = 0; part < N; ++part) {
            piece[part][e] = (T)rest;
            rest -= (float)piece[part][e];
          }
        }
#pragma unroll
        for (int part = 0; part < N; ++part) {
          if (H == 0) {                          // for the operands' halves: ranks in the lower lanes, in the upper ones
            to[(part * HL) * 64] = g < 2 ? piece[part] : x8<T>{};
            to[(part * HL + HL - 1) * 64] = g < 2 ? x8<T>{} : piece[part];
          } else {
            to[(part * HL + h) * 64] = piece[part];
          }
        }
      }
    }
    __syncthreads();
  }
  if (NS == 4 && steps > 0) load_w(w, m_of(begin), 0);
  auto multiply = [&](f32x4 (&acc)[4], const x8<T> (&w)[F], int s, int chunk) {
    const x8<T>* from = vs + s * (N * HL * 64) + lane;
#pragma unroll
    for (int h = 0; h < (H == 0 ? 1 : CH); ++h)
#pragma unroll
      for (int part = 0; part < N; ++part) {
        if (H == 0) {
          const x8<T> a = from[(part * HL) * 64], b = from[(part * HL + HL - 1) * 64];
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[j] = mfma(j & 1 ? b : a, w[(j >> 1) % F], acc[j]);
        } else {
          const x8<T> a = from[(part * HL + CH * chunk + h) * 64];
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[j] = mfma(a, w[(4 * h + j) % F], acc[j]);
        }
      }
  };
  auto zero = [](f32x4 (&acc)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  };
  auto store = [&](const f32x4 (&acc)[4], const Run4<Y> (&before)[4], int s, int m) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float f = factors[16 * s + 4 * g + i];
      Run4<Y> o;
#pragma unroll
      for (int j = 0; j < 4; ++j) o.e[j] = (Y)fmaf(f, acc[j][i], has_y ? (float)before[i].e[j] : 0.f);
      const int r = fresh(row[s][i]);
      if (r >= 0) *reinterpret_cast<Run4<Y>*>(out + r * out_stride + m) = o;
    }
  };
  // A step: its weights in w; at its end the next step's are in next_w (in w, where ranks come in chunks, and
  // with 64 rows, whose elements of y need the registers).  turn: which of `before` has its 16 rows.
  auto step = [&](x8<T> (&w)[F], x8<T> (&next_w)[F], int turn, int m, int next) {
    if (CHUNKS == 1 && NS < 4) load_w(next_w, next, 0);
    if (NS == 1) load_y(before[turn ^ 1], 0, next);
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      f32x4 acc[4];
      zero(acc);
      if (CHUNKS == 1) {
        multiply(acc, w, s, 0);
        if (NS == 4 && s + 1 == NS) load_w(w, next, 0);
      } else {
#pragma unroll
        for (int k = 0; k < CHUNKS; k += 2) {    // w: this chunk, next_w: the one after it
          load_w(next_w, m, k + 1);
          multiply(acc, w, s, k);
          const bool last = k + 2 >= CHUNKS;
          load_w(w, last && s + 1 == NS ? next : m, last ? 0 : k + 2);
          multiply(acc, next_w, s, k + 1);
        }
      }
      store(acc, before[NS == 1 ? turn : s], s, m);
      if (NS > 1) load_y(before[s], s, next);
      __builtin_amdgcn_sched_barrier(0);         // (what further rows need is not asked for here: registers)
    }
  };
  for (int i = begin; i < begin + steps; i += 2) {
    step(w, next_w, 0, m_of(i), m_of(i + 1));
    if (i + 1 == begin + steps) break;
    if (CHUNKS == 1 && NS < 4) step(next_w, w, 1, m_of(i + 1), m_of(i + 2));
    else step(w, next_w, 1, m_of(i + 1), m_of(i + 2));
  }
  // Fewer than 64 m: every element of y is asked for by itself, all of 16 rows at once, those behind the end and of no row too (the last there are).
  const int end = first + 256 * steps;
  if (end < m1)
    for (int s = 0; s < NS; ++s) {
      f32x4 acc[4];
      Y ends[4][4];
      int64_t r[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        r[i] = __shfl(t.row, 16 * (sub0 + s) + 4 * g + i);
#pragma unroll
        for (int j = 0; j < 4; ++j) ends[i][j] = y[max(r[i], (int64_t)0) * y_stride + (has_y ? min(end + j, m1 - 1 - 4 * l16) : 0)];
      }
      zero(acc);
#pragma unroll
      for (int k = 0; k < CHUNKS; ++k) {
        load_w(w, end, k);
        multiply(acc, w, s, k);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (end + 4 * l16 + j < m1 && r[i] >= 0)
            out[r[i] * out_stride + end + j] = (Y)fmaf(factors[16 * s + 4 * g + i], acc[j][i], has_y ? (float)ends[i][j] : 0.f);
    }
}

// Rows that no adapter changes: a wavefront takes 256 elements of a row, eight such pieces on their way at once.
template <typename Y>
__device__ __forceinline__ void copy_rows(const Projection& p, const Tile& t, int m0, int m1) {
  const Y* y = static_cast<const Y*>(p.y);
  Y* out = static_cast<Y*>(p.out);
  if (y == out && p.y_stride == p.out_stride) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), pieces = t.rows * ((m1 - m0 + 255) / 256);
  for (int i0 = wave; i0 < pieces; i0 += 32) {
    Run4<Y> x[8];
    int64_t row[8];
    int m[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int piece = min(i0 + 4 * i, pieces - 1);
      row[i] = __shfl(t.row, piece % t.rows);
      m[i] = m0 + 256 * (piece / t.rows) + 4 * lane;
      if (i0 + 4 * i >= pieces) row[i] = -1;
      const int64_t at = max(row[i], (int64_t)0) * p.y_stride;
      if (!y) x[i] = Run4<Y>{};
      else if (m0 + 256 * (piece / t.rows) + 256 <= m1) x[i] = *reinterpret_cast<const Run4<Y>*>(y + at + m[i]);
      else
#pragma unroll
        for (int e = 0; e < 4; ++e) x[i].e[e] = y[at + min(m[i] + e, m1 - 1)];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (row[i] >= 0) {
        Y* to = out + row[i] * p.out_stride + m[i];
        if (m[i] + 4 <= m1) *reinterpret_cast<Run4<Y>*>(to) = x[i];
        else
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (m[i] + e < m1) to[e] = x[i].e[e];
      }
  }
}

// The outputs' rows lie in a line, tile after tile, projection after projection, 256 elements a piece; a workgroup takes an equal part of it, as long as
// no projection of a tile ends.  (A grid of pieces of 1024, whose last ones leave half of the card idle: 150 us in place of 103 for those 5000 rows, which take 98 to 100 now.)
// KIND: steps of up to 16 rows (registers for twice the workgroups), any rows, ranks above 64.
enum Kind { kFew, kAny, kLong };
template <typename T, typename Y, Kind KIND>
__global__ void __launch_bounds__(256, KIND == kLong ? 1 : KIND == kAny ? 2 : 3) expand_kernel(Call c) {
  constexpr bool LONG = KIND == kLong;
  constexpr int N = Parts<T>::N;
  __shared__ f32x4 sums[16 * 64];
  __shared__ x8<T> vs[N * 8 * 64];               // 64 rows of 64 ranks, or 16 of 256
  __shared__ float factors[kTile];
  // (Ranks above 64 take 16 rows at a time: where pieces are few, 64 rows are four of them.)
  const unsigned all = min(uniform(c.count), c.max_tiles) * c.pieces, parts = LONG && all * 4 <= gridDim.x ? 4 : 1;
  const unsigned pieces = all * parts, each = pieces / gridDim.x, more = pieces % gridDim.x;
  unsigned at = each * blockIdx.x + min(blockIdx.x, more);
  const unsigned end = at + each + (blockIdx.x < more);
  while (at < end) {
    int piece = (int)(at % c.pieces), which = 0;
    const int tile = (int)(at / c.pieces / parts), part = (int)(at / c.pieces % parts);
    for (; piece >= (c.p[which].m + 255) / 256; ++which) piece -= (c.p[which].m + 255) / 256;
    const Projection& p = c.p[which];
    const int run = (int)min(end - at, (unsigned)((p.m + 255) / 256 - piece)), m0 = 256 * piece, m1 = min(p.m, m0 + 256 * run);
    at += run;
    const Tile t = tile_at(c, tile);
    if (t.rows == 0) continue;
    const int rank = rank_of(p, t.slot);
    if (part > 0 && (rank <= 64 || 16 * part >= t.rows)) continue;
    if (rank <= 0) {
      copy_rows<Y>(p, t, m0, m1);
      continue;
    }
    __syncthreads();                             // everyone is done with the last rows
#define SPQR_EXPAND(H, NS, SUB) expand_rows<T, Y, H, NS>(c, p, t, tile, SUB, rank, m0, m1, sums, vs, factors)
#define SPQR_EXPAND_ROWS(H) do { if (KIND == kFew || t.rows <= 16) SPQR_EXPAND(H, 1, 0); else if (t.rows <= 32) SPQR_EXPAND(H, 2, 0); else SPQR_EXPAND(H, 4, 0); } while (0)
    if (LONG && rank > 64) {
      for (int sub = part; 16 * sub < t.rows; sub += LONG && parts > 1 ? 4 : 1) {
        if (sub > part) __syncthreads();
        if (rank <= 128) SPQR_EXPAND(LONG ? 4 : 2, 1, sub);
        else SPQR_EXPAND(LONG ? 8 : 2, 1, sub);
      }
    } else if (p.max_rank <= 16) SPQR_EXPAND_ROWS(0);
    else if (rank <= 32) SPQR_EXPAND_ROWS(1);
    else SPQR_EXPAND_ROWS(2);
#undef SPQR_EXPAND_ROWS
#undef SPQR_EXPAND
  }
}

static int check_bank(const spqr_adapters_t* a) {
  if (!a) return SPQR_ERR_NULL;
  if (a->count < 1 || a->count > SPQR_MAX_FUSED) return SPQR_ERR_PARAM;
  if (a->width < 1 || a->width > SPQR_MAX_WIDTH || a->slots < 1 || a->slots > SPQR_MAX_SLOTS) return SPQR_ERR_SHAPE;
  for (int p = 0; p < a->count; ++p) {
    if (a->max_rank[p] < 1 || a->max_rank[p] > SPQR_MAX_RANK) return SPQR_ERR_PARAM;
    if (a->m[p] < 1 || a->m[p] > SPQR_MAX_WIDTH) return SPQR_ERR_SHAPE;
  }
  return SPQR_OK;
}

static Cut cut_of(const spqr_adapters_t* a) {
  Cut c{0, 0, (a->width + kStage - 1) / kStage};
  for (int p = 0; p < a->count; ++p) {
    c.rank_tiles += (a->max_rank[p] + 15) / 16;
    c.rank_halves += (a->max_rank[p] + 31) / 32;
  }
  return c;
}

static Call call_of(const spqr_adapters_t* a, const spqr_adapter_plan_t* plan, int tiles) {
  Call c;
  c.cut = cut_of(a);
  c.x = a->x; c.x_stride = a->x_stride; c.width = a->width; c.slots = a->slots;
  c.count = plan->count; c.tile = plan->tile; c.row = plan->row; c.rows = plan->rows; c.max_tiles = c.v_tiles = tiles;
  c.v = static_cast<float*>(a->workspace);
  int at = 0;
  for (int p = 0; p < SPQR_MAX_FUSED; ++p) {
    if (p >= a->count) { c.p[p] = Projection{}; c.p[p].bank = c.p[0].bank; continue; }       // (a bank to look into, of no ranks)
    c.p[p] = Projection{static_cast<const uint8_t*>(a->bank[p]), a->scale[p], a->y[p], a->out[p], a->y_stride[p], a->out_stride[p], a->m[p], a->max_rank[p], at};
    at += (a->max_rank[p] + 31) / 32;
  }
  return c;
}

template <typename T, typename Y>
static void launch_expand(const Call& c, bool longer, int pieces, hipStream_t st) {
  // as many workgroups as the card's registers have room for
  if (longer) hipLaunchKernelGGL((expand_kernel<T, Y, kLong>), dim3(min(pieces, 64) * 4), dim3(256), 0, st, c);
  else if (c.rows <= 16) hipLaunchKernelGGL((expand_kernel<T, Y, kFew>), dim3(min(pieces, 768)), dim3(256), 0, st, c);
  else hipLaunchKernelGGL((expand_kernel<T, Y, kAny>), dim3(min(pieces, 512)), dim3(256), 0, st, c);
}

template <typename T>
static int launch_adapters(Call& c, int count, int y_dtype, int tiles, hipStream_t st) {
  int groups = 0;
  bool longer = false;
  c.pieces = 0;
  for (int p = 0; p < count; ++p) {
    c.pieces += (c.p[p].m + 255) / 256;
    groups += (c.p[p].max_rank + 16 * kWaveTiles - 1) / (16 * kWaveTiles);
    longer = longer || c.p[p].max_rank > 64;
  }
  // Workgroups for the most tiles and parts that there can be; those that are too many end at once.
  const dim3 shrink(c.cut.splits(1, c.rows), tiles, groups);
  const int pieces = tiles * c.pieces;           // 20481 tiles of 2048 pieces at most
  hipLaunchKernelGGL((shrink_kernel<T>), shrink, dim3(256), 0, st, c);
  if (y_dtype == SPQR_F32) launch_expand<T, float>(c, longer, pieces, st);
  else if (y_dtype == SPQR_F16) launch_expand<T, _Float16>(c, longer, pieces, st);
  else launch_expand<T, __bf16>(c, longer, pieces, st);
  return launched();
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
  if (!p->adapter && p->requests > 0) return SPQR_ERR_NULL;      // (an array of nothing has no address)
  if (!aligned(p->adapter, 4) || !aligned(p->q_start, 4)) return SPQR_ERR_ALIGN;
  const dim3 grid(p->slots + 1);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  // (4 wavefronts: fewer barriers' worth of them; 64 requests 4.2 us, by 16 5.4)
  if (p->q_start) hipLaunchKernelGGL((adapter_plan_kernel<false, 4>), grid, dim3(256), 0, st, *p);
  else if (p->requests <= 1024) hipLaunchKernelGGL((adapter_plan_kernel<true, 4>), grid, dim3(256), 0, st, *p);
  else hipLaunchKernelGGL((adapter_plan_kernel<true, 16>), grid, dim3(1024), 0, st, *p);
  return launched();
}

extern "C" int64_t spqr_adapters_bank_bytes(const spqr_adapters_t* a, int32_t p) {
  const int rc = check_bank(a);
  if (rc) return rc;
  if (p < 0 || p >= a->count) return SPQR_ERR_PARAM;
  return header_bytes(a->slots) + a->slots * Bank(a->width, a->m[p], a->max_rank[p]).operands() * 1024;
}

extern "C" int spqr_adapters_pack(const spqr_adapters_t* a, int32_t p, int32_t first, int32_t slots, const void* A, const void* B, const int32_t* rank,
                                  void* stream) {
  const int rc = check_bank(a);
  if (rc) return rc;
  if (p < 0 || p >= a->count || first < 0 || slots < 0 || first > a->slots - slots) return SPQR_ERR_PARAM;
  if (a->dtype != SPQR_F16 && a->dtype != SPQR_BF16) return SPQR_ERR_DTYPE;
  if (slots == 0) return SPQR_OK;
  if (!A || !B || !a->bank[p]) return SPQR_ERR_NULL;
  if (!aligned(A, 2) || !aligned(B, 2) || !aligned(rank, 4) || !aligned(a->bank[p], 256)) return SPQR_ERR_ALIGN;
  const Pack args{static_cast<const uint16_t*>(A), static_cast<const uint16_t*>(B), rank, static_cast<uint8_t*>(const_cast<void*>(a->bank[p])), a->width, a->m[p],
                  a->max_rank[p], a->slots, first};
  const int64_t groups = (Bank(a->width, a->m[p], a->max_rank[p]).operands() * 64 + 255) / 256;
  hipLaunchKernelGGL(pack_kernel, dim3((unsigned)(groups < 1024 ? groups : 1024), slots), dim3(256), 0, static_cast<hipStream_t>(stream), args);
  return launched();
}

extern "C" int64_t spqr_adapters_workspace_bytes(const spqr_adapters_t* a, int32_t rows) {
  const int rc = check_bank(a);
  if (rc) return rc;
  if (rows < 0 || rows > SPQR_MAX_ROWS) return SPQR_ERR_SHAPE;
  // as many parts of the sums, for as many tiles, as a step of up to so many rows can have
  const Cut cut = cut_of(a);
  int64_t most = 0;
  for (int64_t n = rows; n > 0; n = ((n + kTile - 1) / kTile - 1) * kTile) {
    const int64_t parts = (int64_t)spqr_adapter_tiles((int32_t)n, a->slots) * cut.splits(1, (int)n);
    most = parts > most ? parts : most;
  }
  return most * cut.rank_halves * (4 * 512 * 4);
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
    if ((a->y[p] && (a->y_stride[p] < a->m[p] || a->y_stride[p] > most)) || a->out_stride[p] < a->m[p] || a->out_stride[p] > most) return SPQR_ERR_SHAPE;
  if (rows == 0) return SPQR_OK;
  if (!a->x || !a->workspace) return SPQR_ERR_NULL;
  if (!aligned(a->x, 2) || !aligned(a->workspace, 256)) return SPQR_ERR_ALIGN;
  for (int p = 0; p < a->count; ++p) {
    if (!a->bank[p] || !a->out[p]) return SPQR_ERR_NULL;
    if (!aligned(a->bank[p], 256) || !aligned(a->scale[p], 4) || !aligned(a->y[p], size_of(a->y_dtype)) || !aligned(a->out[p], size_of(a->y_dtype)))
      return SPQR_ERR_ALIGN;
  }
  if (a->workspace_bytes < spqr_adapters_workspace_bytes(a, rows)) return SPQR_ERR_WORKSPACE;
  const int tiles = spqr_adapter_tiles(rows, plan->slots);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  Call c = call_of(a, plan, tiles);
  return a->dtype == SPQR_F16 ? launch_adapters<_Float16>(c, a->count, a->y_dtype, tiles, st) : launch_adapters<__bf16>(c, a->count, a->y_dtype, tiles, st);
}
