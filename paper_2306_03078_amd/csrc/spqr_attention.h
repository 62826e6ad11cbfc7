// The attention kernels (spqr_attention.hip launches them; one source a head width instantiates them).
//
// One wavefront takes 32 keys at a time.  S^T = K Q^T on the matrix cores: a 16 x 16 x 32 instruction's A operand has a key a lane
// (lane & 15; its group lane >> 4 has 8 of every 32 elements: 16 bytes as they lie in the cache), its result a query
// row a lane and four keys a group.  Two such results give a lane eight keys of one row, which is what the B operand of
// O^T = V^T P^T wants: probabilities never leave their lane.  V^T's A operand needs one element of eight keys a lane: a lane
// loads D / 16 neighbouring elements of the group's eight keys (whole rows, so every line is read once and in order) and
// exchanges 16-bit halves between its own registers; the n-th instruction then takes the n-th element of each lane.
// A key's bytes are read once for all rows of a chunk (16 to 256: tokens times the query heads of one key head).
//
// The softmax's reference m of a row is put kLift below the largest score (in powers of two) and moves only when a score passes it
// by kLift + 8: a tile then costs no exchange between lanes.  Probabilities stay below 2^(kLift + 8); binary16 has 2^15 as its largest
// power, so 7 there: keys of 2^-32 of the largest probability still count (2^-25 without: 600 light keys beside a heavy one lost
// a quarter of their share), and all above 2^-21 with 11 bits.  bfloat16 has binary32's range and needs none.  Sums of probabilities
// are binary32 and of the unrounded ones, a partial sum a lane; probabilities are rounded to the cache's type for the matrix
// cores, as their other operand is of it.
//
// Work is a line of tiles (request, key head, chunk of rows, 32 keys) that is cut into equal parts, one a workgroup, wherever
// the cuts fall: lengths are known on the card only.  What a cut divides goes to the workspace as a partial result
// and join_kernel adds the parts in their order.
//
// What bounds it.  Few rows: memory; 16 requests of up to 8192 keys, 52 heads of 128 elements, reads 1.25 GB in 223 us, 5.6 TB/s
// (a copy reads and writes 4.7 TB/s); 40 rows over 131067 keys, 8 heads, 537 MB in 108 us, 5.0 TB/s.  Short prefixes: two launches
// and four trips to memory one after the other (lengths, pages, keys, parts); 1024 keys, 32 heads 15.7 us.  Many rows: issue of
// the matrix cores' and the softmax's instructions; 4096 rows over 260000 keys 580 us, 940 TFLOP/s; 4 requests of up to 64
// tokens, 64 heads on 8, up to 32000 keys 130 us, 550 TFLOP/s (chunks in part empty, parts written and joined).
#ifndef SPQR_ATTENTION_INTERNAL_H_
#define SPQR_ATTENTION_INTERNAL_H_
#include <cmath>
#include <type_traits>

#include "spqr_serve.h"

namespace spqr_srv {

struct Join {                    // what the cut behind a workgroup divides; parts = 0: nothing
  int parts, slot, first_row, row0, live_rows, h, unused[2];
};

struct Attend {
  const void *q, *k, *v;
  void* out;
  int64_t q_stride, out_stride;
  const int32_t *cached, *table, *q_start;
  const uint64_t* mask;
  Join* joins;                   // [workgroups]
  float *part_o, *part_ml;       // [2 * workgroups][rows of a chunk][D], [...][2]: reference, sum
  int requests, tokens, group, kv_heads, log_page, pages, max_pages, words;
  float scale2;                  // |scale| * log2(e)
  uint32_t turn;                 // 0x80008000 where scale < 0: queries change their signs
  float inv_group;
  int workgroups;
  int chunk_rows, start;         // of a chunk; places of the line in front of its tiles
  int whole;                     // 1: a chunk is one place, nothing is cut
  double inv_workgroups;
};

struct AttendPlan {              // of a launch; host
  int workgroups;
  bool by_chunk;                 // join_kernel: workgroups for chunks, not for cuts
  int join_x, join_y;
};

// D = 64, 96, 128, 256; T = _Float16, __bf16.  a.chunk_rows: 16, 32, 64 (not with D = 256), or what four
// wavefronts have with rows of their own: 256 (D = 256: 128).
template <typename T, int D> hipError_t launch_attend(const Attend& a, const AttendPlan& p, hipStream_t st);

constexpr int kTile = 32;        // keys
constexpr int kLeast = 4;        // of the line, a part: a tile a wavefront
constexpr float kFar = 1 << 20;  // a reference beyond it, either way: see `far`

#ifdef __HIP_DEVICE_COMPILE__
#define SPQR_SCALAR __attribute__((address_space(4)))
#else
#define SPQR_SCALAR
#endif

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

template <typename T> struct Matrix;
template <> struct Matrix<_Float16> {
  typedef _Float16 x8 __attribute__((ext_vector_type(8)));
  typedef _Float16 x2 __attribute__((ext_vector_type(2)));
  static __device__ __forceinline__ f32x4 product(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
  }
  static constexpr uint32_t kExponent = 0x7C00;
  static constexpr float kLift = 7.f;
};
template <> struct Matrix<__bf16> {
  typedef __bf16 x8 __attribute__((ext_vector_type(8)));
  typedef __bf16 x2 __attribute__((ext_vector_type(2)));
  static __device__ __forceinline__ f32x4 product(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
  }
  static constexpr uint32_t kExponent = 0x7F80;
  static constexpr float kLift = 0.f;
};

template <typename T>
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{lo, hi}), typename Matrix<T>::x2));
}

// What is the same in all lanes, told to the compiler: loops over it and addresses from it are scalar.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t uniform(int64_t v) {
  return (int64_t)(((uint64_t)(uint32_t)uniform((int)(v >> 32)) << 32) | (uint32_t)uniform((int)v));
}

// A request's rows and keys, cut to what the step's arrays and the table hold.
struct Request {
  int first_row, rows, cached, keys;         // cached may be beyond `keys` where the table is too narrow
};

__device__ __forceinline__ Request request_of(const Attend& a, int r) {
  Request x;
  const int from = min(max(a.q_start[r], 0), a.tokens), to = min(max(a.q_start[r + 1], 0), a.tokens);
  x.first_row = from;
  x.rows = min(max(to - from, 0), SPQR_MAX_FRESH);
  x.cached = max(a.cached[r], 0);
  const int64_t room = min((int64_t)a.max_pages << a.log_page, (int64_t)0x7FFFFFC0);
  x.keys = x.rows == 0 ? 0 : (int)min((int64_t)x.cached + x.rows, room);
  return x;
}

__device__ __forceinline__ int tiles_of(const Request& x) { return (x.keys + kTile - 1) / kTile; }
__device__ __forceinline__ int chunks_of(const Attend& a, const Request& x) { return (x.rows * a.group + a.chunk_rows - 1) / a.chunk_rows; }

// The requests, and inclusive prefix sums of their parts of the line, in LDS; returns the line's length.  A (key head, chunk) has
// a place for each of its tiles, and a.start in front of them for what it costs beside them.  All 256
// threads; ends with a barrier.
template <int kWaves>
__device__ __forceinline__ int64_t lay_line(const Attend& a, int64_t* ends, Request* requests, int64_t* wave_sums) {
  const int tid = threadIdx.x, lane = tid & 63, each = (a.requests + 64 * kWaves - 1) / (64 * kWaves);
  int64_t sum = 0;
#pragma unroll 1
  for (int i = 0; i < each; ++i) {
    const int r = tid * each + i;
    if (r >= a.requests) break;
    const Request x = request_of(a, r);
    requests[r] = x;
    ends[r] = sum += x.rows == 0 ? 0 : (int64_t)(a.whole ? 1 : tiles_of(x) + a.start) * chunks_of(a, x) * a.kv_heads;
  }
  int64_t upto = sum;
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t v = __shfl_up(upto, d);
    if (lane >= d) upto += v;
  }
  if (lane == 63) wave_sums[tid >> 6] = upto;
  __syncthreads();
  int64_t before = upto - sum, all = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < tid >> 6) before += wave_sums[w];
    all += wave_sums[w];
  }
#pragma unroll 1
  for (int i = 0; i < each; ++i)
    if (tid * each + i < a.requests) ends[tid * each + i] += before;
  __syncthreads();
  return uniform(all);
}

// A workgroup's part of the line: enough for all parts together.
__device__ __forceinline__ int64_t part_size(const Attend& a, int64_t line) {
  int64_t q = uniform((int64_t)((double)line * a.inv_workgroups));
  if (q * a.workgroups < line) ++q;
  return max((int64_t)(a.whole ? 1 : kLeast), q);
}

// x / cost, x < cost * 2^24: by the reciprocal, put right.
__device__ __forceinline__ int which_pair(int64_t x, int cost) {
  int q = uniform((int)((double)x * __builtin_amdgcn_rcp((double)cost)));
  if ((int64_t)q * cost > x) --q;
  if ((int64_t)(q + 1) * cost <= x) ++q;
  return q;
}

// row / group for rows of a request, group <= 1024: the quotient is at most 256 and off by less than 2^-14 before it is cut.
__device__ __forceinline__ int token_of(const Attend& a, int row) { return (int)(((float)row + 0.5f) * a.inv_group); }

// The part that has place x of the line.
__device__ __forceinline__ int64_t part_of(int64_t x, int64_t part) {
  int64_t q = uniform((int64_t)((double)x * __builtin_amdgcn_rcp((double)part)));
  if (q * part > x) --q;
  if ((q + 1) * part <= x) ++q;
  return q;
}

// The request that has place x of the line, x < ends[requests - 1].
__device__ __forceinline__ int find_request(const int64_t* ends, int requests, int64_t x) {
  int lo = 0, hi = requests - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (uniform(ends[mid]) > x) hi = mid; else lo = mid + 1;
  }
  return lo;
}

template <typename T, int E>
__device__ __forceinline__ void store_run(T* to, const float* y) {     // E elements, 4-byte aligned at least
  uint32_t w[E / 2];
#pragma unroll
  for (int e = 0; e < E / 2; ++e) w[e] = pack<T>(y[2 * e], y[2 * e + 1]);
  __builtin_memcpy(__builtin_assume_aligned(to, E % 8 == 0 ? 16 : E % 4 == 0 ? 8 : 4), w, 2 * E);
}

// A (key head, chunk of rows) and the tiles of it that a workgroup takes.
struct Segment {
  Request rq;
  int r, h, row0, live_rows, t0, t1, tiles;
  int64_t line;                              // place of its first tile
};

// The largest of three, NaN where one is NaN: an instruction.  (fmaxf makes each operand pass through an instruction of its own first,
// lest it be a signalling NaN.)
__device__ __forceinline__ float max3(float a, float b, float c) {
  return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c);
}

// MT: 16-row tiles of a wavefront.  KW = 4: four wavefronts take every fourth tile of keys for the same rows, out of the cache into
// registers.  KW = 1: eight wavefronts have rows of their own, for many rows over the same keys: nothing to add up, and full tiles
// pass through LDS, loaded once for all.
template <typename T, int D, int MT, int KW>
__global__ void __launch_bounds__(KW == 1 ? 512 : 256) attend_kernel(Attend a) {
  constexpr int kWaves = KW == 1 ? 8 : 4;
  constexpr int DC = D / 32;                 // 32-element pieces of a key
  constexpr int E = D / 16, EW = E / 2;      // elements and dwords of a value that a lane loads
  constexpr int kTiles = KW == 1 ? MT * kWaves : MT, kRows = 16 * kTiles;
  constexpr int kParts = KW == 4 ? 4 / MT : 1;                 // wavefronts that share 16 rows' results at the end
  extern __shared__ __align__(16) Request requests[];        // [requests], then the ends of their parts of the line
  __shared__ int64_t wave_sums[kWaves];
  constexpr int kMeet = 4 * MT * E * 256, kQueries = kTiles * DC * 256;        // floats
  constexpr int kST = D == 256 ? 1 : 2, kKeyRow = D / 8 + 1;                   // tiles of a stage; 16-byte places of a key in LDS
  constexpr int kStageK = 32 * kST * kKeyRow, kStageV = 4 * kST * D;           // 16-byte places
  __shared__ __align__(16) float shared[KW == 1 ? 8 * (kStageK + kStageV) : kMeet > kQueries ? kMeet : kQueries];
  float(*so)[MT][E][kParts][64][4 / kParts] = reinterpret_cast<float(*)[MT][E][kParts][64][4 / kParts]>(shared);      // [4]
  __shared__ int taken[2][2];                // by segments in turn, stages in turn
  __shared__ float sm[4][KW == 4 ? kRows : 1], sl[4][KW == 4 ? kRows : 1];

  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), x16 = lane & 15, g = lane >> 4;
  const int key_wave = KW == 4 ? wave : 0, m0 = KW == 4 ? 0 : wave * MT;      // m0: the first of this wavefront's 16-row tiles
  int64_t* line_ends = reinterpret_cast<int64_t*>(requests + a.requests);
  if (tid == 0 && !a.whole) a.joins[blockIdx.x].parts = 0;
  const int64_t line = lay_line<kWaves>(a, line_ends, requests, wave_sums);
  const int64_t part = part_size(a, line);
  const int64_t begin = blockIdx.x * part, end = min(line, begin + part);
  if (begin >= end) return;
  const int page = 1 << a.log_page;
  // The thread as the compiler cannot know it: what is computed from it is computed where it is used, and takes no registers elsewhere.
  auto thread = [&] {
    uint32_t id = tid;
    asm volatile("" : "+v"(id));
    return id;
  };
  const int64_t page_elements = (int64_t)a.kv_heads * page * D;

  int64_t at = begin;
  int r = find_request(line_ends, a.requests, begin);
  auto next_segment = [&](Segment& x) {      // false: the part is done
    while (at < end) {
      while (uniform(line_ends[r]) <= at) ++r;
      const int4 packed = *reinterpret_cast<const int4*>(requests + r);
      x.rq = {uniform(packed.x), uniform(packed.y), uniform(packed.z), uniform(packed.w)};
      x.r = r;
      x.tiles = tiles_of(x.rq);
      const int chunks = chunks_of(a, x.rq), cost = a.whole ? 1 : x.tiles + a.start;
      const int64_t first = r == 0 ? 0 : uniform(line_ends[r - 1]);
      const int pair = a.whole ? (int)(at - first) : which_pair(at - first, cost);
      x.line = first + (int64_t)pair * cost + a.start;
      x.h = pair / chunks;
      x.row0 = (pair - x.h * chunks) * kRows;
      x.live_rows = min(x.rq.rows * a.group - x.row0, kRows);
      x.t0 = a.whole ? 0 : (int)max(at - x.line, (int64_t)0);
      x.t1 = a.whole ? x.tiles : (int)min(end - x.line, (int64_t)x.tiles);
      at = a.whole ? at + 1 : x.line + x.tiles;
      if (x.t0 < x.t1) return true;
    }
    return false;
  };
  auto there = [&](int id) { return (unsigned)id < (unsigned)a.pages; };
  // one that is not there is page 0, of which nothing is seen
  auto half_offset = [&](int id, int key) { return (int64_t)(there(id) ? id : 0) * page_elements + (key & (page - 1)) * D; };

  // Queries stay in registers where one wavefront's are few, else in LDS, where all four read them: in the place of what the
  // results meet in later.
  constexpr bool kShared = KW == 4 && kTiles > 1;
  u32x4(*shared_q)[DC][64] = reinterpret_cast<u32x4(*)[DC][64]>(shared);
  u32x4 q[kShared ? 1 : MT][DC];
  u32x4 kf[2][DC];                           // the next tile's, on their way while this one is computed
  uint32_t vf[8][EW];
  int token[MT], id0 = 0, id1 = 0;
  const uint32_t k_lane = x16 * D + 8 * g, v_lane = 4 * g * D + E * x16;
  const T *kh, *vh;
  const SPQR_SCALAR int32_t* table;
  auto page_ids = [&](int t, int& i0, int& i1) {
    i0 = table[min((t * kTile) >> a.log_page, a.max_pages - 1)];
    i1 = table[min((t * kTile + 16) >> a.log_page, a.max_pages - 1)];
  };
  auto load_keys = [&](int t, int i0, int i1, uint32_t from) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const T* base = kh + half_offset(u ? i1 : i0, t * kTile + 16 * u);
#pragma unroll
      for (int c = 0; c < DC; ++c) kf[u][c] = *reinterpret_cast<const u32x4*>(base + (from + 32 * c));
    }
  };
  auto load_values = [&](int t, int i0, int i1, uint32_t from) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const T* base = vh + half_offset(u ? i1 : i0, t * kTile + 16 * u);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        __builtin_memcpy(vf[4 * u + i], __builtin_assume_aligned(base + (from + i * D), E % 8 == 0 ? 16 : E % 4 == 0 ? 8 : 4), 4 * EW);
    }
  };
  auto load_tile = [&](int t) {
    page_ids(t, id0, id1);
    load_keys(t, id0, id1, k_lane);
    load_values(t, id0, id1, v_lane);
  };
  // a segment's queries and this wavefront's first tile; a row is (token, query head of the group)
  auto open = [&](const Segment& x) {
    table = (const SPQR_SCALAR int32_t*)(a.table + (int64_t)x.r * a.max_pages);
    kh = static_cast<const T*>(a.k) + (int64_t)x.h * page * D;
    vh = static_cast<const T*>(a.v) + (int64_t)x.h * page * D;
    if (KW == 4 && x.t0 + key_wave < x.t1) load_tile(x.t0 + key_wave);
    auto query = [&](int m, int c) {         // (rows that are none: the last one, without a branch, taken as 0)
      const int row = x.row0 + min(16 * m + x16, x.live_rows - 1), tok = token_of(a, row);
      const T* from = static_cast<const T*>(a.q) + (int64_t)(x.rq.first_row + tok) * a.q_stride + (x.h * a.group + row - tok * a.group) * D + 8 * g;
      const uint32_t live = 16 * m + x16 < x.live_rows ? ~0u : 0u;
      return (*reinterpret_cast<const u32x4*>(from + 32 * c) ^ a.turn) & live;
    };
#pragma unroll
    for (int m = 0; m < MT; ++m) token[m] = 16 * (m0 + m) + x16 < x.live_rows ? token_of(a, x.row0 + 16 * (m0 + m) + x16) : -1;
    if constexpr (kShared) {
      __syncthreads();
#pragma unroll
      for (int f = 0; f < (kTiles * DC + 3) / 4; ++f) {
        const int m = (4 * f + wave) / DC, c = (4 * f + wave) % DC;
        if (m < kTiles) shared_q[m][c][lane] = query(m, c);
      }
      __syncthreads();
    } else {
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int c = 0; c < DC; ++c) q[m][c] = query(m0 + m, c);
    }
  };

  int segment = 0;
  Segment now;
  bool work = next_segment(now);
  if (work) open(now);
  while (work) {
    const Request rq = now.rq;
    const int live_rows = now.live_rows, t1 = now.t1;
    f32x4 o[MT][E];
    float top[MT], sum[MT];
    auto nothing = [&] {
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        top[m] = -INFINITY;
        sum[m] = 0.f;
#pragma unroll
        for (int n = 0; n < E; ++n) o[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
    };
    nothing();
    // Some row's reference in the loops without masks is so large that its own rounding is what an exponent would be made of (a fused
    // score * scale - reference is off by up to half of its last place): the wavefront takes all its tiles through the loop with
    // masks once more, which rounds the product as the reference was, so that differences are exact.
    bool far = false;

    // The steps of a tile.  All 16 * MT rows are computed, also those that are none: straight code, in which the matrix cores'
    // work and the rest alternate as written (a wavefront issues in order, and on chunks of 64 rows it is alone on its
    // SIMD: what is not between two products waits for them).
    f32x4 s[MT][2];
    u32x4 vt[E];
    uint32_t p[MT][4], seen[MT];
    auto transpose = [&](int k) {       // the k-th of 4 E exchanges
      const int n = k / 4, j = k % 4;
      vt[n][j] = __builtin_amdgcn_perm(vf[2 * j + 1][n / 2], vf[2 * j][n / 2], n & 1 ? 0x07060302 : 0x05040100);
    };
    auto scores = [&] {
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        u32x4 query[DC];
#pragma unroll
        for (int c = 0; c < DC; ++c) query[c] = kShared ? shared_q[m0 + m][c][lane] : q[kShared ? 0 : m][c];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          s[m][u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int c = 0; c < DC; ++c) s[m][u] = Matrix<T>::product(kf[u][c], query[c], s[m][u]);
        }
      }
    };
    auto references = [&](auto masked_tile, int of4) {  // where scores are too large for a row's reference, a new one
#pragma clang fp contract(off)
      constexpr bool masked = decltype(masked_tile)::value;
      constexpr float lift = Matrix<T>::kLift;
      float most[MT];
      bool moves = false, beyond = false;
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        if constexpr (masked) {                // (scaled before: a scale of 0 leaves what is not seen out)
#pragma unroll
          for (int j = 0; j < 8; ++j)
            s[m][j >> 2][j & 3] = seen[m] >> (16 * (j >> 2) + 4 * of4 + (j & 3)) & 1 ? s[m][j >> 2][j & 3] * a.scale2 : -INFINITY;
        }
        const f32x4 x = s[m][0], y = s[m][1];
        most[m] = max3(max3(x[0], x[1], x[2]), max3(x[3], y[0], y[1]), max3(y[2], y[3], y[3])) * (masked ? 1.f : a.scale2);
        moves |= most[m] - top[m] > lift + 8.f;
      }
      if (__any(moves)) {
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          most[m] = fmaxf(most[m], __shfl_xor(most[m], 16));
          most[m] = fmaxf(most[m], __shfl_xor(most[m], 32));
          const float now = most[m] - top[m] > lift + 8.f ? most[m] - lift : top[m];
          if (!masked) beyond |= fabsf(now) > kFar && now != -INFINITY;
          const float back = now == top[m] ? 1.f : __builtin_amdgcn_exp2f(top[m] - now);
          top[m] = now;
          sum[m] *= back;
#pragma unroll
          for (int n = 0; n < E; ++n) {
            o[m][n] *= back;
            if (MT > 1 && n % 2) __builtin_amdgcn_sched_barrier(0);    // few of them out of the accumulation registers at a time
          }
        }
        if (!masked) far |= __any(beyond) != 0;
      }
    };
    auto exponentials = [&](auto masked_tile, int m, int k) {  // the k-th pair of keys of rows m
#pragma clang fp contract(off)
      constexpr bool masked = decltype(masked_tile)::value;
      const float ref = top[m] == -INFINITY ? 0.f : top[m], x = s[m][k >> 1][2 * (k & 1)], y = s[m][k >> 1][2 * (k & 1) + 1];
      const float one = __builtin_amdgcn_exp2f(masked ? x - ref : fmaf(x, a.scale2, -ref));
      const float two = __builtin_amdgcn_exp2f(masked ? y - ref : fmaf(y, a.scale2, -ref));
      sum[m] += one + two;
      p[m][k] = pack<T>(one, two);
    };
    auto output = [&](int m, int n) {
      const u32x4 b = {p[m][0], p[m][1], p[m][2], p[m][3]};
      o[m][n] = Matrix<T>::product(vt[n], b, o[m][n]);
    };
    auto outputs = [&] {                       // O^T of one row tile beside the probabilities of the next
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < E; ++n) {
          if (MT > 1) __builtin_amdgcn_sched_barrier(0);
          output(m, n);
          if (m + 1 < MT) {
#pragma unroll
            for (int k = n * 4 / E; k < (n + 1) * 4 / E; ++k) exponentials(std::false_type(), m + 1, k);
          }
        }
    };

    // Tiles of cached keys that are all there.  The next tile's loads go into the registers that this one's products have read;
    // behind the last tile they are made all the same, without a branch (behind which the compiler would wait), but of one
    // line.
    const int plain_end = min(t1, min(rq.cached, rq.keys) / kTile);
    int t = 16 * m0 < live_rows ? now.t0 + key_wave : t1;      // (a wavefront whose rows are none)
    if constexpr (KW == 1) {
      // A stage of one or two tiles lies in LDS in the order in which the matrix cores take it: keys row by row, each row 16 bytes
      // longer than it is, so that 16 keys' pieces lie in different banks; of the values the eight keys of a group element by element,
      // transposed once for all eight wavefronts, the places of neighbouring pairs of elements exchanged (^) so that a thread's two
      // stores meet no bank twice.  The next stage is on its way through registers: pieces of 16 bytes of the keys, two
      // elements of eight keys of the values a thread.  A barrier a stage: behind it the last stage's buffer is free and this one's
      // is full.
      // Measured against four wavefronts of 64 rows that each load every tile (KW = 4's way): 512 rows, 8 heads of 128 over up to
      // 32000 keys, 4 requests 142 -> 132 us; 4096 rows over 260000 keys of one head 631 -> 580 us (940 TFLOP/s); heads of 64
      // elements 60 -> 49 us, of 256 194 -> 154 us (where 160 to 172 bytes of a lane's registers do not fit and go to memory; of 128: 12).  Dropped, by the first of these: two stages on their way with the
      // queries in LDS, in whose registers they are (12 % slower), priorities around the products (1 %), halves of the wavefronts
      // half a stage apart (8 %), half-full chunks' tiles shared among twice the wavefronts (equal).
      constexpr int kK = (4 * kST * D + 511) / 512, kV = (2 * kST * D + 511) / 512;
      u32x4* stage = reinterpret_cast<u32x4*>(shared);                         // [2][kStageK + kStageV]
      u32x4 k_on_way[kK];
      uint32_t v_on_way[kV][8];
      const int last = t1 - 1;
      int at_tile = now.t0;
      // pages of a stage: those of the keys and values that this wavefront loads, and whether all are there
      int k_id[kK], v_id[kV][2];
      auto half_id = [&](int half) { return table[min((min(half >> 1, last) * kTile + 16 * (half & 1)) >> a.log_page, a.max_pages - 1)]; };
      auto stage_ids = [&](int from) {
#pragma unroll
        for (int i = 0; i < kK; ++i) k_id[i] = half_id(2 * from + (64 * wave + 512 * i) / (2 * D));
#pragma unroll
        for (int i = 0; i < kV; ++i)
#pragma unroll
          for (int u = 0; u < 2; ++u) v_id[i][u] = half_id(2 * (from + (64 * wave + 512 * i) / (2 * D)) + u);
        bool all = from + kST <= plain_end;
#pragma unroll
        for (int i = 0; i < 2 * kST; ++i) all &= there(half_id(2 * from + i));
        return all;
      };
      auto fetch = [&](int from, bool whole_stage) {
        const uint32_t me = thread();
#pragma unroll
        for (int i = 0; i < kK; ++i) {
          const int first = 64 * wave + 512 * i;
          if (512 * (i + 1) <= 4 * kST * D || first < 4 * kST * D) {
            const int half = first / (2 * D);
            const T* base = kh + half_offset(k_id[i], min(from + half / 2, last) * kTile + 16 * (half & 1));
            const uint32_t unit = me + 512 * i, key = unit / (D / 8);
            k_on_way[i] = *reinterpret_cast<const u32x4*>(base + (whole_stage ? (key & 15) * D + 8 * (unit - key * (D / 8)) : 0));
          }
        }
#pragma unroll
        for (int i = 0; i < kV; ++i) {
          const int first = 64 * wave + 512 * i;
          if (512 * (i + 1) <= 2 * kST * D || first < 2 * kST * D) {
            const int tile = first / (2 * D);
            const uint32_t unit = me + 512 * i - tile * 2 * D, group = unit / (D / 2);
            const uint32_t from_lane = whole_stage ? 4 * group * D + 2 * (unit - group * (D / 2)) : 0;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              const T* base = vh + half_offset(v_id[i][u], min(from + tile, last) * kTile + 16 * u);
#pragma unroll
              for (int j = 0; j < 4; ++j) v_on_way[i][4 * u + j] = *reinterpret_cast<const uint32_t*>(base + (from_lane + j * D));
            }
          }
        }
      };
      auto lay_down = [&](int b) {
        const uint32_t me = thread();
        u32x4* to_k = stage + b * (kStageK + kStageV);
        u32x4* to_v = to_k + kStageK;
#pragma unroll
        for (int i = 0; i < kK; ++i)
          if (512 * (i + 1) <= 4 * kST * D || 64 * wave + 512 * i < 4 * kST * D) {
            const uint32_t unit = me + 512 * i, key = unit / (D / 8);
            to_k[key * kKeyRow + unit - key * (D / 8)] = k_on_way[i];
          }
#pragma unroll
        for (int i = 0; i < kV; ++i)
          if (512 * (i + 1) <= 2 * kST * D || 64 * wave + 512 * i < 2 * kST * D) {
            const uint32_t unit = me + 512 * i, group = unit / (D / 2), d = 2 * (unit - group * (D / 2)), n = d % E;
            u32x4 even, odd;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              even[j] = __builtin_amdgcn_perm(v_on_way[i][2 * j + 1], v_on_way[i][2 * j], 0x05040100);
              odd[j] = __builtin_amdgcn_perm(v_on_way[i][2 * j + 1], v_on_way[i][2 * j], 0x07060302);
            }
            u32x4* to = to_v + (group * E + n) * 16 + ((d / E) ^ (n * (16 / E)));
            to[0] = even;
            to[16] = odd;
          }
      };
      auto meet = [&] {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
      };
      // Whether a stage is taken: one thread's word for all, so that all meet as often whatever happens to the table meanwhile.
      bool ok = stage_ids(at_tile);
      fetch(at_tile, ok);
      if (tid == 0) taken[segment][0] = ok;
      ok = stage_ids(at_tile + kST);
      if (tid == 0) taken[segment][1] = ok;
      meet();                                  // the last segment's stages are read
      if (uniform(taken[segment][0])) {
        lay_down(0);
        fetch(at_tile + kST, ok);
        ok = stage_ids(at_tile + 2 * kST);
        bool more;
        int b = 0;
        do {
          meet();
          more = uniform(taken[segment][b ^ 1]);
          const uint32_t me = thread(), x = me & 15, of = me >> 4 & 3;
          const u32x4* keys = stage + b * (kStageK + kStageV) + x * kKeyRow + of;
          const u32x4* values = stage + b * (kStageK + kStageV) + kStageK + of * E * 16;
          u32x4 key[2][DC];
          auto read_keys = [&](int i) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
              for (int c = 0; c < DC; ++c) key[u][c] = keys[(32 * i + 16 * u) * kKeyRow + 4 * c];
          };
          auto read_values = [&](int i) {
#pragma unroll
            for (int n = 0; n < E; ++n) vt[n] = values[(4 * i * E + n) * 16 + (x ^ ((n & ~1) * (16 / E)))];
          };
          read_keys(0);
#pragma unroll
          for (int i = 0; i < kST; ++i) {
            __builtin_amdgcn_sched_barrier(0);
            if (t < t1) {
#pragma unroll
              for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                  s[m][u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                  for (int c = 0; c < DC; ++c) s[m][u] = Matrix<T>::product(key[u][c], q[m][c], s[m][u]);
                }
              __builtin_amdgcn_sched_barrier(0);
              read_values(i);
              references(std::false_type(), 0);
#pragma unroll
              for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int k = 0; k < 4; ++k) exponentials(std::false_type(), m, k);
#pragma unroll
              for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int n = 0; n < E; ++n) output(m, n);
            }
            __builtin_amdgcn_sched_barrier(0);
            if (i + 1 < kST) read_keys(i + 1);
            if (i == 0) {
              lay_down(b ^ 1);
              fetch(at_tile + 2 * kST, ok);
              if (tid == 0) taken[segment][b] = ok;
              ok = stage_ids(at_tile + 3 * kST);
            }
          }
          at_tile += kST;
          b ^= 1;
        } while (more);
      }
      segment ^= 1;
      if (t < t1) t = at_tile;
      load_tile(min(t, t1 - 1));             // (also where there is none: then no registers keep the last segment's)
    } else if (t < plain_end) {
      const int last = t1 - 1;
      int next0, next1, then0, then1;        // page ids of the next tile and, on their way, of the one behind it
      page_ids(min(t + KW, last), next0, next1);
      page_ids(min(t + 2 * KW, last), then0, then1);
      while (t < plain_end && there(id0) && there(id1)) {
        const bool more = t + KW < t1;
        const int following = min(t + KW, last);
        scores();
        __builtin_amdgcn_sched_barrier(0);
        load_keys(following, next0, next1, more ? k_lane : 0);
        references(std::false_type(), 0);
#pragma unroll
        for (int k = 0; k < 4; ++k) exponentials(std::false_type(), 0, k);
#pragma unroll
        for (int k = 0; k < 4 * E; ++k) transpose(k);
        __builtin_amdgcn_sched_barrier(0);
        load_values(following, next0, next1, more ? v_lane : 0);
        outputs();
        t += KW;
        id0 = next0;
        id1 = next1;
        next0 = then0;
        next1 = then1;
        page_ids(min(t + 2 * KW, last), then0, then1);
      }
    }
    // the last cached keys, the new ones, and what lies on and behind pages that are not there
    if (far) {
      nothing();
      t = now.t0 + key_wave;
      load_tile(t);
    }
    while (t < t1) {
      const int key0 = t * kTile, me = thread(), row16 = me & 15, of4 = me >> 4 & 3;
      scores();
      {
        const bool there0 = there(id0) && key0 >> a.log_page < a.max_pages, there1 = there(id1) && (key0 + 16) >> a.log_page < a.max_pages;
        const int left = rq.keys - key0;
        uint32_t exist = left >= 32 ? ~0u : (1u << left) - 1;
        if (!there0) exist &= 0xFFFF0000u;
        if (!there1) exist &= 0x0000FFFFu;
        const int n0 = key0 - rq.cached;     // the first key of the tile among the new tokens
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          uint64_t w;                        // bit i: the row sees the tile's i-th key
          if (n0 <= -kTile) {
            w = ~0ull;
          } else if (a.words == 0) {
            const int n = token[m] - n0 + 1;
            w = n <= 0 ? 0 : n >= 32 ? ~0ull : (1ull << n) - 1;
          } else {
            const uint64_t* words = a.mask + (int64_t)(rq.first_row + max(token[m], 0)) * a.words;
            if (n0 < 0) {
              w = words[0] << -n0 | ((1ull << -n0) - 1);
            } else {
              const int at_word = n0 >> 6, shift = n0 & 63;
              w = at_word < a.words ? words[at_word] >> shift : 0;
              if (shift > 32 && at_word + 1 < a.words) w |= words[at_word + 1] << (64 - shift);
            }
          }
          seen[m] = token[m] < 0 ? 0 : (uint32_t)w & exist;
        }
        // values of keys that no row sees are taken as 0
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const bool on = exist >> (16 * (j >> 2) + 4 * of4 + (j & 3)) & 1;
#pragma unroll
          for (int e = 0; e < EW; ++e) vf[j][e] = on ? vf[j][e] : 0;
        }
      }
      references(std::true_type(), of4);
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int k = 0; k < 4; ++k) exponentials(std::true_type(), m, k);
      {
        // Infinities and NaN among the values: 0 * inf would reach rows that do not see the key.  Such a key is taken out of
        // the matrix product and added by the rows that see it.
        uint32_t bad = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          bool mine = false;
#pragma unroll
          for (int e = 0; e < EW; ++e)
            mine |= (vf[j][e] & Matrix<T>::kExponent) == Matrix<T>::kExponent || (vf[j][e] >> 16 & Matrix<T>::kExponent) == Matrix<T>::kExponent;
          const uint64_t votes = __ballot(mine);
#pragma unroll
          for (int k = 0; k < 4; ++k) bad |= (votes >> (16 * k) & 0xFFFF) != 0 ? 1u << (16 * (j >> 2) + 4 * k + (j & 3)) : 0;
        }
        if (bad != 0) {
#pragma unroll 1
          for (uint32_t left = bad; left != 0; left &= left - 1) {
            const int key = __builtin_ctz(left), j = 4 * (key >> 4) + (key & 3), from = 16 * (key >> 2 & 3) + row16;
            const T* v = vh + half_offset(key < 16 ? id0 : id1, key0 + (key & 16)) + (key & 15) * D + E * 4 * of4;
#pragma unroll
            for (int m = 0; m < MT; ++m) {
              const uint32_t b0 = __shfl(p[m][0], from), b1 = __shfl(p[m][1], from), b2 = __shfl(p[m][2], from), b3 = __shfl(p[m][3], from);
              const uint32_t both = j < 4 ? (j < 2 ? b0 : b1) : (j < 6 ? b2 : b3);
              const float weight = (float)__builtin_bit_cast(T, (uint16_t)(j & 1 ? both >> 16 : both));
              if (seen[m] >> key & 1) {
#pragma unroll
                for (int n = 0; n < E; ++n)
#pragma unroll
                  for (int i = 0; i < 4; ++i) o[m][n][i] += weight * (float)v[E * i + n];
              }
            }
          }
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const bool out = bad >> (16 * (j >> 2) + 4 * of4 + (j & 3)) & 1;
#pragma unroll
            for (int e = 0; e < EW; ++e) vf[j][e] = out ? 0 : vf[j][e];
          }
        }
      }
#pragma unroll
      for (int k = 0; k < 4 * E; ++k) transpose(k);
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < E; ++n) output(m, n);
      t += KW;
      if (t < t1) load_tile(t);
    }

    // the next segment's first loads are in flight while this one's results meet, where its queries have a place
    constexpr bool kEarly = KW == 4 && !kShared;
    const Segment done = now;
    work = next_segment(now);
    if (kEarly && work) open(now);

    const bool whole = done.t0 == 0 && done.t1 == done.tiles;
    const int64_t slot = 2 * (int64_t)blockIdx.x + (begin >= done.line ? 0 : 1);
    // E elements from d on of a row of the chunk, whose sum is `all`
    auto put = [&](int in_chunk, int d, float* y, float all) {
      if (whole) {
        const int row = done.row0 + in_chunk, tok = token_of(a, row);
        const float c = all == 0.f ? 0.f : 1.f / all;
#pragma unroll
        for (int n = 0; n < E; ++n) y[n] = all == 0.f ? 0.f : y[n] * c;
        store_run<T, E>(static_cast<T*>(a.out) + (int64_t)(done.rq.first_row + tok) * a.out_stride + (done.h * a.group + row - tok * a.group) * D + d, y);
      } else {
        float* to = a.part_o + (slot * kRows + in_chunk) * D + d;
        __builtin_memcpy(__builtin_assume_aligned(to, E % 4 == 0 ? 16 : 8), y, 4 * E);
      }
    };
    auto put_sums = [&](int in_chunk, float reference, float all) {
      if (!whole) *reinterpret_cast<float2*>(a.part_ml + 2 * (slot * kRows + in_chunk)) = make_float2(reference, all);
    };
    if constexpr (KW == 1) {
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const int row = 16 * (m0 + m) + x16;
        float l = sum[m];
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if (row < live_rows) {
          if (g == 0) put_sums(row, top[m], l);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float y[E];
#pragma unroll
            for (int n = 0; n < E; ++n) y[n] = o[m][n][i];
            put(row, E * (4 * g + i), y, l);
          }
        }
      }
    } else {
      // The wavefronts add up in LDS: each takes a 16-row tile, or as many of its elements as kParts leave it: those that a lane
      // holds in i = i0 .. of a result, E neighbouring elements an i.
      constexpr int kI = 4 / kParts;
      const int tile = wave % MT, i0 = wave / MT * kI;
      __syncthreads();
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const int row = 16 * m + x16;
        float l = sum[m];
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if (g == 0) { sm[wave][row] = top[m]; sl[wave][row] = l; }
        if (row < live_rows) {
#pragma unroll
          for (int n = 0; n < E; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) so[wave][m][n][i / kI][lane][i % kI] = o[m][n][i];
        }
      }
      __syncthreads();
      const int in_chunk = 16 * tile + x16;
      if (wave / MT < kParts && in_chunk < live_rows) {
        const float best = fmaxf(fmaxf(sm[0][in_chunk], sm[1][in_chunk]), fmaxf(sm[2][in_chunk], sm[3][in_chunk]));
        float y[kI][E], all = 0.f;
#pragma unroll
        for (int k = 0; k < kI; ++k)
#pragma unroll
          for (int n = 0; n < E; ++n) y[k][n] = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const float c = sm[w][in_chunk] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sm[w][in_chunk] - best);
          all = fmaf(c, sl[w][in_chunk], all);
#pragma unroll
          for (int n = 0; n < E; ++n)
#pragma unroll
            for (int k = 0; k < kI; ++k) y[k][n] = fmaf(c, so[w][tile][n][wave / MT][lane][k], y[k][n]);
        }
#pragma unroll
        for (int k = 0; k < kI; ++k) put(in_chunk, E * (4 * g + i0 + k), y[k], all);
        if (i0 == 0 && g == 0) put_sums(in_chunk, best, all);
      }
    }
    if (tid == 0 && done.t0 == 0 && !whole) {  // the first part of what the cut behind this workgroup divides
      Join j;
      j.parts = (int)(part_of(done.line + done.tiles - 1, part) - blockIdx.x + 1);
      j.slot = (int)slot;
      j.first_row = done.rq.first_row;
      j.row0 = done.row0;
      j.live_rows = live_rows;
      j.h = done.h;
      a.joins[blockIdx.x] = j;
    }
    if (!kEarly && work) open(now);
  }
}

// Adds the parts of what the cuts divided, in their order, and writes the rows out.  kLanes lanes have a row's elements: a quarter
// of a wavefront, so that it takes four rows at once.
// by_chunk = false: workgroup x takes the cut behind workgroup x of the attention, 16 rows at a time.  true, where there are few
// chunks, each of them in many parts: the x-th chunk, four rows at a time, its wavefronts every fourth part.
template <typename T, int D, bool by_chunk>
__global__ void __launch_bounds__(256) join_kernel(Attend a) {
  constexpr int kLanes = 16, E = D / kLanes;
  __shared__ float meet[by_chunk ? 3 : 1][4][D + 2];
  __shared__ int64_t wave_sums[4];
  extern __shared__ __align__(16) Request requests[];
  const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6), of_row = lane & 15, quarter = lane >> 4, d = of_row * E;
  int from = blockIdx.x, r = 0;
  int64_t part = 0, at = 0;
  int64_t* line_ends = reinterpret_cast<int64_t*>(requests + a.requests);
  if constexpr (by_chunk) {
    part = part_size(a, lay_line<4>(a, line_ends, requests, wave_sums));
    at = blockIdx.x;                         // of the chunks of request r and those behind it
  }
  for (;;) {
    if constexpr (by_chunk) {
      int64_t chunks;
      while (r < a.requests && at >= (chunks = uniform((int64_t)chunks_of(a, requests[r]) * a.kv_heads))) { at -= chunks; ++r; }
      if (r >= a.requests) return;
      const int tiles = tiles_of(requests[r]);
      const int64_t first = uniform((r == 0 ? 0 : line_ends[r - 1]) + at * (tiles + a.start) + a.start);
      at += gridDim.x;
      from = (int)part_of(first, part);
      if (part_of(uniform(first + tiles - 1), part) == from) continue;     // whole
    }
    const Join j = a.joins[from];
    if (j.parts == 0) return;
    constexpr int kStep = by_chunk ? 4 : 1;
    const int part0 = by_chunk ? wave : 0;
    for (int row0 = by_chunk ? 4 * (int)blockIdx.y : 4 * (4 * (int)blockIdx.y + wave); row0 < j.live_rows; row0 += (by_chunk ? 4 : 16) * (int)gridDim.y) {
      const int row = min(row0 + quarter, j.live_rows - 1);
      // the parts behind the first lie in the first slots of the next workgroups
      auto place = [&](int i) { return (int64_t)(i == 0 ? j.slot : 2 * (from + i)) * a.chunk_rows + row; };
      float best = -INFINITY, all = 0.f, y[E];
#pragma unroll
      for (int e = 0; e < E; ++e) y[e] = 0.f;
      for (int i0 = part0; i0 < j.parts; i0 += 16 * kStep) {
        const int mine = i0 + of_row * kStep;
        const float2 ml = mine < j.parts ? *reinterpret_cast<const float2*>(a.part_ml + 2 * place(mine)) : make_float2(-INFINITY, 0.f);
        float most = ml.x;
        for (int k = 8; k > 0; k >>= 1) most = fmaxf(most, __shfl_xor(most, k));
        const float top = fmaxf(best, most);
        const float c = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - top), back = best == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(best - top);
        float l = c * ml.y;
        for (int k = 8; k > 0; k >>= 1) l += __shfl_xor(l, k);
        all = all * back + l;
        best = top;
#pragma unroll
        for (int e = 0; e < E; ++e) y[e] *= back;
        const int n = min(16, (j.parts - i0 + kStep - 1) / kStep);
#pragma unroll 8
        for (int i = 0; i < n; ++i) {
          const float w = __shfl(c, 16 * quarter + i);
          float v[E];
          __builtin_memcpy(v, __builtin_assume_aligned(a.part_o + place(i0 + i * kStep) * D + d, E % 4 == 0 ? 16 : 8), 4 * E);
#pragma unroll
          for (int e = 0; e < E; ++e) y[e] = fmaf(w, v[e], y[e]);
        }
      }
      if constexpr (by_chunk) {
        __syncthreads();
        if (wave != 0) {
#pragma unroll
          for (int e = 0; e < E; ++e) meet[wave - 1][quarter][d + e] = y[e];
          if (of_row == 0) { meet[wave - 1][quarter][D] = best; meet[wave - 1][quarter][D + 1] = all; }
        }
        __syncthreads();
        if (wave != 0) continue;
        for (int w = 0; w < 3; ++w) {
          const float m = meet[w][quarter][D], top = fmaxf(best, m);
          const float c = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top), back = best == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(best - top);
          all = all * back + c * meet[w][quarter][D + 1];
#pragma unroll
          for (int e = 0; e < E; ++e) y[e] = y[e] * back + c * meet[w][quarter][d + e];
          best = top;
        }
      }
      if (row0 + quarter >= j.live_rows) continue;
      const float c = 1.f / all;
#pragma unroll
      for (int e = 0; e < E; ++e) y[e] = all == 0.f ? 0.f : y[e] * c;
      const int full = j.row0 + row, tok = token_of(a, full);
      store_run<T, E>(static_cast<T*>(a.out) + (int64_t)(j.first_row + tok) * a.out_stride + (j.h * a.group + full - tok * a.group) * D + d, y);
    }
    if constexpr (!by_chunk) return;
  }
}

template <typename T, int D, int MT, int KW>
static hipError_t launch_chunks(const Attend& a, const AttendPlan& p, hipStream_t st) {
  const size_t lds = (size_t)a.requests * (sizeof(int64_t) + sizeof(Request));
  hipLaunchKernelGGL((attend_kernel<T, D, MT, KW>), dim3(p.workgroups), dim3(KW == 1 ? 512 : 256), lds, st, a);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_attend(const Attend& a, const AttendPlan& p, hipStream_t st) {
  constexpr int kWide = D == 256 ? 1 : 2;
  hipError_t e = hipErrorInvalidValue;
  if (a.chunk_rows == 16) e = launch_chunks<T, D, 1, 4>(a, p, st);
  else if (a.chunk_rows == 32) e = launch_chunks<T, D, 2, 4>(a, p, st);
  else if (a.chunk_rows == 128 * kWide) e = launch_chunks<T, D, kWide, 1>(a, p, st);
  else if constexpr (D < 256) e = launch_chunks<T, D, 4, 4>(a, p, st);
  if (e != hipSuccess || a.whole) return e;
  const size_t lds = (size_t)a.requests * (sizeof(int64_t) + sizeof(Request));
  if (p.by_chunk) hipLaunchKernelGGL((join_kernel<T, D, true>), dim3(p.join_x, p.join_y), dim3(256), lds, st, a);
  else hipLaunchKernelGGL((join_kernel<T, D, false>), dim3(p.join_x, p.join_y), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace spqr_srv
#endif
