// The attention kernels (spqr_attention.hip launches them; one source a head width instantiates them).
//
// One wavefront takes 32 keys at a time.  S^T = K Q^T on the matrix cores: a 16 x 16 x 32 instruction's A operand has a key a lane
// (lane & 15; its group lane >> 4 has 8 of every 32 elements: 16 bytes as they lie in the cache), its result a query
// row a lane and four keys a group.  Two such results give a lane eight keys of one row, which is what the B operand of
// O^T = V^T P^T wants: probabilities never leave their lane.  V^T's A operand needs one element of eight keys a lane: a lane
// loads D / 16 neighbouring elements of the group's eight keys (whole rows, so every line is read once and in order) and
// exchanges 16-bit halves between its own registers; the n-th instruction then takes the n-th element of each lane.
// K and V pass through no LDS, a key's bytes are read once for all rows of a chunk (16 * MT rows: tokens times the query
// heads of one key head).
//
// The softmax's reference m of a row moves only when a score passes it by 8 (in powers of two; probabilities stay below
// 2^8): a tile then costs no exchange between lanes.  Sums of probabilities are binary32 and of the unrounded ones, a
// partial sum a lane; probabilities are rounded to the cache's type for the matrix cores, as their other operand is of it.
//
// Work is a line of tiles (request, key head, chunk of rows, 32 keys) that is cut into equal parts, one a workgroup, wherever
// the cuts fall: lengths are known on the card only.  What a cut divides goes to the workspace as a partial result
// and join_kernel adds the parts in their order.
#ifndef SPQR_ATTENTION_INTERNAL_H_
#define SPQR_ATTENTION_INTERNAL_H_
#include <cmath>
#include <type_traits>

#include "spqr_serve.h"

namespace spqr_srv {

struct Join {                    // what a workgroup's cut leaves for join_kernel; parts = 0: nothing
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
  float scale2;                  // scale * log2(e)
  float inv_group;
  int workgroups;
  double inv_workgroups;
};

struct AttendPlan {              // of a launch; host
  int rows;                      // of a chunk: 16 * MT
  int workgroups;
  int join_y;                    // workgroups of join_kernel a cut, four rows each at a time
};

// D = 64, 96, 128, 256; T = _Float16, __bf16.  rows: 16, 32 or 64 (D = 256: 32 at most).
template <typename T, int D> hipError_t launch_attend(const Attend& a, const AttendPlan& p, hipStream_t st);

constexpr int kTile = 32;        // keys
constexpr int kLeast = 4;        // of the line, a part: a tile a wavefront

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
};
template <> struct Matrix<__bf16> {
  typedef __bf16 x8 __attribute__((ext_vector_type(8)));
  typedef __bf16 x2 __attribute__((ext_vector_type(2)));
  static __device__ __forceinline__ f32x4 product(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
  }
  static constexpr uint32_t kExponent = 0x7F80;
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
template <int MT>
__device__ __forceinline__ int chunks_of(const Attend& a, const Request& x) { return (x.rows * a.group + 16 * MT - 1) / (16 * MT); }

// What a (key head, chunk) costs beside its tiles, in tiles: its start and end were measured to take as long.
template <int MT> constexpr int kStart = MT == 1 ? 4 : MT == 2 ? 8 : 16;

// The requests, and inclusive prefix sums of their parts of the line, in LDS; returns the line's length.  All 256 threads;
// ends with a barrier.
template <int MT>
__device__ __forceinline__ int64_t lay_line(const Attend& a, int64_t* ends, Request* requests, int64_t* wave_sums) {
  const int tid = threadIdx.x, lane = tid & 63, each = (a.requests + 255) / 256;
  int64_t sum = 0;
#pragma unroll 1
  for (int i = 0; i < each; ++i) {
    const int r = tid * each + i;
    if (r >= a.requests) break;
    const Request x = request_of(a, r);
    requests[r] = x;
    ends[r] = sum += x.rows == 0 ? 0 : (int64_t)(tiles_of(x) + kStart<MT>) * chunks_of<MT>(a, x) * a.kv_heads;
  }
  int64_t upto = sum;
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t v = __shfl_up(upto, d);
    if (lane >= d) upto += v;
  }
  if (lane == 63) wave_sums[tid >> 6] = upto;
  __syncthreads();
  int64_t before = upto - sum, all = 0;
  for (int w = 0; w < 4; ++w) {
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
  return max((int64_t)kLeast, q);
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

template <typename T, int D, int MT>
__global__ void __launch_bounds__(256) attend_kernel(Attend a) {
  constexpr int DC = D / 32;                 // 32-element pieces of a key
  constexpr int E = D / 16, EW = E / 2;      // elements and dwords of a value that a lane loads
  constexpr int kRows = 16 * MT;
  extern __shared__ __align__(16) Request requests[];        // [requests], then the ends of their parts of the line
  __shared__ int64_t wave_sums[4];
  __shared__ float so[4][MT][E][4 / MT][64][MT];
  __shared__ float sm[4][kRows], sl[4][kRows];

  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), x16 = lane & 15, g = lane >> 4;
  int64_t* line_ends = reinterpret_cast<int64_t*>(requests + a.requests);
  if (tid == 0) a.joins[blockIdx.x].parts = 0;
  const int64_t line = lay_line<MT>(a, line_ends, requests, wave_sums);
  const int64_t part = part_size(a, line);
  const int64_t begin = blockIdx.x * part, end = min(line, begin + part);
  if (begin >= end) return;
  const int page = 1 << a.log_page;
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
      const int chunks = chunks_of<MT>(a, x.rq), cost = x.tiles + kStart<MT>;
      const int64_t first = r == 0 ? 0 : uniform(line_ends[r - 1]);
      const int pair = which_pair(at - first, cost);
      x.line = first + (int64_t)pair * cost + kStart<MT>;
      x.h = pair / chunks;
      x.row0 = (pair - x.h * chunks) * kRows;
      x.live_rows = min(x.rq.rows * a.group - x.row0, kRows);
      x.t0 = (int)max(at - x.line, (int64_t)0);
      x.t1 = (int)min(end - x.line, (int64_t)x.tiles);
      at = x.line + x.tiles;
      if (x.t0 < x.t1) return true;
    }
    return false;
  };
  auto there = [&](int id) { return (unsigned)id < (unsigned)a.pages; };
  // one that is not there is page 0, of which nothing is seen
  auto half_offset = [&](int id, int key) { return (int64_t)(there(id) ? id : 0) * page_elements + (key & (page - 1)) * D; };

  // Queries stay in registers where one wavefront's are few, else in LDS, where all four read them: in the place of what the
  // results meet in later.
  constexpr bool kShared = MT > 1;
  u32x4(*shared_q)[DC][64] = reinterpret_cast<u32x4(*)[DC][64]>(&so[0][0][0][0][0][0]);
  u32x4 q[kShared ? 1 : MT][DC], kf[2][DC];
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
    if (x.t0 + wave < x.t1) load_tile(x.t0 + wave);
    auto query = [&](int m, int c) {         // (rows that are none: the last one, without a branch, taken as 0)
      const int row = x.row0 + min(16 * m + x16, x.live_rows - 1), tok = token_of(a, row);
      const T* from = static_cast<const T*>(a.q) + (int64_t)(x.rq.first_row + tok) * a.q_stride + (x.h * a.group + row - tok * a.group) * D + 8 * g;
      const u32x4 v = *reinterpret_cast<const u32x4*>(from + 32 * c);
      return 16 * m + x16 < x.live_rows ? v : u32x4{0, 0, 0, 0};
    };
#pragma unroll
    for (int m = 0; m < MT; ++m) token[m] = 16 * m + x16 < x.live_rows ? token_of(a, x.row0 + 16 * m + x16) : -1;
    if constexpr (kShared) {
      __syncthreads();
#pragma unroll
      for (int f = 0; f < (MT * DC + 3) / 4; ++f) {
        const int m = (4 * f + wave) / DC, c = (4 * f + wave) % DC;
        if (m < MT) shared_q[m][c][lane] = query(m, c);
      }
      __syncthreads();
    } else {
#pragma unroll
      for (int c = 0; c < DC; ++c) q[0][c] = query(0, c);
    }
  };

  Segment now;
  bool work = next_segment(now);
  if (work) open(now);
  while (work) {
    const Request rq = now.rq;
    const int live_rows = now.live_rows, t1 = now.t1;
    f32x4 o[MT][E];
    float top[MT], sum[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      top[m] = -INFINITY;
      sum[m] = 0.f;
#pragma unroll
      for (int n = 0; n < E; ++n) o[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // the steps of a tile
    f32x4 s[MT][2];
    uint32_t p[MT][4], seen[MT];
    auto scores = [&] {
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        if (m > 0 && 16 * m >= live_rows) continue;
        u32x4 query[DC];
#pragma unroll
        for (int c = 0; c < DC; ++c) query[c] = kShared ? shared_q[m][c][lane] : q[kShared ? 0 : m][c];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          s[m][u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int c = 0; c < DC; ++c) s[m][u] = Matrix<T>::product(kf[u][c], query[c], s[m][u]);
        }
      }
    };
    auto probabilities = [&](auto masked_tile) {
      constexpr bool masked = decltype(masked_tile)::value;
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        if (m > 0 && 16 * m >= live_rows) continue;
        float z[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) z[j] = s[m][j >> 2][j & 3] * a.scale2;
        if constexpr (masked) {
#pragma unroll
          for (int j = 0; j < 8; ++j) z[j] = seen[m] >> (16 * (j >> 2) + 4 * g + (j & 3)) & 1 ? z[j] : -INFINITY;
        }
        float most = fmaxf(fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])), fmaxf(fmaxf(z[4], z[5]), fmaxf(z[6], z[7])));
        if (__any(most > top[m] + 8.f)) {
          most = fmaxf(most, __shfl_xor(most, 16));
          most = fmaxf(most, __shfl_xor(most, 32));
          const float now = most > top[m] + 8.f ? most : top[m];
          const float back = now == top[m] ? 1.f : __builtin_amdgcn_exp2f(top[m] - now);
          top[m] = now;
          sum[m] *= back;
#pragma unroll
          for (int n = 0; n < E; ++n) o[m][n] *= back;
        }
        const float ref = top[m] == -INFINITY ? 0.f : top[m];
#pragma unroll
        for (int j = 0; j < 8; ++j) z[j] = __builtin_amdgcn_exp2f(z[j] - ref);
        sum[m] += ((z[0] + z[1]) + (z[2] + z[3])) + ((z[4] + z[5]) + (z[6] + z[7]));
#pragma unroll
        for (int j = 0; j < 4; ++j) p[m][j] = pack<T>(z[2 * j], z[2 * j + 1]);
      }

    };
    u32x4 vt[E];
    auto transpose = [&] {
#pragma unroll
      for (int n = 0; n < E; ++n)
#pragma unroll
        for (int j = 0; j < 4; ++j) vt[n][j] = __builtin_amdgcn_perm(vf[2 * j + 1][n / 2], vf[2 * j][n / 2], n & 1 ? 0x07060302 : 0x05040100);
    };
    auto outputs = [&] {
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        if (m > 0 && 16 * m >= live_rows) continue;
        const u32x4 b = {p[m][0], p[m][1], p[m][2], p[m][3]};
#pragma unroll
        for (int n = 0; n < E; ++n) o[m][n] = Matrix<T>::product(vt[n], b, o[m][n]);
      }
    };

    // Tiles of cached keys that are all there.  The next tile's loads go into the registers that this one's products have read;
    // behind the last tile they are made all the same, without a branch (behind which the compiler would wait), but of one
    // line.
    const int plain_end = min(t1, min(rq.cached, rq.keys) / kTile);
    int t = now.t0 + wave;
    if (t < plain_end) {
      const int last = t1 - 1;
      int next0, next1, later0, later1;      // page ids are on their way for two tiles
      page_ids(min(t + 4, last), next0, next1);
      page_ids(min(t + 8, last), later0, later1);
      while (t < plain_end && there(id0) && there(id1)) {
        const bool more = t + 4 < t1;
        const int following = min(t + 4, last);
        scores();
        __builtin_amdgcn_sched_barrier(0);
        load_keys(following, next0, next1, more ? k_lane : 0);
        probabilities(std::false_type());
        transpose();
        __builtin_amdgcn_sched_barrier(0);
        load_values(following, next0, next1, more ? v_lane : 0);
        outputs();
        t += 4;
        id0 = next0;
        id1 = next1;
        next0 = later0;
        next1 = later1;
        page_ids(min(t + 8, last), later0, later1);
      }
    }
    // the last cached keys, the new ones, and what lies on and behind pages that are not there
    while (t < t1) {
      const int key0 = t * kTile;
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
          const bool on = exist >> (16 * (j >> 2) + 4 * g + (j & 3)) & 1;
#pragma unroll
          for (int e = 0; e < EW; ++e) vf[j][e] = on ? vf[j][e] : 0;
        }
      }
      probabilities(std::true_type());
      {
        // Infinities and NaN among the values: 0 * inf would reach rows that do not see the key.  Such a key is taken out of
        // the matrix product and added by the rows that see it; the probabilities pass through this wavefront's part of `so`.
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
            const int key = __builtin_ctz(left), j = 4 * (key >> 4) + (key & 3), from = 16 * (key >> 2 & 3) + x16;
            const T* v = vh + half_offset(key < 16 ? id0 : id1, key0 + (key & 16)) + (key & 15) * D + E * 4 * g;
#pragma unroll
            for (int m = 0; m < MT; ++m) {
              const uint32_t mine = j < 4 ? (j < 2 ? p[m][0] : p[m][1]) : (j < 6 ? p[m][2] : p[m][3]);
              const uint32_t both = __shfl(mine, from);
              const float weight = (float)__builtin_bit_cast(T, (uint16_t)(j & 1 ? both >> 16 : both));
              if (16 * m < live_rows && (seen[m] >> key & 1)) {
#pragma unroll
                for (int n = 0; n < E; ++n)
#pragma unroll
                  for (int i = 0; i < 4; ++i) o[m][n][i] += weight * (float)v[E * i + n];
              }
            }
          }
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const bool out = bad >> (16 * (j >> 2) + 4 * g + (j & 3)) & 1;
#pragma unroll
            for (int e = 0; e < EW; ++e) vf[j][e] = out ? 0 : vf[j][e];
          }
        }
      }
      transpose();
      outputs();
      t += 4;
      if (t < t1) load_tile(t);
    }

    // the next segment's first loads are in flight while this one's results meet, where its queries have a place
    constexpr bool kEarly = !kShared;
    const Segment done = now;
    work = next_segment(now);
    if (kEarly && work) open(now);

    // The wavefronts add up in LDS: each takes 16 rows (MT = 4), or a half (2) or a quarter (1) of their elements: those that
    // a lane holds in i = MT * (wave / MT) .. of a result, E neighbouring elements an i.
    const bool whole = done.t0 == 0 && done.t1 == done.tiles;
    const int64_t slot = 2 * (int64_t)blockIdx.x + (begin >= done.line ? 0 : 1);
    __syncthreads();
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      if (m > 0 && 16 * m >= live_rows) continue;
      float l = sum[m];
      l += __shfl_xor(l, 16);
      l += __shfl_xor(l, 32);
      if (g == 0) { sm[wave][16 * m + x16] = top[m]; sl[wave][16 * m + x16] = l; }
      if (16 * m + x16 < live_rows) {
#pragma unroll
        for (int n = 0; n < E; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) so[wave][m][n][i / MT][lane][i % MT] = o[m][n][i];
      }
    }
    __syncthreads();
    const int in_chunk = 16 * (wave % MT) + x16;
    if (in_chunk < live_rows) {
      const float best = fmaxf(fmaxf(sm[0][in_chunk], sm[1][in_chunk]), fmaxf(sm[2][in_chunk], sm[3][in_chunk]));
      float y[MT][E], all = 0.f;
#pragma unroll
      for (int k = 0; k < MT; ++k)
#pragma unroll
        for (int n = 0; n < E; ++n) y[k][n] = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float c = sm[w][in_chunk] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sm[w][in_chunk] - best);
        all = fmaf(c, sl[w][in_chunk], all);
#pragma unroll
        for (int n = 0; n < E; ++n)
#pragma unroll
          for (int k = 0; k < MT; ++k) y[k][n] = fmaf(c, so[w][wave % MT][n][wave / MT][lane][k], y[k][n]);
      }
      const int d = E * (4 * g + MT * (wave / MT));
      if (whole) {
        const int row = done.row0 + in_chunk, tok = token_of(a, row);
        const float c = 1.f / all;
        T* to = static_cast<T*>(a.out) + (int64_t)(done.rq.first_row + tok) * a.out_stride + (done.h * a.group + row - tok * a.group) * D + d;
#pragma unroll
        for (int k = 0; k < MT; ++k) {
#pragma unroll
          for (int n = 0; n < E; ++n) y[k][n] = all == 0.f ? 0.f : y[k][n] * c;
          store_run<T, E>(to + E * k, y[k]);
        }
      } else {
        float* to = a.part_o + (slot * kRows + in_chunk) * D + d;
#pragma unroll
        for (int k = 0; k < MT; ++k)
#pragma unroll
          for (int n = 0; n < E; n += 2) *reinterpret_cast<float2*>(to + E * k + n) = make_float2(y[k][n], y[k][n + 1]);
        if (wave / MT == 0 && g == 0) *reinterpret_cast<float2*>(a.part_ml + 2 * (slot * kRows + in_chunk)) = make_float2(best, all);
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

// Adds the parts of what the cut behind workgroup x divided, in their order: a wavefront a row.
template <typename T, int D>
__global__ void __launch_bounds__(256) join_kernel(Attend a, int chunk_rows) {
  constexpr int PE = D >= 128 ? D / 64 : D == 96 ? 2 : 1;      // elements a lane
  const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6);
  const Join j = a.joins[blockIdx.x];
  if (j.parts == 0) return;
  const int d = min(lane * PE, D - PE);      // (D = 96: the last lanes repeat the last elements)
  for (int row = 4 * blockIdx.y + wave; row < j.live_rows; row += 4 * gridDim.y) {
    // the parts behind the first lie in the first slots of the next workgroups
    auto place = [&](int i) { return (int64_t)(i == 0 ? j.slot : 2 * ((int)blockIdx.x + i)) * chunk_rows + row; };
    float best = -INFINITY, all = 0.f, y[PE];
#pragma unroll
    for (int e = 0; e < PE; ++e) y[e] = 0.f;
    for (int i0 = 0; i0 < j.parts; i0 += 64) {
      const bool have = i0 + lane < j.parts;
      const float2 ml = have ? *reinterpret_cast<const float2*>(a.part_ml + 2 * place(i0 + lane)) : make_float2(-INFINITY, 0.f);
      float most = ml.x;
      for (int k = 32; k > 0; k >>= 1) most = fmaxf(most, __shfl_xor(most, k));
      const float top = fmaxf(best, most);
      const float c = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - top), back = best == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(best - top);
      float l = c * ml.y;
      for (int k = 32; k > 0; k >>= 1) l += __shfl_xor(l, k);
      all = all * back + l;
      best = top;
#pragma unroll
      for (int e = 0; e < PE; ++e) y[e] *= back;
      const int n = min(64, j.parts - i0);
#pragma unroll 8
      for (int i = 0; i < n; ++i) {
        const float w = __shfl(c, i);
        float v[PE];
        __builtin_memcpy(v, __builtin_assume_aligned(a.part_o + place(i0 + i) * D + d, 4 * PE), 4 * PE);
#pragma unroll
        for (int e = 0; e < PE; ++e) y[e] = fmaf(w, v[e], y[e]);
      }
    }
    const float c = 1.f / all;
    const int full = j.row0 + row, tok = token_of(a, full);
    T out[PE];
#pragma unroll
    for (int e = 0; e < PE; ++e) out[e] = (T)(all == 0.f ? 0.f : y[e] * c);
    T* to = static_cast<T*>(a.out) + (int64_t)(j.first_row + tok) * a.out_stride + (j.h * a.group + full - tok * a.group) * D + d;
    __builtin_memcpy(__builtin_assume_aligned(to, 2 * PE), out, 2 * PE);
  }
}

template <typename T, int D, int MT>
static hipError_t launch_chunks(const Attend& a, const AttendPlan& p, hipStream_t st) {
  const size_t lds = (size_t)a.requests * (sizeof(int64_t) + sizeof(Request));
  hipLaunchKernelGGL((attend_kernel<T, D, MT>), dim3(p.workgroups), dim3(256), lds, st, a);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_attend(const Attend& a, const AttendPlan& p, hipStream_t st) {
  hipError_t e = hipErrorInvalidValue;
  if (p.rows == 16) e = launch_chunks<T, D, 1>(a, p, st);
  else if (p.rows == 32) e = launch_chunks<T, D, 2>(a, p, st);
  else if constexpr (D < 256) e = launch_chunks<T, D, 4>(a, p, st);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((join_kernel<T, D>), dim3(p.workgroups, p.join_y), dim3(256), 0, st, a, p.rows);
  return hipGetLastError();
}

}  // namespace spqr_srv
#endif
