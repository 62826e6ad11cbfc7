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

struct Attend {
  const void *q, *k, *v;
  void* out;
  int64_t q_stride, out_stride;
  const int32_t *cached, *table, *q_start;
  const uint64_t* mask;
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
  int join_x, join_y;            // grid of join_kernel
};

// D = 64, 96, 128, 256; T = _Float16, __bf16.  rows: 16, 32 or 64 (D = 256: 32 at most).
template <typename T, int D> hipError_t launch_attend(const Attend& a, const AttendPlan& p, hipStream_t st);

constexpr int kTile = 32;        // keys
constexpr int kLeast = 4;        // tiles of a workgroup's part: one a wavefront

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

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// A request's rows and keys, cut to what the step's arrays and the table hold.
struct Request {
  int first_row, rows, keys, tiles, chunks;
  int cached;                    // may be beyond `keys` where the table is too narrow
  __device__ __forceinline__ int64_t work(int kv_heads) const { return (int64_t)tiles * chunks * kv_heads; }
};

__device__ __forceinline__ Request request_of(const Attend& a, int r, int chunk_rows) {
  Request x;
  const int from = min(max(a.q_start[r], 0), a.tokens), to = min(max(a.q_start[r + 1], 0), a.tokens);
  x.first_row = from;
  x.rows = min(max(to - from, 0), SPQR_MAX_FRESH);
  x.cached = max(a.cached[r], 0);
  const int64_t room = min((int64_t)a.max_pages << a.log_page, (int64_t)0x7FFFFFC0);
  x.keys = (int)min((int64_t)x.cached + x.rows, room);
  x.tiles = x.rows == 0 ? 0 : (x.keys + kTile - 1) / kTile;
  x.chunks = (x.rows * a.group + chunk_rows - 1) / chunk_rows;
  return x;
}

// Inclusive prefix sums of the requests' work in LDS; returns the whole.  All 256 threads; ends with a barrier.
__device__ __forceinline__ int64_t scan_requests(const Attend& a, int chunk_rows, int64_t* ends, int64_t* wave_sums) {
  const int tid = threadIdx.x, lane = tid & 63, each = (a.requests + 255) / 256;
  int64_t sum = 0;
#pragma unroll 1
  for (int i = 0; i < each; ++i) {
    const int r = tid * each + i;
    if (r < a.requests) sum += request_of(a, r, chunk_rows).work(a.kv_heads), ends[r] = sum;
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
  return all;
}

// Tiles of a workgroup's part: enough for all parts together.
__device__ __forceinline__ int64_t part_size(const Attend& a, int64_t work) {
  int64_t q = (int64_t)((double)work * a.inv_workgroups);
  if (q * a.workgroups < work) ++q;
  return max((int64_t)kLeast, q);
}

// x / tiles, x < tiles * 2^24: by the reciprocal, put right.
__device__ __forceinline__ int which_pair(int64_t x, int tiles) {
  int q = (int)((double)x * __builtin_amdgcn_rcp((double)tiles));
  if ((int64_t)q * tiles > x) --q;
  if ((int64_t)(q + 1) * tiles <= x) ++q;
  return q;
}

// row / group for rows of a request, group <= 1024: the quotient is at most 256 and off by less than 2^-14 before it is cut.
__device__ __forceinline__ int token_of(const Attend& a, int row) { return (int)(((float)row + 0.5f) * a.inv_group); }

// Parts that start at or before tile x.
__device__ __forceinline__ int64_t parts_to(int64_t x, int64_t part) {
  int64_t q = (int64_t)((double)x * __builtin_amdgcn_rcp((double)part));
  if (q * part > x) --q;
  if ((q + 1) * part <= x) ++q;
  return q + 1;
}

// The request that has tile x of the line, x < ends[requests - 1].
__device__ __forceinline__ int find_request(const int64_t* ends, int requests, int64_t x) {
  int lo = 0, hi = requests - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (ends[mid] > x) hi = mid; else lo = mid + 1;
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

template <typename T, int D, int MT>
__global__ void __launch_bounds__(256) attend_kernel(Attend a) {
  constexpr int DC = D / 32;                 // 32-element pieces of a key
  constexpr int E = D / 16, EW = E / 2;      // elements and dwords of a value that a lane loads
  constexpr int kRows = 16 * MT;
  __shared__ int64_t ends[SPQR_MAX_REQUESTS];
  __shared__ int64_t wave_sums[4];
  __shared__ float so[4][E][4][64];
  __shared__ float sm[4][16], sl[4][16];

  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), x16 = lane & 15, g = lane >> 4;
  const int64_t work = scan_requests(a, kRows, ends, wave_sums);
  const int64_t part = part_size(a, work);
  const int64_t begin = blockIdx.x * part, end = min(work, begin + part);
  if (begin >= end) return;
  int r = find_request(ends, a.requests, begin);
  const int page = 1 << a.log_page;
  const int64_t page_elements = (int64_t)a.kv_heads * page * D;

  for (int64_t at = begin; at < end;) {
    while (ends[r] <= at) ++r;
    r = uniform(r);
    const Request rq = request_of(a, r, kRows);
    const int64_t in_request = at - (r == 0 ? 0 : ends[r - 1]);
    const int pair = uniform(which_pair(in_request, rq.tiles));
    const int t0 = uniform((int)(in_request - (int64_t)pair * rq.tiles));
    const int t1 = uniform((int)min((int64_t)rq.tiles, t0 + (end - at)));
    const int h = pair / rq.chunks, chunk = pair - h * rq.chunks;
    const int row0 = chunk * kRows, live_rows = min(rq.rows * a.group - row0, kRows);
    const SPQR_SCALAR int32_t* table = (const SPQR_SCALAR int32_t*)(a.table + (int64_t)r * a.max_pages);
    const T* kh = static_cast<const T*>(a.k) + (int64_t)h * page * D;
    const T* vh = static_cast<const T*>(a.v) + (int64_t)h * page * D;

    // the rows' queries; a row is (token, query head of the group)
    u32x4 q[MT][DC];
    int token[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      const int row = row0 + 16 * m + x16;
      const bool live = row < rq.rows * a.group;
      token[m] = live ? token_of(a, row) : -1;
      const T* from = static_cast<const T*>(a.q) + (int64_t)(rq.first_row + token[m]) * a.q_stride + (h * a.group + row - token[m] * a.group) * D + 8 * g;
#pragma unroll
      for (int c = 0; c < DC; ++c) q[m][c] = live ? *reinterpret_cast<const u32x4*>(from + 32 * c) : u32x4{0, 0, 0, 0};
    }
    f32x4 o[MT][E];
    float top[MT], sum[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      top[m] = -INFINITY;
      sum[m] = 0.f;
#pragma unroll
      for (int n = 0; n < E; ++n) o[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // page ids of a tile's two halves
    auto page_ids = [&](int t, int& id0, int& id1) {
      id0 = table[min((t * kTile) >> a.log_page, a.max_pages - 1)];
      id1 = table[min((t * kTile + 16) >> a.log_page, a.max_pages - 1)];
    };
    auto there = [&](int id) { return (unsigned)id < (unsigned)a.pages; };
    // one that is not there is page 0, of which nothing is seen
    auto half_offset = [&](int id, int key) { return (int64_t)(there(id) ? id : 0) * page_elements + (key & (page - 1)) * D; };

    const uint32_t k_lane = x16 * D + 8 * g, v_lane = 4 * g * D + E * x16;
    u32x4 kf[2][DC];
    uint32_t vf[8][EW];
    int id0, id1, next0, next1;
    auto load_keys = [&](int t, int i0, int i1, uint32_t k_lane) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const T* base = kh + half_offset(u ? i1 : i0, t * kTile + 16 * u);
#pragma unroll
        for (int c = 0; c < DC; ++c) kf[u][c] = *reinterpret_cast<const u32x4*>(base + (k_lane + 32 * c));
      }
    };
    auto load_values = [&](int t, int i0, int i1, uint32_t v_lane) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const T* base = vh + half_offset(u ? i1 : i0, t * kTile + 16 * u);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          __builtin_memcpy(vf[4 * u + i], __builtin_assume_aligned(base + (v_lane + i * D), E % 8 == 0 ? 16 : E % 4 == 0 ? 8 : 4), 4 * EW);
      }
    };

    // the steps of a tile
    f32x4 s[MT][2];
    uint32_t p[MT][4], seen[MT];
    auto scores = [&] {
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        if (m > 0 && 16 * m >= live_rows) continue;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          s[m][u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int c = 0; c < DC; ++c) s[m][u] = Matrix<T>::product(kf[u][c], q[m][c], s[m][u]);
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
    int t = t0 + wave;
    if (t < plain_end) {
      page_ids(t, id0, id1);
      load_keys(t, id0, id1, k_lane);
      load_values(t, id0, id1, v_lane);
      int following = min(t + 4, plain_end - 1);
      page_ids(following, next0, next1);
      while (there(id0) && there(id1)) {
        const bool more = t + 4 < plain_end;
        scores();
        __builtin_amdgcn_sched_barrier(0);
        load_keys(following, next0, next1, more ? k_lane : 0);
        probabilities(std::false_type());
        transpose();
        __builtin_amdgcn_sched_barrier(0);
        load_values(following, next0, next1, more ? v_lane : 0);
        outputs();
        t += 4;
        if (!more) break;
        id0 = next0;
        id1 = next1;
        following = min(t + 4, plain_end - 1);
        page_ids(following, next0, next1);
      }
    }
    // the last cached keys, the new ones, and what lies on and behind pages that are not there
    for (; t < t1; t += 4) {
      page_ids(t, id0, id1);
      load_keys(t, id0, id1, k_lane);
      load_values(t, id0, id1, v_lane);
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
          uint32_t* kept = reinterpret_cast<uint32_t*>(&so[wave][0][0][0]);
#pragma unroll
          for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int j = 0; j < 4; ++j) kept[(4 * m + j) * 64 + lane] = 16 * m < live_rows ? p[m][j] : 0;
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll 1
          for (uint32_t left = bad; left != 0; left &= left - 1) {
            const int key = __builtin_ctz(left), j = 4 * (key >> 4) + (key & 3), of = key >> 2 & 3;
            const T* v = vh + half_offset(key < 16 ? id0 : id1, key0 + (key & 16)) + (key & 15) * D + E * 4 * g;
#pragma unroll
            for (int m = 0; m < MT; ++m) {
              const uint32_t both = kept[(4 * m + (j >> 1)) * 64 + 16 * of + x16];
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
    }

    // the four wavefronts' parts, 16 rows at a time
    const bool whole = t0 == 0 && t1 == rq.tiles;
    const int64_t slot = 2 * (int64_t)blockIdx.x + (at == begin ? 0 : 1);
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      if (16 * m >= live_rows) continue;
      float l = sum[m];
      l += __shfl_xor(l, 16);
      l += __shfl_xor(l, 32);
      if (g == 0) { sm[wave][x16] = top[m]; sl[wave][x16] = l; }
#pragma unroll
      for (int n = 0; n < E; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) so[wave][n][i][lane] = o[m][n][i];
      __syncthreads();
      // thread: row x16, elements E * (4 g + i) .. + E - 1, i = wave
      float best = fmaxf(fmaxf(sm[0][x16], sm[1][x16]), fmaxf(sm[2][x16], sm[3][x16]));
      float y[E], all = 0.f;
#pragma unroll
      for (int n = 0; n < E; ++n) y[n] = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float c = sm[w][x16] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sm[w][x16] - best);
        all = fmaf(c, sl[w][x16], all);
#pragma unroll
        for (int n = 0; n < E; ++n) y[n] = fmaf(c, so[w][n][wave][lane], y[n]);
      }
      const int in_chunk = 16 * m + x16, d = E * (4 * g + wave);
      if (in_chunk < live_rows) {
        if (whole) {
          const int row = row0 + in_chunk, tok = token_of(a, row);
          const float c = all == 0.f ? 0.f : 1.f / all;
#pragma unroll
          for (int n = 0; n < E; ++n) y[n] = all == 0.f ? 0.f : y[n] * c;
          store_run<T, E>(static_cast<T*>(a.out) + (int64_t)(rq.first_row + tok) * a.out_stride + (h * a.group + row - tok * a.group) * D + d, y);
        } else {
          float* to = a.part_o + (slot * kRows + in_chunk) * D + d;
#pragma unroll
          for (int n = 0; n < E; n += 2) *reinterpret_cast<float2*>(to + n) = make_float2(y[n], y[n + 1]);
          if (wave == 0 && g == 0) {
            a.part_ml[2 * (slot * kRows + in_chunk)] = best;
            a.part_ml[2 * (slot * kRows + in_chunk) + 1] = all;
          }
        }
      }
      __syncthreads();
    }
    at += t1 - t0;
  }
}

// Adds the parts of what the cuts of the line divided.  Workgroup x: the x-th (request, key head, chunk) where there are no more of
// them than parts, else the one that the x-th cut divides, if it is its first cut; y: rows.  A quarter of a wavefront (or less)
// has a row's D elements, the others take the next parts.
template <typename T, int D>
__global__ void __launch_bounds__(256) join_kernel(Attend a, int chunk_rows) {
  constexpr int kLanes = D / 4, kAtOnce = 256 / kLanes;      // 16, 24, 32 or 64 threads a part
  __shared__ int64_t ends[SPQR_MAX_REQUESTS];
  __shared__ int64_t wave_sums[4];
  __shared__ float so[kAtOnce][D], sm[kAtOnce], sl[kAtOnce];
  const int tid = threadIdx.x;
  const int64_t work = scan_requests(a, chunk_rows, ends, wave_sums);
  const int64_t part = part_size(a, work);
  for (int64_t cut = blockIdx.x + 1; cut * part < work; cut += gridDim.x) {
    const int64_t x = cut * part;
    const int r = find_request(ends, a.requests, x);
    const Request rq = request_of(a, r, chunk_rows);
    const int64_t first = r == 0 ? 0 : ends[r - 1];
    const int pair = which_pair(x - first, rq.tiles);
    const int64_t from = first + (int64_t)pair * rq.tiles, to = from + rq.tiles;
    if (x == from || x - part > from) continue;                // divides nothing; not the first cut
    const int h = pair / rq.chunks, chunk = pair - h * rq.chunks;
    const int row0 = chunk * chunk_rows, live_rows = min(rq.rows * a.group - row0, chunk_rows);
    const int64_t w0 = cut - 1, count = parts_to(to - 1, part) - w0;
    const int mine = tid / kLanes, d = (tid - mine * kLanes) * 4;
    for (int row = blockIdx.y; row < live_rows; row += gridDim.y) {
      float best = -INFINITY, all = 0.f;
      f32x4 y = {0.f, 0.f, 0.f, 0.f};
      if (mine < kAtOnce) {
#pragma unroll 4
        for (int64_t i = mine; i < count; i += kAtOnce) {
          const int64_t slot = 2 * (w0 + i) + ((w0 + i) * part >= from ? 0 : 1), at = slot * chunk_rows + row;
          const float m = a.part_ml[2 * at], l = a.part_ml[2 * at + 1];
          const f32x4 v = *reinterpret_cast<const f32x4*>(a.part_o + at * D + d);
          const float now = fmaxf(best, m);
          const float old = best == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(best - now), c = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - now);
          all = all * old + l * c;
          y = y * old + v * c;
          best = now;
        }
        *reinterpret_cast<f32x4*>(&so[mine][d]) = y;
        if (d == 0) { sm[mine] = best; sl[mine] = all; }
      }
      __syncthreads();
      if (tid < D / 2) {
        float top = -INFINITY, l = 0.f, y0 = 0.f, y1 = 0.f;
        for (int i = 0; i < kAtOnce; ++i) top = fmaxf(top, sm[i]);
        for (int i = 0; i < kAtOnce; ++i) {
          const float c = sm[i] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sm[i] - top);
          l = fmaf(c, sl[i], l);
          y0 = fmaf(c, so[i][2 * tid], y0);
          y1 = fmaf(c, so[i][2 * tid + 1], y1);
        }
        const float c = l == 0.f ? 0.f : 1.f / l;
        const int full = row0 + row, tok = token_of(a, full);
        T* out = static_cast<T*>(a.out) + (int64_t)(rq.first_row + tok) * a.out_stride + (h * a.group + full - tok * a.group) * D + 2 * tid;
        *reinterpret_cast<uint32_t*>(out) = l == 0.f ? 0 : pack<T>(y0 * c, y1 * c);
      }
      __syncthreads();
    }
  }
}

template <typename T, int D>
hipError_t launch_attend(const Attend& a, const AttendPlan& p, hipStream_t st) {
  const dim3 grid(p.workgroups), block(256);
  if (p.rows == 16) hipLaunchKernelGGL((attend_kernel<T, D, 1>), grid, block, 0, st, a);
  else if (p.rows == 32) hipLaunchKernelGGL((attend_kernel<T, D, 2>), grid, block, 0, st, a);
  else if constexpr (D < 256) hipLaunchKernelGGL((attend_kernel<T, D, 4>), grid, block, 0, st, a);
  else return hipErrorInvalidValue;
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((join_kernel<T, D>), dim3(p.join_x, p.join_y), block, 0, st, a, p.rows);
  return hipGetLastError();
}

}  // namespace spqr_srv
#endif
