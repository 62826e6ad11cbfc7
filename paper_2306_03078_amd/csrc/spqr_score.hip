// Log probabilities of given tokens, entropy and the most probable tokens of rows of logits (spqr_token_logprobs).
#include "spqr_block.h"

namespace spqr_blk {

constexpr float kLog2e = 1.44269504088896341f;
constexpr int kCandidates = 2048;                // logits that can be among the best which there is room for
constexpr int kJoined = 1024;                    // keys of the parts of a row
constexpr int kPartGroups = 512, kShortest = 4096;         // rows are cut for so many workgroups, parts no shorter than this
constexpr int kResident = 1024, kMiddling = 49152;         // workgroups of 512 threads that run at once; rows that 256 threads take where there are more

// c = scale * log2(e), as binary32: probabilities go by powers of two, 2^(l c - ref) over their sum.  A thread's reference is a whole number near its
// largest l c, so that one fused multiply and subtract gives l c - ref with one rounding; sums of another reference move by a power of two.
// It moves up when a logit passes it by 2^8, and never lies below -2^24.  Where the largest l c is 2^24 or more in size (or has no number), a loop that
// subtracts the largest logit first takes the row again: there l c has no bits below 1, its rounding (128 and more from 2^31 on) would be a power of
// two by itself.  For the same reason a thread whose logits all lie below -2^24 (masks by -1e10 and the like) keeps the lowest reference:
// theirs are powers of two that are 0 beside any other logit.
constexpr float kFar = 16777216.f;               // 2^24
constexpr double kLn2 = 0.693147180559945309;

struct Soft { float ref, sum, dot; };            // sum of 2^(l c - ref), of (l c - ref) 2^(l c - ref)

__device__ __forceinline__ void rebase(Soft& s, float ref) {
  const float d = fmaxf(s.ref - ref, -1000.f), f = __builtin_amdgcn_exp2f(d);    // 2^-1000 is 0; a finite one, so that 0 times it is 0
  s.dot = f * fmaf(d, s.sum, s.dot);
  s.sum *= f;
  s.ref = ref;
}

// A part of a row, or all of it: what the parts of a row are joined from.
struct Part { double ref; float sum, dot, max; };          // sum 0: there is no logit above -infinity; max: the largest

// A wavefront's parts, one a lane, as one.
__device__ __forceinline__ Part joined(Part p) {
  const int lane = threadIdx.x & 63;
  const double mine = p.sum == 0.f ? -1e300 : p.ref;       // (NaN is a sum)
  double ref = mine;
  float max = p.max;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    ref = fmax(ref, __shfl_xor(ref, d));
    max = fmaxf(max, __shfl_xor(max, d));
  }
  const float d = (float)fmax(mine - ref, -1000.0), f = __builtin_amdgcn_exp2f(d);
  return Part{ref, spqr::wave_allreduce(f * p.sum, lane), spqr::wave_allreduce(f * fmaf(d, p.sum, p.dot), lane), max};
}

// Logits in the order of their values as whole numbers, the two zeros alike.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t k) { return __uint_as_float(k ^ (k >> 31 ? 0x80000000u : 0xFFFFFFFFu)); }
// A candidate: larger is better, the lowest id first among equal logits.
__device__ __forceinline__ uint64_t key_of(float x, int id) { return (uint64_t)ordered(x) << 32 | (uint32_t)~id; }

template <typename T>
__device__ __forceinline__ void load_logits(const T* row, int at, int n, float (&v)[8]) {
  load_row8(row, at, n, v);
  if (at + 8 > n)
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (at + e >= n) v[e] = -INFINITY;
}

// log2 of a positive number: of its significand, near 1, by the card's instruction (off by 2^-23 or so), and its exponent.
__device__ __forceinline__ double log2_of(float x) {
  int e;
  float m = frexpf(x, &e);                       // 0.5 .. 1
  if (m < 0.70710678f) { m *= 2.f; --e; }
  return (double)e + (double)__builtin_amdgcn_logf(m);
}

// A number that the k-th largest of a wavefront's 64 is not below, and no more than its last 12 bits under it: bit by bit, by how many reach it.  (A
// loop of few instructions: code that runs once waits for its own instructions, 64 comparisons written out took 2 us more.)
__device__ __forceinline__ uint32_t kth_largest(uint32_t key, int k) {
  uint32_t bound = 0;
#pragma unroll 1
  for (uint32_t bit = 0x80000000u; bit >= 0x1000u; bit >>= 1)
    if (__popcll(__ballot(key >= (bound | bit))) >= k) bound |= bit;
  return bound;
}

// What is written of a row, once its sums are known: l c was rounded alike in all of them, so that it is differences from the largest logit
// that count, and that one's own come from the scale itself.
struct Row {
  Part soft;
  double scale, log_sum;                         // of 2^((l - max) c)
  __device__ __forceinline__ Row(const Part& p, float s)
      : soft(p), scale(s), log_sum(p.sum == 0.f ? 0.0 : log2_of(p.sum) + (p.ref - (double)p.max * (s * kLog2e))) {}
  __device__ __forceinline__ float logprob(float x) const {
    return soft.sum == 0.f ? -INFINITY : (float)(((double)x - soft.max) * scale - log_sum * kLn2);
  }
  __device__ __forceinline__ float entropy() const { return soft.sum == 0.f ? 0.f : (float)((log2_of(soft.sum) - (double)soft.dot / soft.sum) * kLn2); }
};

template <typename T>
__device__ __forceinline__ void write_row(const spqr_token_logprobs_t& p, int64_t r, const Row& row, int tid, int threads) {
  const T* logits = static_cast<const T*>(p.logits) + r * p.stride;
  for (int g = tid; g < p.given; g += threads) {
    const int64_t at = r * p.given + g;
    const int id = p.tokens[at];
    p.logprob[at] = id >= 0 && id < p.vocab ? row.logprob((float)logits[id]) : 0.f;
  }
  if (tid == 0 && p.entropy) p.entropy[r] = row.entropy();
}
__device__ __forceinline__ void write_top(const spqr_token_logprobs_t& p, int64_t r, const Row& row, const uint64_t* best, int count, int tid, int threads) {
  for (int i = tid; i < p.top; i += threads) {
    const uint64_t key = i < count ? best[i] : 0;
    const int64_t at = r * p.top + i;
    p.top_token[at] = i < count ? (int32_t)~(uint32_t)key : -1;
    // (a row with a NaN or +infinity has no log probabilities, in places without a token neither)
    p.top_logprob[at] = i < count ? row.logprob(unordered((uint32_t)(key >> 32))) : row.soft.sum != row.soft.sum ? NAN : -INFINITY;
  }
}

// The best `k` of `count` different keys, in order, by how many are better.
__device__ __forceinline__ void rank_keys(const uint64_t* keys, int count, int k, uint64_t* best, int tid, int threads) {
  for (int i = tid; i < count; i += threads) {
    const uint64_t key = keys[i];
    int before = 0;
    for (int j = 0; j < count; ++j) before += keys[j] > key;
    if (before < k) best[before] = key;
  }
}

// A part of a row a workgroup (blockIdx.y of gridDim.y): one pass for the sums and every thread's largest logit; then the few threads that can
// have one of the best look at theirs again.  WHOLE: all of the row.
template <typename T, int NT, bool WHOLE>
__global__ void __launch_bounds__(NT) score_kernel(spqr_token_logprobs_t p, int length, Part* parts, uint64_t* keys) {
  constexpr int WAVES = NT / 64, AHEAD = WHOLE ? 4 : 2;      // (parts are short)
  __shared__ float maxima[NT];
  __shared__ float red[3][WAVES];
  __shared__ uint64_t cand[kCandidates];
  __shared__ uint64_t best[SPQR_MAX_TOP];
  __shared__ int found;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t r = blockIdx.x;
  const int begin = WHOLE ? 0 : (int)blockIdx.y * length, n = WHOLE ? p.vocab : min(length, p.vocab - begin);
  const T* row = static_cast<const T*>(p.logits) + r * p.stride + begin;
  const float c = p.scale * kLog2e;

  Soft s{-kFar, 0.f, 0.f};
  // a thread's largest logit, the stretch of its logits that has it, and the largest of the other stretches
  float mine = -INFINITY, other = -INFINITY;
  int where = 0;
  auto note = [&](float top, int at) {
    other = fmaxf(other, fminf(mine, top));
    where = top > mine ? at : where;
    mine = fmaxf(mine, top);
  };
  auto take = [&](const float (&v)[8]) {
    const float largest = fmaxf(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), fmaxf(fmaxf(v[4], v[5]), fmaxf(v[6], v[7])));
    const float top = largest * c;
    if (top > s.ref + 8.f) rebase(s, rintf(top));
    float sum = 0.f, dot = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float d = fmaf(v[e], c, -s.ref), x = __builtin_amdgcn_exp2f(d);
      sum += x;
      dot = fmaf(x, fmaxf(d, -1000.f), dot);     // (-infinity times 0; a NaN is in the sum)
    }
    s.sum += sum;
    s.dot += dot;
    return largest;
  };
  int at = 8 * tid;
  for (; at + 8 * NT * (AHEAD - 1) + 8 <= n; at += 8 * NT * AHEAD) {
    Run8<T> x[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) x[i] = *reinterpret_cast<const Run8<T>*>(row + at + 8 * NT * i);
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = (float)x[i].e[e];
      top = fmaxf(top, take(v));
    }
    note(top, at);
  }
  const int rest = at;                           // behind here a stretch is eight logits, before it AHEAD times as many
  for (; at < n; at += 8 * NT) {
    float v[8];
    load_logits(row, at, n, v);
    note(take(v), at);
  }
  // the largest of all, and sums by its reference
  maxima[tid] = mine;
  if (tid == 0) found = 0;
  float top = mine, ref = s.ref;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    top = fmaxf(top, __shfl_xor(top, d));
    ref = fmaxf(ref, __shfl_xor(ref, d));
  }
  if (lane == 0) { red[0][wave] = top; red[1][wave] = ref; }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < WAVES; ++w) { top = fmaxf(top, red[0][w]); ref = fmaxf(ref, red[1][w]); }
  Part part;
  part.ref = ref;
  part.max = top;
  const bool far = top > -INFINITY && !(fabsf(top * c) < kFar);
  if (far) {                                     // by the largest logit itself
    part.ref = (double)top * c;
    s.sum = s.dot = 0.f;
    for (int i = 8 * tid; i < n; i += 8 * NT) {
      float v[8];
      load_logits(row, i, n, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float d = (v[e] - top) * c, x = __builtin_amdgcn_exp2f(d);
        s.sum += x;
        s.dot = fmaf(x, fmaxf(d, -1000.f), s.dot);
      }
    }
  } else {
    rebase(s, ref);
  }
  s.sum = spqr::wave_allreduce(s.sum, lane);
  s.dot = spqr::wave_allreduce(s.dot, lane);
  __syncthreads();                               // everyone has read the largest ones
  if (lane == 0) { red[0][wave] = s.sum; red[1][wave] = s.dot; }
  // The k-th largest of the maxima of disjoint groups of threads is no larger than the k-th largest of all: what is below is out.
  const int k = p.top;
  float bound = INFINITY;
  if (k > 0) {
    float g = maxima[lane];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) g = fmaxf(g, maxima[64 * w + lane]);
    const uint32_t key = kth_largest(ordered(g), k);
    bound = key <= 0x007FFFFFu ? -INFINITY : unordered(key);                              // (0x007FFFFF: -infinity; below it are no numbers)
    if (mine >= bound && mine > -INFINITY) {
      // as a rule one stretch has all that count
      const bool one = other < bound;
      const int last = one ? where < rest ? where + 8 * NT * AHEAD : where + 1 : n;
      for (int i = one ? where : 8 * tid; i < last; i += 8 * NT * AHEAD) {
        float v[AHEAD][8];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) load_logits(row, min(i + 8 * NT * k, n - 1), n, v[k]);
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
          const int from = i + 8 * NT * k;
          if (from < min(last, n))
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (v[k][e] >= bound && v[k][e] > -INFINITY) {
                const int to = atomicAdd(&found, 1);
                if (to < kCandidates) cand[to] = key_of(v[k][e], begin + from + e);
              }
        }
      }
    }
  }
  __syncthreads();
  part.sum = part.dot = 0.f;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) { part.sum += red[0][w]; part.dot += red[1][w]; }
  if (k > 0) {
    int count = found;
    if (count > kCandidates) {
      // Many equal logits around the bound (all of a row alike; masks by the type's lowest value that leave fewer than k): one after the other, each the
      // best below the last, the row read again for each.  2048 rows of 65537 with 10 alternatives 663 us in place of 61, one row of 32000 28 in place of 10.
      uint64_t last = ~0ull;
      for (count = 0; count < k; ++count) {
        uint64_t b = 0;
        if (mine >= bound && mine > -INFINITY)
          for (int i = 8 * tid; i < n; i += 8 * NT) {
            float v[8];
            load_logits(row, i, n, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const uint64_t key = key_of(v[e], begin + i + e);
              if (v[e] >= bound && v[e] > -INFINITY && key < last && key > b) b = key;
            }
          }
        for (int d = 32; d > 0; d >>= 1) {
          const uint64_t o = __shfl_xor(b, d);
          b = o > b ? o : b;
        }
        __syncthreads();
        if (lane == 0) cand[wave] = b;
        __syncthreads();
        b = cand[0];
        for (int w = 1; w < WAVES; ++w) b = cand[w] > b ? cand[w] : b;
        if (b == 0) break;
        last = b;
        if (tid == 0) best[count] = b;
      }
    } else {
      rank_keys(cand, count, k, best, tid, NT);
      count = min(count, k);
    }
    __syncthreads();
    if (WHOLE) {
      const Row of(part, p.scale);
      write_top(p, r, of, best, count, tid, NT);
    } else {
      for (int i = tid; i < k; i += NT) keys[(r * gridDim.y + blockIdx.y) * k + i] = i < count ? best[i] : 0;
    }
  }
  if (WHOLE) write_row<T>(p, r, Row(part, p.scale), tid, NT);
  else if (tid == 0) parts[r * gridDim.y + blockIdx.y] = part;
}

// The parts of a row, a workgroup a row; their best by the same bound.
template <typename T>
__global__ void __launch_bounds__(256) score_join_kernel(spqr_token_logprobs_t p, int count, const Part* parts, const uint64_t* keys) {
  __shared__ uint64_t maxima[256], cand[kJoined], best[SPQR_MAX_TOP];
  __shared__ int found;
  const int tid = threadIdx.x, lane = tid & 63, k = p.top;
  const int64_t r = blockIdx.x;
  uint64_t mine[kJoined / 256], top = 0;
#pragma unroll
  for (int i = 0; i < kJoined / 256; ++i) {
    mine[i] = tid + 256 * i < count * k ? keys[r * count * k + tid + 256 * i] : 0;
    top = mine[i] > top ? mine[i] : top;
  }
  const Part part = lane < count ? parts[r * count + lane] : Part{0.0, 0.f, 0.f, -INFINITY};
  maxima[tid] = top;
  if (tid == 0) found = 0;
  const Row row(joined(part), p.scale);
  write_row<T>(p, r, row, tid, 256);
  if (k == 0) return;
  __syncthreads();
  uint64_t g = maxima[lane];
#pragma unroll
  for (int w = 1; w < 4; ++w) g = maxima[64 * w + lane] > g ? maxima[64 * w + lane] : g;
  const uint64_t bound = (uint64_t)kth_largest((uint32_t)(g >> 32), k) << 32;
#pragma unroll
  for (int i = 0; i < kJoined / 256; ++i)
    if (mine[i] != 0 && mine[i] >= bound) cand[atomicAdd(&found, 1)] = mine[i];
  __syncthreads();
  rank_keys(cand, found, k, best, tid, 256);
  __syncthreads();
  write_top(p, r, row, best, min(found, k), tid, 256);
}

// How many parts a row is cut into, and how long they are.
struct Cut { int parts, length; };
static Cut cut_of(int64_t rows, int vocab, int top) {
  int64_t parts = rows > 0 ? kPartGroups / rows : 1;
  const int64_t by_length = (vocab + kShortest - 1) / kShortest, by_keys = top > 0 ? kJoined / top : 64;
  if (parts > by_length) parts = by_length;
  if (parts > by_keys) parts = by_keys;
  if (parts > 64) parts = 64;
  if (parts <= 1) return Cut{1, vocab};
  const int length = (int)(((vocab + parts - 1) / parts + 2047) / 2048 * 2048);
  return Cut{(vocab + length - 1) / length, length};
}

static int check_scores(const spqr_token_logprobs_t* p) {
  if (!p) return SPQR_ERR_NULL;
  if (p->rows < 0 || p->vocab < 1 || p->vocab >= 1 << 24) return SPQR_ERR_SHAPE;
  if (p->given < 0 || p->given > SPQR_MAX_GIVEN || p->top < 0 || p->top > SPQR_MAX_TOP) return SPQR_ERR_PARAM;
  return SPQR_OK;
}

// Rows of one launch: 2^31 threads (a grid of 2^32 threads in one direction loses what is beyond them, without an error).
constexpr int kMostRows = 1 << 22;

template <typename T>
static spqr_token_logprobs_t rows_from(const spqr_token_logprobs_t& p, int64_t from) {
  spqr_token_logprobs_t q = p;
  q.rows = p.rows - from < kMostRows ? (int)(p.rows - from) : kMostRows;
  q.logits = static_cast<const T*>(p.logits) + from * p.stride;
  if (p.given > 0) { q.tokens = p.tokens + from * p.given; q.logprob = p.logprob + from * p.given; }
  if (p.entropy) q.entropy = p.entropy + from;
  if (p.top > 0) { q.top_token = p.top_token + from * p.top; q.top_logprob = p.top_logprob + from * p.top; }
  return q;
}

template <typename T>
static int launch_score(const spqr_token_logprobs_t& p, hipStream_t st) {
  const Cut cut = cut_of(p.rows, p.vocab, p.top);
  Part* parts = static_cast<Part*>(p.workspace);
  uint64_t* keys = reinterpret_cast<uint64_t*>(parts + (int64_t)p.rows * cut.parts);
  if (cut.parts == 1) {
    // 256 threads where a row is short, or where rows are more than 512 threads each have room for at once and not so long that the row's length is all
    // that counts: 2048 rows of 10001 20 us (512 threads: 28), of 32000 39 (45), of 48000 54 (57), but of 65537 80 (74); 600 rows of 32000 22 (19), 1024 of 40000 42 (38).
    const bool small = p.vocab <= 8192 || (p.rows > kResident && p.vocab <= kMiddling);
    for (int64_t from = 0; from < p.rows; from += kMostRows) {
      const spqr_token_logprobs_t q = rows_from<T>(p, from);
      if (small) hipLaunchKernelGGL((score_kernel<T, 256, true>), dim3(q.rows), dim3(256), 0, st, q, q.vocab, nullptr, nullptr);
      else hipLaunchKernelGGL((score_kernel<T, 512, true>), dim3(q.rows), dim3(512), 0, st, q, q.vocab, nullptr, nullptr);
    }
    return launched();
  }
  hipLaunchKernelGGL((score_kernel<T, 256, false>), dim3(p.rows, cut.parts), dim3(256), 0, st, p, cut.length, parts, keys);
  hipLaunchKernelGGL((score_join_kernel<T>), dim3(p.rows), dim3(256), 0, st, p, cut.parts, parts, keys);
  return launched();
}

static int64_t workspace_bytes(int64_t rows, const spqr_token_logprobs_t* p) {
  const Cut cut = cut_of(rows, p->vocab, p->top);
  return cut.parts == 1 ? 0 : rows * cut.parts * ((int64_t)sizeof(Part) + 8 * p->top);
}

}  // namespace spqr_blk

using namespace spqr_blk;

extern "C" int64_t spqr_token_logprobs_workspace_bytes(const spqr_token_logprobs_t* p) {
  const int rc = check_scores(p);
  if (rc) return rc;
  int64_t most = 0;              // of any number of rows up to these: above kPartGroups rows are whole
  for (int64_t rows = 1; rows <= p->rows && rows <= kPartGroups; ++rows) {
    const int64_t bytes = workspace_bytes(rows, p);
    most = bytes > most ? bytes : most;
  }
  return (most + 255) / 256 * 256;
}

extern "C" int spqr_token_logprobs(const spqr_token_logprobs_t* p, void* stream) {
  const int rc = check_scores(p);
  if (rc) return rc;
  if (!known(p->dtype)) return SPQR_ERR_DTYPE;
  if (!(p->scale > 0.f) || !isfinite(p->scale * kLog2e) || !(p->scale * kLog2e > 0.f)) return SPQR_ERR_PARAM;
  if (p->stride < p->vocab || p->stride > INT64_MAX / 8 / (p->rows > 0 ? p->rows : 1)) return SPQR_ERR_SHAPE;
  if (p->rows == 0) return SPQR_OK;
  if (!p->logits || (p->given > 0 && (!p->tokens || !p->logprob)) || (p->top > 0 && (!p->top_token || !p->top_logprob)) ||
      (p->given == 0 && p->top == 0 && !p->entropy))
    return SPQR_ERR_NULL;
  if (!aligned(p->logits, size_of(p->dtype)) || !aligned(p->tokens, 4) || !aligned(p->logprob, 4) || !aligned(p->entropy, 4) ||
      !aligned(p->top_token, 4) || !aligned(p->top_logprob, 4))
    return SPQR_ERR_ALIGN;
  const int64_t need = workspace_bytes(p->rows, p);
  if (need > 0) {
    if (!p->workspace) return SPQR_ERR_NULL;
    if (!aligned(p->workspace, 256)) return SPQR_ERR_ALIGN;
    if (p->workspace_bytes < need) return SPQR_ERR_WORKSPACE;
  }
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if (p->dtype == SPQR_F32) return launch_score<float>(*p, st);
  if (p->dtype == SPQR_F16) return launch_score<_Float16>(*p, st);
  return launch_score<__bf16>(*p, st);
}
