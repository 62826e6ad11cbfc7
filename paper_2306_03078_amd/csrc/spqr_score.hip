// Log probabilities of given tokens, entropy and the most probable tokens of rows of logits (spqr_token_logprobs).
#include "spqr_block.h"

namespace spqr_blk {

constexpr float kLog2e = 1.44269504088896341f;
constexpr float kLowest = -3.402823466e38f;
constexpr int kGroups = 64;                      // groups of threads whose maxima give the bound
constexpr int kCandidates = 2048;                // logits that pass it which there is room for

// A row's (or a thread's) softmax so far, c = scale * log2(e): max the largest logit (or the lowest number), sum the sum of
// 2^((l - max) c), dot that of (l - max) c 2^((l - max) c).
struct Soft { float max, sum, dot; };

__device__ __forceinline__ void rebase(Soft& s, float max, float c) {
  const float d = fmaxf((s.max - max) * c, -1000.f);       // 2^-1000 is 0; a finite one, so that 0 times it is 0
  const float f = __builtin_amdgcn_exp2f(d);
  s.dot = f * fmaf(d, s.sum, s.dot);
  s.sum *= f;
  s.max = max;
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

template <typename T, int NT>
__global__ void __launch_bounds__(NT) score_kernel(spqr_token_logprobs_t p) {
  constexpr int WAVES = NT / 64;
  __shared__ Soft parts[WAVES];
  __shared__ float maxima[NT];
  __shared__ uint64_t cand[kCandidates];
  __shared__ uint64_t best[SPQR_MAX_TOP];
  __shared__ int found;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = p.vocab;
  const int64_t r = blockIdx.x;
  const T* row = static_cast<const T*>(p.logits) + r * p.stride;
  const float c = p.scale * kLog2e;
  Soft s{kLowest, 0.f, 0.f};
  for (int at = 8 * tid; at < n; at += 8 * NT) {
    float v[8];
    load_logits(row, at, n, v);
    float top = v[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) top = fmaxf(top, v[e]);
    if (top > s.max) rebase(s, top, c);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float d = (v[e] - s.max) * c, x = __builtin_amdgcn_exp2f(d);
      s.sum += x;
      s.dot += x == 0.f ? 0.f : x * d;
    }
  }
  const float mine = s.max;                      // the lowest number also where there is only -infinity
  maxima[tid] = mine;
  if (tid == 0) found = 0;
  for (int d = 32; d > 0; d >>= 1) {
    Soft o{__shfl_xor(s.max, d), __shfl_xor(s.sum, d), __shfl_xor(s.dot, d)};
    const float max = fmaxf(s.max, o.max);
    rebase(s, max, c);
    rebase(o, max, c);
    s.sum += o.sum;
    s.dot += o.dot;
  }
  if (lane == 0) parts[wave] = s;
  __syncthreads();
  s = parts[0];
  for (int w = 1; w < WAVES; ++w) {
    Soft o = parts[w];
    const float max = fmaxf(s.max, o.max);
    rebase(s, max, c);
    rebase(o, max, c);
    s.sum += o.sum;
    s.dot += o.dot;
  }
  const double log_sum = log((double)s.sum);     // -infinity for a row of -infinity only
  auto logprob = [&](float x) { return (float)((s.sum == 0.f ? -INFINITY : ((double)x - s.max) * p.scale) - (s.sum == 0.f ? 0.0 : log_sum)); };
  for (int g = tid; g < p.given; g += NT) {
    const int64_t at = r * p.given + g;
    const int id = p.tokens[at];
    p.logprob[at] = id >= 0 && id < n ? logprob((float)row[id]) : 0.f;
  }
  if (tid == 0 && p.entropy) p.entropy[r] = s.sum == 0.f ? 0.f : (float)(log_sum - (double)s.dot / s.sum * 0.693147180559945309);
  const int k = p.top;
  if (k == 0) return;
  // The k-th largest of the maxima of disjoint groups is no larger than the k-th largest of all: what is below is out.
  float g = maxima[lane];
  for (int w = 1; w < WAVES; ++w) g = fmaxf(g, maxima[64 * w + lane]);
  int rank = 0;
  for (int i = 0; i < 64; ++i) {
    const float o = __shfl(g, i);
    rank += o > g || (o == g && i < lane);
  }
  const float bound = __shfl(g, __ffsll(__ballot(rank == k - 1)) - 1);
  if (mine >= bound)
    for (int at = 8 * tid; at < n; at += 8 * NT) {
      float v[8];
      load_logits(row, at, n, v);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (v[e] >= bound) {
          const int to = atomicAdd(&found, 1);
          if (to < kCandidates) cand[to] = key_of(v[e], at + e);
        }
    }
  __syncthreads();
  int count = found;
  if (count > kCandidates) {
    // Many equal logits around the bound: one after the other, each the best below the last.
    uint64_t last = ~0ull;
    for (count = 0; count < k; ++count) {
      uint64_t b = 0;
      if (mine >= bound)
        for (int at = 8 * tid; at < n; at += 8 * NT) {
          float v[8];
          load_logits(row, at, n, v);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const uint64_t key = key_of(v[e], at + e);
            if (v[e] >= bound && key < last && key > b) b = key;
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
    __syncthreads();
  } else {
    for (int i = tid; i < count; i += NT) {
      const uint64_t key = cand[i];
      int before = 0;
      for (int j = 0; j < count; ++j) before += cand[j] > key;
      if (before < k) best[before] = key;
    }
    __syncthreads();
    count = min(count, k);
  }
  for (int i = tid; i < k; i += NT) {
    const uint64_t key = i < count ? best[i] : 0;
    const int64_t at = r * k + i;
    p.top_token[at] = i < count ? (int32_t)~(uint32_t)key : -1;
    p.top_logprob[at] = i < count ? logprob(unordered((uint32_t)(key >> 32))) : -INFINITY;
  }
}

static int check_scores(const spqr_token_logprobs_t* p) {
  if (!p) return SPQR_ERR_NULL;
  if (p->rows < 0 || p->vocab < 1 || p->vocab >= 1 << 24) return SPQR_ERR_SHAPE;
  if (p->given < 0 || p->given > SPQR_MAX_GIVEN || p->top < 0 || p->top > SPQR_MAX_TOP) return SPQR_ERR_PARAM;
  return SPQR_OK;
}

template <typename T>
static int launch_score(const spqr_token_logprobs_t& p, hipStream_t st) {
  hipLaunchKernelGGL((score_kernel<T, 1024>), dim3(p.rows), dim3(1024), 0, st, p);
  return launched();
}

}  // namespace spqr_blk

using namespace spqr_blk;

extern "C" int64_t spqr_token_logprobs_workspace_bytes(const spqr_token_logprobs_t* p) {
  const int rc = check_scores(p);
  return rc ? rc : 0;
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
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if (p->dtype == SPQR_F32) return launch_score<float>(*p, st);
  if (p->dtype == SPQR_F16) return launch_score<_Float16>(*p, st);
  return launch_score<__bf16>(*p, st);
}
