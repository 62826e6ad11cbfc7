// The steps around the attention of a decode step over a paged cache: page tables, slots and masks from request lengths
// (spqr_cache_plan), rotary embedding and store (spqr_cache_store), the accepted path's rows (spqr_cache_keep).
#include "spqr_serve.h"

namespace spqr_srv {

__device__ __forceinline__ int clamp_to(int64_t v, int64_t hi) { return (int)(v < 0 ? 0 : v > hi ? hi : v); }

// ---------------------------------------------------------------------------------------------------------------------
// Page tables, slots, positions, masks.
// ---------------------------------------------------------------------------------------------------------------------
struct Pages {                   // what a request needs of the ring
  int fresh, held, need;
  int64_t cut;                   // pages that the table has no columns for
};

__device__ __forceinline__ Pages pages_of(const spqr_step_t& s, int r, int log_page) {
  Pages p;
  const int64_t cached = max(0, s.cached[r]);
  p.fresh = min(max(0, s.fresh[r]), SPQR_MAX_FRESH);
  p.held = min(max(0, s.held[r]), s.max_pages);
  const int64_t whole = (cached + p.fresh + s.page - 1) >> log_page;
  p.need = (int)min(whole, (int64_t)s.max_pages);
  p.cut = whole - p.need;
  return p;
}

__device__ __forceinline__ int64_t wave_sum(int64_t v) {
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
  return v;
}

// One workgroup a request, a thread a new token.  Each workgroup sums over the requests by itself (12 bytes a request out of the
// L2): one launch, where a scan of its own in front would be two.  What bounds it are trips to memory one after the other:
// lengths, then everything that they place (pages, parents) asked for at once, then the stores.  Ancestors by doubling: after
// k rounds a token's row of bits has its 2^k nearest ones, so a chain of 256 takes 8 rounds in LDS.  16 trees of up to 16 tokens:
// 5.9 us; 256 prompts of up to 256 tokens: 4.8 us, 1.4 MB written.
__global__ void __launch_bounds__(256) plan_kernel(spqr_step_t s) {
  __shared__ int64_t part[4][5];
  __shared__ int rows_part[4][2];
  __shared__ uint64_t bits[SPQR_MAX_FRESH][4];
  __shared__ int up[SPQR_MAX_FRESH];
  const int r = blockIdx.x, tid = threadIdx.x, R = s.requests, log_page = __ffs(s.page) - 1;
  const bool last = r == R - 1;

  const Pages p = pages_of(s, r, log_page);
  const int64_t cached = max(0, s.cached[r]), taken = s.ends[0], given = s.ends[1];
  // of the requests before this one and (rows, and for the last workgroup the rest) of all: rows, pages wanted, pages given back
  int rows_before = 0, rows_all = 0;
  int64_t sum[5] = {0, 0, 0, 0, 0};          // wanted and given back before; of all; pages cut off
  for (int q = tid; q < R; q += 256) {
    const Pages x = pages_of(s, q, log_page);
    const int64_t want = max(0, x.need - x.held), back = max(0, x.held - x.need);
    rows_all += x.fresh;
    if (q < r) { rows_before += x.fresh; sum[0] += want; sum[1] += back; }
    sum[2] += want; sum[3] += back; sum[4] += x.cut;
  }
  for (int d = 32; d > 0; d >>= 1) {
    rows_before += __shfl_xor(rows_before, d);
    rows_all += __shfl_xor(rows_all, d);
  }
  const int sums = last ? 5 : 2;
  for (int i = 0; i < sums; ++i) {
    sum[i] = wave_sum(sum[i]);
    if ((tid & 63) == 0) part[tid >> 6][i] = sum[i];
  }
  if ((tid & 63) == 0) { rows_part[tid >> 6][0] = rows_before; rows_part[tid >> 6][1] = rows_all; }
  __syncthreads();
  const int64_t first = part[0][0] + part[1][0] + part[2][0] + part[3][0], first_back = part[0][1] + part[1][1] + part[2][1] + part[3][1];
  const int base = min(rows_part[0][0] + rows_part[1][0] + rows_part[2][0] + rows_part[3][0], s.tokens);
  const int total = min(rows_part[0][1] + rows_part[1][1] + rows_part[2][1] + rows_part[3][1], s.tokens);
  const int rows = min(p.fresh, s.tokens - base), want = max(0, p.need - p.held), back = max(0, p.held - p.need);
  const int64_t P = s.pages, free_pages = min(max((int64_t)0, given - taken), P);
  const int64_t ring_from = (uint64_t)taken < 0x100000000ull ? (uint32_t)taken % (uint32_t)P : (taken % P + P) % P;
  int32_t* table = s.table + (int64_t)r * s.max_pages;

  // places of the ring behind ring_from (less than P, as all numbers of free pages are)
  auto in_ring = [&](int64_t i) { const int64_t at = ring_from + i; return at < P ? at : at - P; };
  // the page at place i of those that the request is to take
  auto ring_page = [&](int i) { return first + i < free_pages ? s.pool[in_ring(first + i)] : -1; };
  // the first of each kind of load together, the stores behind them
  const int64_t key = cached + tid, at = key >> log_page;
  int id = -1, near = -1, page0 = -1, gone0 = 0;
  if (tid < rows) {
    id = at >= s.max_pages ? -1 : at < p.held ? table[at] : ring_page((int)at - p.held);
    near = s.parent != nullptr ? s.parent[base + tid] : tid - 1;
  }
  if (tid < want) page0 = ring_page(tid);
  if (tid < back) gone0 = table[p.need + tid];

  for (int i = tid; i < want; i += 256) table[p.held + i] = i == tid ? page0 : ring_page(i);
  // behind the ring's end; what would run into its beginning (more free pages than there are) is left out
  for (int i = tid; i < back; i += 256) {
    const int64_t to = (given - taken) + first_back + i;
    if (to >= 0 && to < P) s.pool[in_ring(to)] = i == tid ? gone0 : table[p.need + i];
  }
  if (tid == 0) {
    s.q_start[r] = base;
    const int64_t granted = min((int64_t)want, max((int64_t)0, free_pages - first));
    s.held_out[r] = p.held > p.need ? p.need : p.held + (int)granted;
    if (last) {
      int64_t all[3];
      for (int i = 0; i < 3; ++i) all[i] = part[0][i + 2] + part[1][i + 2] + part[2][i + 2] + part[3][i + 2];
      s.q_start[R] = total;
      s.ends_out[0] = taken + min(all[0], free_pages);
      s.ends_out[1] = given + all[1];
      s.ends_out[2] = max((int64_t)0, all[0] - free_pages) + all[2];
    }
  }

  uint64_t own[4] = {0, 0, 0, 0};
  int depth = tid;
  if (s.parent == nullptr) {
    for (int w = 0; w < 4; ++w) {
      const int n = min(max(tid + 1 - 64 * w, 0), 64);
      own[w] = n == 0 ? 0 : ~0ull >> (64 - n);
    }
  } else {                       // every wavefront takes part, also one without rows
    for (int w = 0; w < 4; ++w) bits[tid][w] = own[w] = w == tid >> 6 ? 1ull << (tid & 63) : 0;
    int next = near >= 0 && near < tid ? near : -1;
    up[tid] = next;
    while (__syncthreads_or(next >= 0)) {
      int behind = -1;
      if (next >= 0) {
        for (int w = 0; w < 4; ++w) own[w] |= bits[next][w];
        behind = up[next];
      }
      __syncthreads();
      for (int w = 0; w < 4; ++w) bits[tid][w] = own[w];
      up[tid] = next = behind;
    }
    depth = __popcll(own[0]) + __popcll(own[1]) + __popcll(own[2]) + __popcll(own[3]) - 1;
  }
  if (tid < rows) {
    const int64_t t = base + tid;
    s.slot[t] = id >= 0 && id < P ? (int32_t)((int64_t)id * s.page + (key & (s.page - 1))) : -1;
    s.position[t] = (int32_t)min(cached + depth, (int64_t)0x7FFFFFFF);
    for (int w = 0; w < s.mask_words; ++w) s.mask[t * s.mask_words + w] = own[w];
  }
  for (int64_t t = total + (int64_t)r * 256 + tid; t < s.tokens; t += (int64_t)R * 256) {
    s.slot[t] = -1;
    s.position[t] = -1;
    for (int w = 0; w < s.mask_words; ++w) s.mask[t * s.mask_words + w] = 0;
  }
}

// ---------------------------------------------------------------------------------------------------------------------
// Rotary embedding, store.
// ---------------------------------------------------------------------------------------------------------------------
// What spqr_cache_store does with a row, and spqr_cache_keep counts by: a row is in use; its k and v have a place in the cache.
__device__ __forceinline__ bool row_in_use(int position, int rot, int positions) { return position >= 0 && (rot == 0 || position < positions); }
__device__ __forceinline__ bool in_cache(int slot, int slots) { return slot >= 0 && slot < slots; }

struct Store {
  spqr_rows_t x;
  void *q_out, *kc, *vc;         // the caches: those of the layer
  const int32_t *position, *slot;
  const float* rotary;
  int heads, kv_heads, D, page, slots, rot, positions, pairs;
};

template <typename T, int V>
struct alignas(sizeof(T) * V > 16 ? 16 : sizeof(T) * V) Run { T e[V]; };

template <typename X, int V>
__device__ __forceinline__ void load_run(const X* p, float* out) {
  const Run<X, V> x = *reinterpret_cast<const Run<X, V>*>(p);
#pragma unroll
  for (int e = 0; e < V; ++e) out[e] = (float)x.e[e];
}

// A thread turns the same V elements of several heads of one token: the cosines and sines are read once for them.  The partner
// elements of the half-and-half form are read by the thread that owns them too (once from memory, once from the L1).  Memory bounds
// it: 4096 tokens of 80 heads of 128 elements, bfloat16 to bfloat16, 36 us, 4.7 TB/s read and written, as fast as a copy; few
// tokens take a launch, 4.3 us on the card for 16 tokens of 192 heads.
// V = 8 where every row is 16-byte aligned and no 8 elements straddle an end of the rotated part, else V = 1 (the 4096 tokens:
// 82 us; 16 and 64 tokens: equal).
template <typename X, typename T, int V>
__global__ void __launch_bounds__(256) store_kernel(Store a) {
  const int chunks = a.D / V, lanes = 256 / chunks, head0 = threadIdx.x / chunks;
  const int o = (threadIdx.x - head0 * chunks) * V;
  if (head0 >= lanes) return;
  const int64_t t = blockIdx.x;
  const int pos = a.position[t];
  const bool live = row_in_use(pos, a.rot, a.positions);
  const int slot = a.slot[t];
  const bool stored = live && in_cache(slot, a.slots);
  const int half = a.rot / 2;
  const bool turns = live && o < a.rot, upper = o >= half;
  const int partner = a.pairs ? (V == 1 ? o ^ 1 : o) : upper ? o - half : o + half;
  float c[V], s[V];
  if (turns) {
    const float* row = a.rotary + (int64_t)pos * a.rot;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const int i = a.pairs ? (o + e) / 2 : (upper ? o - half : o) + e;
      c[e] = row[i];
      s[e] = row[half + i];
      if (a.pairs ? ((o + e) & 1) == 0 : !upper) s[e] = -s[e];
    }
  }
  const int page = slot / a.page, in_page = slot - page * a.page;
  for (int h = head0 + lanes * blockIdx.y; h < a.heads + 2 * a.kv_heads; h += lanes * gridDim.y) {
    const bool is_q = h < a.heads, is_v = h >= a.heads + a.kv_heads;
    const int g = is_q ? h : is_v ? h - a.heads - a.kv_heads : h - a.heads;
    if (!is_q && !stored) continue;
    float y[V];
#pragma unroll
    for (int e = 0; e < V; ++e) y[e] = 0.f;
    if (live) {
      const X* x = static_cast<const X*>(is_q ? a.x.q : is_v ? a.x.v : a.x.k) +
                   t * (is_q ? a.x.q_stride : is_v ? a.x.v_stride : a.x.k_stride) + g * a.D;
      load_run<X, V>(x + o, y);
      if (turns && !is_v) {
        float z[V];
        if (V == 1 || !a.pairs) {
          load_run<X, V>(x + partner, z);
        } else {
#pragma unroll
          for (int e = 0; e < V; ++e) z[e] = y[V == 1 ? 0 : e ^ 1];
        }
#pragma unroll
        for (int e = 0; e < V; ++e) y[e] = fmaf(y[e], c[e], z[e] * s[e]);
      }
    }
    Run<T, V> out;
#pragma unroll
    for (int e = 0; e < V; ++e) out.e[e] = (T)y[e];
    T* to = is_q ? static_cast<T*>(a.q_out) + (t * a.heads + g) * a.D
                 : static_cast<T*>(is_v ? a.vc : a.kc) + (((int64_t)page * a.kv_heads + g) * a.page + in_page) * a.D;
    *reinterpret_cast<Run<T, V>*>(to + o) = out;
  }
}

template <typename X, typename T>
static int launch_store(const Store& a, int tokens, bool wide, hipStream_t st) {
  const int lanes = 256 / (a.D / (wide ? 8 : 1)), rounds = (a.heads + 2 * a.kv_heads + lanes - 1) / lanes;
  // Few tokens: a round of heads a workgroup (64 tokens of 192 heads: 7.4 us; all of a token's in one 9.0 us).  Many: all of a token's,
  // the cosines stay in registers (256 tokens: 11.4 us; a round each 16.3 us; 1024 tokens 33 and 55 us).
  const int split = tokens <= 128 ? rounds : 1;
  const dim3 grid(tokens, split), block(256);
  if (wide) hipLaunchKernelGGL((store_kernel<X, T, 8>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((store_kernel<X, T, 1>), grid, block, 0, st, a);
  return launched();
}

template <typename T>
static int store_from(int x_dtype, const Store& a, int tokens, bool wide, hipStream_t st) {
  if (x_dtype == SPQR_F32) return launch_store<float, T>(a, tokens, wide, st);
  if (x_dtype == SPQR_F16) return launch_store<_Float16, T>(a, tokens, wide, st);
  return launch_store<__bf16, T>(a, tokens, wide, st);
}

// ---------------------------------------------------------------------------------------------------------------------
// The accepted path.
// ---------------------------------------------------------------------------------------------------------------------
// A workgroup finds the path of its request and moves 256 columns of 16 bytes, each thread its column row by row: the path ascends
// and its a-th entry is at least a, so a row is read before it is overwritten as long as rows are taken in order, eight
// loads ahead of their stores included.  A trip to memory a group of eight rows and one for the path bound it: 4 rows of 32 layers of
// 32 heads of 128 elements 4.5 us; 32 requests of 7 rows, 48 layers of 8 heads (44 MB read and written) 13 us, 3.3 TB/s.
// What spqr_cache_store left out is asked for beside the path, in the same trip (0.3 us of the second).
constexpr int kAhead = 8;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__global__ void __launch_bounds__(256) keep_kernel(spqr_step_t s, const int32_t* __restrict__ last, int64_t columns) {
  __shared__ int64_t from[SPQR_MAX_FRESH], to[SPQR_MAX_FRESH];
  __shared__ bool has_slot[SPQR_MAX_FRESH];
  __shared__ int moved_from, path_end;
  const int r = blockIdx.x, tid = threadIdx.x, log_page = __ffs(s.page) - 1;
  const int base = clamp_to(s.q_start[r], s.tokens), end = clamp_to(s.q_start[r + 1], s.tokens);
  const int rows = min(max(0, end - base), SPQR_MAX_FRESH);
  const int64_t cached = max(0, s.cached[r]);
  const int leaf = last == nullptr ? rows - 1 : last[r];
  const bool path = leaf >= 0 && leaf < rows;
  const bool by_mask = last != nullptr && s.mask_words > 0;
  const bool slotted = tid < rows && (s.slot == nullptr || in_cache(s.slot[base + tid], s.pages * s.page));
  const bool stored = slotted && (s.position == nullptr || row_in_use(s.position[base + tid], s.rotary_dim, s.rotary_positions));
  // thread j: token j is on the path as the rank-th
  int count = path ? leaf + 1 : 0, rank = tid;
  bool on = tid < count;
  if (by_mask) {
    rank = count = 0;
    on = false;
    for (int w = 0; path && w < s.mask_words; ++w) {
      uint64_t m = s.mask[(int64_t)(base + leaf) * s.mask_words + w];
      const int n = min(max(rows - 64 * w, 0), 64);
      m = n == 0 ? 0 : m & (~0ull >> (64 - n));
      count += __popcll(m);
      if (w < tid >> 6) rank += __popcll(m);
      if (w == tid >> 6) { rank += __popcll(m & ((1ull << (tid & 63)) - 1)); on = m >> (tid & 63) & 1; }
    }
  }
  has_slot[tid] = slotted;
  if (tid == 0) moved_from = path_end = count;
  __syncthreads();
  if (on) {
    // The path ends at its first token that was not stored, or for which there is no place.
    if (!stored || !has_slot[rank]) atomicMin(&path_end, rank);
    if (by_mask) {
      // (page id, row) of a key as a row of a page-and-head grid; -1 where there is none
      auto place = [&](int64_t key) -> int64_t {
        const int64_t at = key >> log_page;
        const int id = at < s.max_pages ? s.table[(int64_t)r * s.max_pages + at] : -1;
        return id >= 0 && id < s.pages ? (int64_t)id * s.kv_heads * s.page + (key & (s.page - 1)) : -1;
      };
      from[rank] = place(cached + tid);
      to[rank] = place(cached + rank);
      if (from[rank] < 0 || to[rank] < 0) from[rank] = to[rank] = -1;
      if (tid > rank) atomicMin(&moved_from, rank);      // the first that moves; all behind it do
    }
  }
  __syncthreads();
  count = path_end;
  if (blockIdx.y == 0 && tid == 0) s.cached_out[r] = (int32_t)min(cached + count, (int64_t)0x7FFFFFFF);
  if (!by_mask) return;
  const int64_t column = (int64_t)blockIdx.y * 256 + tid;
  if (column >= columns) return;
  const int chunks = s.head_dim / 8;
  const int chunk = (int)(column % chunks);
  const int64_t rest = column / chunks;
  const int h = (int)(rest % s.kv_heads);
  const int64_t which = rest / s.kv_heads;
  const int layer = (int)(which >> 1);
  u32x4* cache = static_cast<u32x4*>(which & 1 ? s.v : s.k) + ((int64_t)layer * s.pages * s.kv_heads + h) * s.page * chunks + chunk;
  for (int a = moved_from; a < count; a += kAhead) {
    u32x4 x[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) x[i] = a + i < count && from[a + i] >= 0 ? cache[from[a + i] * chunks] : u32x4{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (a + i < count && from[a + i] >= 0) cache[to[a + i] * chunks] = x[i];
  }
}

}  // namespace spqr_srv

using namespace spqr_srv;

extern "C" int spqr_cache_plan(const spqr_step_t* s, void* stream) {
  const int rc = check_sizes(s);
  if (rc) return rc;
  if (!s->cached || !s->fresh || !s->held || !s->table || !s->pool || !s->ends || !s->q_start || !s->position || !s->slot ||
      !s->held_out || !s->ends_out || (s->mask_words > 0 && !s->mask))
    return SPQR_ERR_NULL;
  if (!aligned(s->cached, 4) || !aligned(s->fresh, 4) || !aligned(s->held, 4) || !aligned(s->table, 4) || !aligned(s->parent, 4) ||
      !aligned(s->pool, 4) || !aligned(s->ends, 8) || !aligned(s->q_start, 4) || !aligned(s->position, 4) || !aligned(s->slot, 4) ||
      !aligned(s->mask, 8) || !aligned(s->held_out, 4) || !aligned(s->ends_out, 8))
    return SPQR_ERR_ALIGN;
  if (s->held == s->held_out || s->ends == s->ends_out) return SPQR_ERR_PARAM;   // read by all workgroups, written by one
  hipLaunchKernelGGL(plan_kernel, dim3(s->requests), dim3(256), 0, static_cast<hipStream_t>(stream), *s);
  return launched();
}

extern "C" int spqr_cache_store(const spqr_step_t* s, int32_t layer, const spqr_rows_t* x, void* q_out, void* stream) {
  const int rc = check_cache(s);
  if (rc) return rc;
  if (!x) return SPQR_ERR_NULL;
  if (layer < 0 || layer >= s->layers) return SPQR_ERR_PARAM;
  if (x->x_dtype != SPQR_F32 && x->x_dtype != SPQR_F16 && x->x_dtype != SPQR_BF16) return SPQR_ERR_DTYPE;
  if (!x->q || !x->k || !x->v || !q_out || !s->position || !s->slot) return SPQR_ERR_NULL;
  if (s->rotary_dim < 0 || s->rotary_dim > s->head_dim || s->rotary_dim % 2 != 0) return SPQR_ERR_PARAM;
  if (s->rotary_dim > 0 && !s->rotary) return SPQR_ERR_NULL;
  if (s->rotary_dim > 0 && s->rotary_positions < 1) return SPQR_ERR_SHAPE;
  const int64_t q_row = (int64_t)s->heads * s->head_dim, kv_row = (int64_t)s->kv_heads * s->head_dim;
  if (x->q_stride < q_row || x->k_stride < kv_row || x->v_stride < kv_row) return SPQR_ERR_SHAPE;
  const size_t size = x->x_dtype == SPQR_F32 ? 4 : 2;
  if (!aligned(x->q, size) || !aligned(x->k, size) || !aligned(x->v, size) || !aligned(q_out, 16) || !aligned(s->rotary, 4) ||
      !aligned(s->position, 4) || !aligned(s->slot, 4))
    return SPQR_ERR_ALIGN;
  Store a;
  a.x = *x;
  const int64_t layer_bytes = (int64_t)s->pages * s->kv_heads * s->page * s->head_dim * 2;
  a.q_out = q_out;
  a.kc = static_cast<char*>(s->k) + layer * layer_bytes;
  a.vc = static_cast<char*>(s->v) + layer * layer_bytes;
  a.position = s->position; a.slot = s->slot; a.rotary = s->rotary;
  a.heads = s->heads; a.kv_heads = s->kv_heads; a.D = s->head_dim; a.page = s->page; a.slots = s->pages * s->page;
  a.rot = s->rotary_dim; a.positions = s->rotary_positions; a.pairs = s->rotary_pairs != 0;
  const bool wide = aligned(x->q, 16) && aligned(x->k, 16) && aligned(x->v, 16) && x->q_stride * size % 16 == 0 &&
                    x->k_stride * size % 16 == 0 && x->v_stride * size % 16 == 0 && a.rot % (a.pairs ? 8 : 16) == 0;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return s->dtype == SPQR_F16 ? store_from<_Float16>(x->x_dtype, a, s->tokens, wide, st)
                              : store_from<__bf16>(x->x_dtype, a, s->tokens, wide, st);
}

extern "C" int spqr_cache_keep(const spqr_step_t* s, const int32_t* last, void* stream) {
  const int rc = check_cache(s);
  if (rc) return rc;
  if (!s->cached || !s->table || !s->q_start || !s->cached_out || (s->mask_words > 0 && !s->mask)) return SPQR_ERR_NULL;
  if (!aligned(s->cached, 4) || !aligned(s->table, 4) || !aligned(s->q_start, 4) || !aligned(s->cached_out, 4) || !aligned(s->mask, 8) ||
      !aligned(s->slot, 4) || !aligned(s->position, 4) || !aligned(last, 4))
    return SPQR_ERR_ALIGN;
  if (s->cached == s->cached_out) return SPQR_ERR_PARAM;                         // read by all workgroups, written by one
  const bool moves = last != nullptr && s->mask_words > 0;
  const int64_t columns = (int64_t)s->layers * 2 * s->kv_heads * (s->head_dim / 8);
  const int64_t groups = moves ? (columns + 255) / 256 : 1;
  if (groups > 65535) return SPQR_ERR_SHAPE;
  hipLaunchKernelGGL(keep_kernel, dim3(s->requests, (unsigned)groups), dim3(256), 0, static_cast<hipStream_t>(stream), *s, last, columns);
  return launched();
}
