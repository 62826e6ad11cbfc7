// Softmax attention of a step's rows over a paged cache: checks and launch plan (kernels: spqr_attention.h).
#include "spqr_attention.h"

namespace spqr_srv {

#define SPQR_ATTEND_EXTERN(D)                                                                        \
  extern template hipError_t launch_attend<_Float16, D>(const Attend&, const AttendPlan&, hipStream_t); \
  extern template hipError_t launch_attend<__bf16, D>(const Attend&, const AttendPlan&, hipStream_t);
SPQR_ATTEND_EXTERN(64)
SPQR_ATTEND_EXTERN(96)
SPQR_ATTEND_EXTERN(128)
SPQR_ATTEND_EXTERN(256)

// Short prefixes: up to here a second launch takes longer than a chunk's tiles one after the other.  64 requests of up to 600 keys, 8
// key heads of 64 elements: 13.8 us in one launch, 19.9 us cut and joined; equal at about 600 keys where the chunks are few.
constexpr int kWholeTiles = 20;
// From these bytes of keys and values on, 256 rows a chunk where a request has more than 64.  Fewer bytes come out of the L2s time and
// again, and smaller parts fill the card better: 4096 rows over 8000 keys of one head (4 MB) 42 us in chunks of 64, 61 us in chunks
// of 256, over 32000 keys 108 and 123 us; out of the HBM, up to 512 rows, 4 requests of up to 32000 keys, 8 heads (210 MB),
// 190 and 132 us.
// Counted twice: what the requests may read one after another, and what the cache has, which may be less (tables as wide as a pool
// that many share).  With chunks of 64 in plenty the latter says less, as a workgroup takes several of them one after the other: half
// of it is enough at 256 of them, any of it above, where a small pool loses less than many small chunks.  In chunks of 64 and 256,
// tables as wide as the pool: 64 requests of 128 rows over 2 MB 25 and 32 us; 2 of 512 rows, 8 heads, 60 MB 62 and 75 us; 4 of them,
// 28 MB 45 and 49 us, 60 MB 80 and 69 us; 8 of them, 16 MB 38 and 44 us, 60 MB 95 and 72 us; 32 of 80 rows, 14 MB 24 and 19 us,
// 60 MB 36 and 28 us.
constexpr int64_t kFromMemory = 64 << 20;

// Rows of a chunk: as few as hold the rows of a request's key head, so that keys and values are read once for them (4 rows: 26.8 us
// in chunks of 16, 28.1 of 32, 30.2 of 64; 16 rows 28.6, 28.8, 31.4 us; 32 rows 30.0 us in 32, 33.0 in 64; 16 requests of up to 4000
// keys, 8 heads of 128).  The hint only chooses; any rows are right with any chunks.
static AttendPlan plan_attend(const spqr_step_t* s, Attend* a) {
  AttendPlan p;
  const int64_t rows = (int64_t)(s->max_fresh > 0 ? s->max_fresh : SPQR_MAX_FRESH) * (s->heads / s->kv_heads);
  const int most = s->head_dim == 256 ? 32 : 64;           // rows that one wavefront has registers for
  const int64_t page_bytes = 4ll * s->kv_heads * s->head_dim * s->page, read = s->requests * page_bytes * min(s->max_pages, s->pages);
  const int64_t there = page_bytes * min((int64_t)s->requests * s->max_pages, (int64_t)s->pages);
  const int64_t small = (int64_t)s->requests * s->kv_heads * ((rows + most - 1) / most);        // chunks of `most` rows
  const bool from_memory = read >= kFromMemory && (small > 256 || there >= kFromMemory * 128 / max(small, (int64_t)128));
  a->chunk_rows = rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= most || !from_memory ? most : 4 * most;
  // What a (key head, chunk) costs beside its tiles, in tiles.  Measured with 4 / 8 / 16 / 24 (16 rows: 52 heads of 16 requests of up
  // to 8192 keys 238 / 222 / 226 / 229 us, 32 heads of 64 elements, 64 requests of up to 1500 76 / 67 / 70 / 74 us); with
  // 8 / 16 / 24 (32 rows: 45.5 / 42.4 / 45.1 us).
  a->start = a->chunk_rows == 16 ? 8 : 16;
  // With 16 rows as many as run at once: two or (D = 64; 64 requests of up to 1500 keys, 32 heads: 76 us, two 84 us) three of four
  // wavefronts a CU.  Else and with D = 256 one a CU: registers leave room for no more, but for chunks of 32 rows with D = 64, two of which
  // would fit (not measured).
  p.workgroups = a->chunk_rows > 16 || s->head_dim == 256 ? 256 : s->head_dim == 64 ? 768 : 512;
  a->whole = (int64_t)s->max_pages * s->page <= kWholeTiles * kTile;
  const int64_t live = min(rows, (int64_t)a->chunk_rows);
  const int64_t chunks = (int64_t)s->requests * s->kv_heads * ((rows + a->chunk_rows - 1) / a->chunk_rows);
  // Chunks of many parts: workgroups for chunks, whose wavefronts share the parts (2 requests of up to 60000 keys of one head, 256
  // parts: 43 us, workgroups for cuts 108 us; 4 requests of up to 16000 keys, 8 heads, 16 parts: 29 against 37 us; 8 parts: equal;
  // 8 requests of up to 8000 keys, 8 heads of 64, chunks of 256 rows in 2 parts: 75 against 49 us).
  p.by_chunk = chunks * 16 <= p.workgroups;
  p.join_x = p.by_chunk ? (int)chunks : p.workgroups;
  p.join_y = (int)((live + (p.by_chunk ? 3 : 15)) / (p.by_chunk ? 4 : 16));
  return p;
}

static int64_t workspace_bytes(const AttendPlan& p, int chunk_rows, int D) {
  return (int64_t)p.workgroups * sizeof(Join) + 2ll * p.workgroups * chunk_rows * (D + 2) * 4;
}

template <typename T>
static hipError_t launch(int D, const Attend& a, const AttendPlan& p, hipStream_t st) {
  switch (D) {
    case 64: return launch_attend<T, 64>(a, p, st);
    case 96: return launch_attend<T, 96>(a, p, st);
    case 128: return launch_attend<T, 128>(a, p, st);
    default: return launch_attend<T, 256>(a, p, st);
  }
}

}  // namespace spqr_srv

using namespace spqr_srv;

extern "C" int64_t spqr_tree_attention_workspace_bytes(const spqr_step_t* s) {
  const int rc = check_cache(s);
  if (rc) return rc;
  Attend a;
  const AttendPlan p = plan_attend(s, &a);
  return workspace_bytes(p, a.chunk_rows, s->head_dim);
}

extern "C" int spqr_tree_attention(const spqr_step_t* s, int32_t layer, const void* q, int64_t q_stride, void* out, int64_t out_stride,
                                   void* stream) {
  const int rc = check_cache(s);
  if (rc) return rc;
  if (layer < 0 || layer >= s->layers) return SPQR_ERR_PARAM;
  if (!q || !out || !s->cached || !s->table || !s->q_start || (s->mask_words > 0 && !s->mask) || !s->workspace) return SPQR_ERR_NULL;
  const float scale2 = std::fabs(s->scale) * 1.4426950408889634f;
  if (!std::isfinite(scale2)) return SPQR_ERR_PARAM;
  const int64_t row = (int64_t)s->heads * s->head_dim;
  if (q_stride < row || out_stride < row) return SPQR_ERR_SHAPE;
  if (!aligned(q, 16) || !aligned(out, 16) || q_stride % 8 != 0 || out_stride % 8 != 0 || !aligned(s->cached, 4) || !aligned(s->table, 4) ||
      !aligned(s->q_start, 4) || !aligned(s->mask, 8) || !aligned(s->workspace, 256))
    return SPQR_ERR_ALIGN;
  Attend a;
  const AttendPlan p = plan_attend(s, &a);
  if (s->workspace_bytes < workspace_bytes(p, a.chunk_rows, s->head_dim)) return SPQR_ERR_WORKSPACE;
  const int64_t layer_bytes = (int64_t)s->pages * s->kv_heads * s->page * s->head_dim * 2;
  a.q = q; a.out = out; a.q_stride = q_stride; a.out_stride = out_stride;
  a.k = static_cast<const char*>(s->k) + layer * layer_bytes;
  a.v = static_cast<const char*>(s->v) + layer * layer_bytes;
  a.cached = s->cached; a.table = s->table; a.q_start = s->q_start; a.mask = s->mask;
  a.joins = static_cast<Join*>(s->workspace);
  a.part_o = reinterpret_cast<float*>(a.joins + p.workgroups);
  a.part_ml = a.part_o + 2ll * p.workgroups * a.chunk_rows * s->head_dim;
  a.requests = s->requests; a.tokens = s->tokens; a.kv_heads = s->kv_heads; a.group = s->heads / s->kv_heads;
  a.log_page = __builtin_ctz(s->page); a.pages = s->pages; a.max_pages = s->max_pages; a.words = s->mask_words;
  a.scale2 = scale2;
  a.turn = s->scale < 0.f ? 0x80008000u : 0u;
  a.inv_group = 1.0f / (float)a.group;
  a.workgroups = p.workgroups;
  a.inv_workgroups = 1.0 / p.workgroups;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const hipError_t e = s->dtype == SPQR_F16 ? launch<_Float16>(s->head_dim, a, p, st) : launch<__bf16>(s->head_dim, a, p, st);
  return e == hipSuccess ? SPQR_OK : SPQR_ERR_HIP;
}
