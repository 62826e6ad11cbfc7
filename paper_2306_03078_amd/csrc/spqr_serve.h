// A step's descriptor as the kernels take it, shared by spqr_serve.hip and the attention.
#ifndef SPQR_SERVE_INTERNAL_H_
#define SPQR_SERVE_INTERNAL_H_
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/spqr_serve.h"

namespace spqr_srv {

inline bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

// The sizes that every call shares.
inline int check_sizes(const spqr_step_t* s) {
  if (!s) return SPQR_ERR_NULL;
  if (s->requests < 1 || s->requests > SPQR_MAX_REQUESTS || s->tokens < 1 || s->max_pages < 1) return SPQR_ERR_SHAPE;
  if (s->mask_words < 0 || s->mask_words > SPQR_MAX_FRESH / 64 || s->max_fresh < 0 || s->max_fresh > SPQR_MAX_FRESH) return SPQR_ERR_PARAM;
  if (s->page < 16 || s->page > 256 || (s->page & (s->page - 1)) != 0) return SPQR_ERR_PARAM;
  if (s->pages < 1 || (int64_t)s->pages * s->page > 0x7FFFFFFFll) return SPQR_ERR_SHAPE;
  return SPQR_OK;
}

// ... and those of the calls that touch the cache, with its arrays.
inline int check_cache(const spqr_step_t* s) {
  const int rc = check_sizes(s);
  if (rc) return rc;
  if (s->dtype != SPQR_F16 && s->dtype != SPQR_BF16) return SPQR_ERR_DTYPE;
  if (s->head_dim != 64 && s->head_dim != 96 && s->head_dim != 128 && s->head_dim != 256) return SPQR_ERR_PARAM;
  if (s->kv_heads < 1 || s->heads < 1 || s->heads > 1024 || s->heads % s->kv_heads != 0 || s->layers < 1) return SPQR_ERR_SHAPE;
  if (!s->k || !s->v) return SPQR_ERR_NULL;
  if (!aligned(s->k, 16) || !aligned(s->v, 16)) return SPQR_ERR_ALIGN;
  return SPQR_OK;
}

inline int launched() { return hipGetLastError() == hipSuccess ? SPQR_OK : SPQR_ERR_HIP; }

}  // namespace spqr_srv
#endif
