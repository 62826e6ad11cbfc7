/*
 * spqr_serve.h - C ABI of what stands between the products of a decoder block when sequences are decoded over a
 * paged cache, for AMD MI355X (gfx950): one new token a request, or several drafted ones (a chain or a tree) that
 * one pass over the weights verifies together (spqr.h: a batch of 16 reads the weights once).
 *
 * A step serves `requests` requests.  Request r has cached[r] tokens in the cache and brings fresh[r] new ones
 * (0 .. SPQR_MAX_FRESH, what is above is left out); their rows are q_start[r] .. q_start[r+1] of the step's rows, the
 * rows of every [tokens][...] array here.  Token key j of request r (cached ones first, new ones behind them) lies in
 * page table[r][j / page] at row j % page of the cache:
 *
 *       k, v: [layers][pages][kv_heads][page][head_dim]      16 bits each, 16-byte aligned
 *
 *   spqr_cache_plan       once a step: pages for the new tokens (and back from ended requests), where each new
 *                         token goes, its position, its ancestors in the tree of drafts
 *   spqr_cache_store      a layer: rotary embedding of q and k, k and v to their slots
 *   spqr_tree_attention   a layer: softmax attention of the step's rows over cached and new tokens
 *   spqr_cache_keep       once a step, after verification: the accepted path's rows move together in all layers,
 *                         the lengths grow
 *
 * One descriptor holds the sizes and the device arrays of a step; its arrays stay where they are from step to step, so a
 * step can be captured in a HIP graph (kernel nodes only).  What a call reads and what it writes are different arrays
 * (cached / cached_out, held / held_out, ends / ends_out): the next step's descriptor has them the other way round.
 *
 * Pointers are DEVICE pointers, 4-byte aligned (mask, ends: 8) unless stated otherwise.  All calls are asynchronous on the
 * given HIP stream (hipStream_t as void*, NULL = default stream), allocate nothing, free nothing and never
 * synchronise.  They return SPQR_OK or a negative spqr_status (spqr.h).  Values of the arrays are not trusted with the
 * card: lengths are cut to what the table and the step's rows hold, page ids and slots outside the cache are as
 * pages that are not there.
 */
#ifndef SPQR_SERVE_H_
#define SPQR_SERVE_H_

#include <stddef.h>
#include <stdint.h>

#include "spqr.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SPQR_BF16 2              /* a third element type beside SPQR_F32 and SPQR_F16: bfloat16 */
#define SPQR_MAX_REQUESTS 1024
#define SPQR_MAX_FRESH    256    /* new tokens of a request in one step */

typedef struct spqr_step_t {
  int32_t requests;              /* 1 .. SPQR_MAX_REQUESTS                                                            */
  int32_t tokens;                /* rows of the step, >= 1: what the arrays hold; rows behind q_start[requests] are unused */
  int32_t max_fresh;             /* a hint for the launch plan only: the most new tokens of a request, 0 = unknown      */
  int32_t max_pages;             /* columns of table, >= 1                                                            */
  int32_t mask_words;            /* 64-bit words of a row's mask, 1 .. 4; 0: no masks, new tokens see those before them */
  int32_t dtype;                 /* SPQR_F16 or SPQR_BF16: k, v, and q and out of the attention                        */
  int32_t heads, kv_heads;       /* query heads, a multiple of kv_heads, <= 1024; h reads kv head h / (heads / kv_heads) */
  int32_t head_dim;              /* 64, 96, 128 or 256                                                                */
  int32_t page;                  /* rows of a page: 16, 32, 64, 128 or 256                                            */
  int32_t pages, layers;         /* pages * page < 2^31                                                               */
  int32_t rotary_dim;            /* leading elements of a head that are rotated, even, <= head_dim; 0: none           */
  int32_t rotary_positions;      /* rows of `rotary`                                                                  */
  int32_t rotary_pairs;          /* 0: element i turns with i + rotary_dim / 2; 1: element 2i with 2i + 1              */
  float scale;                   /* of the scores, finite, and times log2(e) too; 0: all keys that a row sees count the same  */
  void* k;
  void* v;
  const int32_t* cached;         /* [requests]                                                                        */
  const int32_t* fresh;          /* [requests], spqr_cache_plan only                                                  */
  const int32_t* held;           /* [requests] pages that table holds for a request                                   */
  int32_t* table;                /* [requests][max_pages] page ids                                                    */
  const int32_t* parent;         /* [tokens] in-request index of the token's parent, smaller than its own; -1 (or
                                    anything else): a root.  NULL: every token follows the one before it              */
  int32_t* pool;                 /* [pages] ring of free page ids                                                     */
  const int64_t* ends;           /* [2] pages taken from and given to the ring so far: pool[i % pages] is free for
                                    ends[0] <= i < ends[1]                                                            */
  int32_t* q_start;              /* [requests + 1]                                                                    */
  int32_t* position;             /* [tokens] -1: unused row                                                           */
  int32_t* slot;                 /* [tokens] page id * page + row; -1: nowhere                                         */
  uint64_t* mask;                /* [tokens][mask_words] bit j: the row sees the j-th new token of its request        */
  int32_t* held_out;             /* [requests]                                                                        */
  int64_t* ends_out;             /* [3]: the ring's ends, pages that were lacking                                     */
  int32_t* cached_out;           /* [requests]                                                                        */
  const float* rotary;           /* [rotary_positions][rotary_dim]: cosines, then sines                               */
  void* workspace;               /* scratch of spqr_tree_attention, 256-byte aligned: written by its kernels, calls that may
                                    overlap need their own                                                            */
  int64_t workspace_bytes;
} spqr_step_t;

/* Rows that a step's products gave: q [tokens][heads][head_dim], k and v [tokens][kv_heads][head_dim], a row
 * contiguous, rows q_stride, k_stride, v_stride elements apart (the three may be parts of one tensor), all of x_dtype
 * (SPQR_F32, SPQR_F16, SPQR_BF16). */
typedef struct spqr_rows_t {
  const void *q, *k, *v;
  int64_t q_stride, k_stride, v_stride;
  int32_t x_dtype;
} spqr_rows_t;

/* Reads cached, fresh, held, ends, parent; writes table, pool, q_start, position, slot, mask, held_out, ends_out.
 *   Pages.  Request r needs min(ceil((cached + fresh) / page), max_pages).  Where it holds fewer it takes the rest from
 *   the ring, in request order, then page order; where it holds more it gives the last ones back in the same order (an
 *   ended request has cached = fresh = 0).  Pages given back in this call are not taken in it.  A page that the ring does
 *   not have is -1 in table and is not held; ends_out[2] counts these and what max_pages cuts off.  Entries of table
 *   that are no longer held keep their values.  held_out, ends_out: the state after the call.
 *   Rows.  q_start = prefix sums of fresh, cut to `tokens`.  The i-th new token of r is key cached + i: slot, or -1 where
 *   its page is missing.  Its mask has its own bit and its ancestors' (all of 0 .. i without parent), as many as
 *   mask_words hold; its position is cached + the number of its ancestors.  Unused rows: position = slot = -1, mask 0.
 * Integers only: same inputs, same outputs; a call may be repeated. */
int spqr_cache_plan(const spqr_step_t* s, void* stream);

/* For every row t with 0 <= position[t] (< rotary_positions where there is a rotation): q_out[t] = q[t] turned by its
 * position, in the cache's type; k[t] turned and v[t] go to slot[t] of `layer` (nowhere if the slot is not in the
 * cache).  Turning (a, b) by position p: (a c - b s, b c + a s), c = rotary[p][i], s = rotary[p][rotary_dim / 2 + i],
 * in binary32, rounded once to the cache's type.  Other rows: q_out[t] = 0, nothing stored.  (Rows whose mask has such a
 * token see what its place held before, if its page is there: what the attention gives for rows with a position behind
 * the end of `rotary` means nothing.)
 * `x` is read during the call (a HOST structure); its rows are aligned to their type (where all addresses are multiples of
 * 16 bytes they are read faster).  q_out [tokens][heads][head_dim], 16-byte aligned, overlaps none of them.  Two rows
 * with one slot: undefined which stays. */
int spqr_cache_store(const spqr_step_t* s, int32_t layer, const spqr_rows_t* x, void* q_out, void* stream);

/* Bytes of device scratch that spqr_tree_attention needs for a step of these sizes; or a negative status.  Host
 * arithmetic only. */
int64_t spqr_tree_attention_workspace_bytes(const spqr_step_t* s);

/* out[t][h] = sum_j p_j v_j, p = softmax over the keys j that row t sees of scale * q[t][h] . k_j: all cached tokens of its
 * request, and the new ones whose bit its mask has (without masks: those up to itself).  A key whose page is not
 * there is seen by nobody.  A row that sees nothing gives zeros; keys that a row does not see do not reach it, whatever
 * they hold (infinities and NaN included).  Products in the type's matrix instructions, sums, maxima and exponentials in
 * binary32, probabilities rounded to the type before they meet v, one rounding at the end.  Deterministic.
 * Reads cached, table, q_start, mask, layer `layer` of k and v, and q [tokens][heads][head_dim]; writes the used rows
 * of out (same shape); both of the cache's type, rows q_stride / out_stride elements apart (a multiple of 8),
 * 16-byte aligned. */
int spqr_tree_attention(const spqr_step_t* s, int32_t layer, const void* q, int64_t q_stride, void* out, int64_t out_stride,
                        void* stream);

/* last[r] is the last accepted new token of request r (in-request index; none if it is no row of r): the tokens of its
 * mask are the accepted path (0 .. last[r] without masks; every new token with last = NULL).  The a-th token of the path
 * moves from key cached + its index to key cached + a, k and v, in all layers; cached_out[r] = cached[r] + the
 * path's length.  The path ends before its first token that spqr_cache_store left out (its slot not in the cache; its
 * position below 0 or, where there is a rotation, no row of `rotary`) or for which the cache has no place: lengths cover
 * stored tokens only, also where pages were lacking.  Reads cached, table, q_start, mask, slot, position (NULL for one of
 * these two: not looked at); pages stay as spqr_cache_plan laid them (the next plan gives back what is no longer needed). */
int spqr_cache_keep(const spqr_step_t* s, const int32_t* last, void* stream);

#ifdef __cplusplus
}
#endif
#endif  /* SPQR_SERVE_H_ */
