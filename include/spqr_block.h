/*
 * spqr_block.h - C ABI of what a decoder's step does beside its products (spqr.h) and its attention (spqr_serve.h), for
 * AMD MI355X (gfx950):
 *
 *   spqr_residual_norm     norms before and after a block, with its gate and the residual sum, in one pass over the rows
 *   spqr_adapter_plan      once a step: the step's rows by low-rank adapter
 *   spqr_adapters          a layer: low-rank adapters of many requests, added to the projections that share their input
 *   spqr_token_logprobs    behind the head: log probabilities of given tokens, entropy, most probable tokens
 *
 * A row is one token of a step (or of a text that is scored).  Element types are SPQR_F32, SPQR_F16 and SPQR_BF16; rows
 * are contiguous, `stride` elements apart, and may begin at any address that their type may have (16-byte aligned rows are
 * read and written fastest).  Statistics, sums and products are held in binary32 or more, results rounded once.
 *
 * Pointers are DEVICE pointers.  All calls are asynchronous on the given HIP stream (hipStream_t as void*, NULL = default
 * stream), allocate nothing, free nothing and never synchronise; captured in a HIP graph they are kernel nodes only.  They
 * return SPQR_OK or a negative spqr_status (spqr.h).  Results are deterministic.  A call of no rows does nothing.
 */
#ifndef SPQR_BLOCK_H_
#define SPQR_BLOCK_H_

#include <stddef.h>
#include <stdint.h>

#include "spqr_serve.h"          /* SPQR_BF16, SPQR_MAX_REQUESTS */

#ifdef __cplusplus
extern "C" {
#endif

/* ---- norms, gate, residual sum -------------------------------------------- */

#define SPQR_MAX_WIDTH  65536

#define SPQR_NORM_NONE  0        /* v                                                                  */
#define SPQR_NORM_RMS   1        /* v / sqrt(mean(v^2) + eps) * (weight_offset + weight) + bias           */
#define SPQR_NORM_LAYER 2        /* (v - mean) / sqrt(var + eps) * (weight_offset + weight) + bias        */

#define SPQR_ACT_NONE    0       /* g                */
#define SPQR_ACT_SILU    1       /* g / (1 + e^-g)   */
#define SPQR_ACT_SIGMOID 2       /* 1 / (1 + e^-g)   */
#define SPQR_ACT_TANH    3

/* One row:  s = skip * x + scale * act(gate) * norm_y(y),  sum = s,  out = norm_x(s). */
typedef struct spqr_residual_norm_t {
  int32_t rows, width;           /* rows >= 0; 1 <= width <= SPQR_MAX_WIDTH                                             */
  int32_t x_dtype;               /* of x and sum                                                                        */
  int32_t y_dtype, gate_dtype, out_dtype;
  int32_t weight_dtype;          /* of the four vectors below                                                           */
  int32_t norm_y, norm_x;        /* SPQR_NORM_*                                                                         */
  int32_t act;                   /* SPQR_ACT_*, of the gate                                                             */
  float eps;                     /* > 0, finite                                                                         */
  float weight_offset;           /* added to weights that are given (a weight that is NULL is 1, a bias 0)              */
  float skip, scale;             /* finite                                                                              */
  const void *x, *y, *gate;      /* [rows][width]; NULL: no such term (gate: 1).  x or y at least                       */
  void *sum, *out;               /* [rows][width]; NULL: not written.  One at least                                     */
  int64_t x_stride, y_stride, sum_stride, out_stride;   /* elements between rows, >= width                              */
  int64_t gate_stride;           /* the same, or 0: one gate for all rows                                               */
  const void *y_weight, *y_bias, *x_weight, *x_bias;    /* [width]                                                       */
} spqr_residual_norm_t;

/* Statistics are of the binary32 values of s before they are rounded to sum; a row's sum of squares must not pass binary32
 * (it does not where the largest magnitude times sqrt(width) is below 1.8e19: 1.9e17 at a width of 8192, 7e16 at 65536).
 * A row with an infinity or NaN gives NaN in that row only.  sum may be x (same address and stride); sum and out overlap
 * nothing else that is read or written. */
int spqr_residual_norm(const spqr_residual_norm_t* p, void* stream);

/* ---- low-rank adapters of many requests ------------------------------------- */

#define SPQR_ADAPTER_TILE 64     /* rows of a tile                                    */
#define SPQR_MAX_SLOTS    4096
#define SPQR_MAX_RANK     256
#define SPQR_MAX_ROWS     (1 << 20)

/* The rows of a step by adapter.  A bank has `slots` places for adapters; request r uses the one in slot adapter[r] (none
 * if that is not in [0, slots)) for its rows q_start[r] .. q_start[r + 1] (spqr_serve.h: spqr_cache_plan writes q_start).
 * q_start NULL: adapter has one entry for each row. */
typedef struct spqr_adapter_plan_t {
  int32_t rows;                  /* 0 .. SPQR_MAX_ROWS: the step's rows                                                 */
  int32_t slots;                 /* 1 .. SPQR_MAX_SLOTS                                                                 */
  int32_t requests;              /* entries of adapter, 0 .. SPQR_MAX_REQUESTS; without q_start: = rows                 */
  int32_t max_tiles;             /* of tile and row; spqr_adapter_tiles(rows, slots) or more                            */
  const int32_t* adapter;        /* [requests]; NULL with requests 0: every row is in no tile                           */
  const int32_t* q_start;        /* [requests + 1], ascending, or NULL                                                  */
  int32_t* count;                /* [1] tiles in use                                                                    */
  int32_t* tile;                 /* [max_tiles][2] slot (-1: rows of no adapter), rows; -1, 0 behind the last           */
  int32_t* row;                  /* [max_tiles][SPQR_ADAPTER_TILE] the tile's rows, -1 behind the last                  */
} spqr_adapter_plan_t;

/* The most tiles that a step of these sizes can have, or a negative status.  Host arithmetic only. */
int32_t spqr_adapter_tiles(int32_t rows, int32_t slots);

/* Reads adapter and q_start (bounds outside the step's rows are cut to them); writes count, tile and row: the rows of every
 * slot in ascending order, slot after slot, then those of no adapter; a new tile for every slot and every
 * SPQR_ADAPTER_TILE rows.  Rows of no request (behind q_start[requests]) are in no tile. */
int spqr_adapter_plan(const spqr_adapter_plan_t* p, void* stream);

/* out_p[t] = y_p[t] + scale_p[a] * B_p[a] (A_p[a] x[t])  for the `count` projections p that share x, a the slot of row t's tile;
 * out_p[t] = y_p[t] for rows of no adapter; rows in no tile are not written. */
typedef struct spqr_adapters_t {
  int32_t count;                 /* 1 .. SPQR_MAX_FUSED                                                                 */
  int32_t width;                 /* elements of a row of x, 1 .. SPQR_MAX_WIDTH                                         */
  int32_t slots;                 /* 1 .. SPQR_MAX_SLOTS; the plan's                                                     */
  int32_t dtype;                 /* SPQR_F16 or SPQR_BF16: x, A, B                                                      */
  int32_t y_dtype;               /* of y and out                                                                        */
  int32_t m[SPQR_MAX_FUSED];     /* rows of B: elements of a row of y, 1 .. SPQR_MAX_WIDTH                              */
  int32_t max_rank[SPQR_MAX_FUSED];      /* 1 .. SPQR_MAX_RANK                                                          */
  const void* bank[SPQR_MAX_FUSED];      /* spqr_adapters_bank_bytes(a, p) bytes, 256-byte aligned, filled by spqr_adapters_pack   */
  const float* scale[SPQR_MAX_FUSED];    /* [slots]; NULL: 1                                                             */
  const void* y[SPQR_MAX_FUSED];         /* [rows][m]; NULL: zero                                                       */
  void* out[SPQR_MAX_FUSED];             /* [rows][m]; may be y (same address and stride), overlaps nothing else        */
  int64_t y_stride[SPQR_MAX_FUSED], out_stride[SPQR_MAX_FUSED];    /* elements between rows, >= m                       */
  const void* x;                         /* [rows][width]                                                               */
  int64_t x_stride;
  void* workspace;                       /* scratch, 256-byte aligned: written by the call's kernels; calls that may overlap
                                            need their own                                                              */
  int64_t workspace_bytes;
} spqr_adapters_t;

/* Bytes of projection p's bank (by count, width, slots, m and max_rank), or a negative status.  Host arithmetic only.  A bank holds its
 * adapters' weights in the order that the kernels read them, ranks rounded up to 16 (A) and 32 (B, above 16), widths to 128, m to 64. */
int64_t spqr_adapters_bank_bytes(const spqr_adapters_t* a, int32_t p);

/* Fills `slots` slots of projection p's bank, from slot `first` on, with the adapters A [slots][max_rank][width], B [slots][m][max_rank]
 * of type a->dtype and rank [slots] (0 .. max_rank, cut to that; NULL: max_rank): what lies behind an adapter's rank in A and B does not
 * count, whatever it holds.  Of `a` the sizes, dtype and bank[p] are looked at; A, B and rank may go after the call has run.  Slots
 * that were never filled must not be used by a plan (their ranks are what the memory held: clear it, and they add nothing). */
int spqr_adapters_pack(const spqr_adapters_t* a, int32_t p, int32_t first, int32_t slots, const void* A, const void* B, const int32_t* rank,
                       void* stream);

/* Bytes of scratch that spqr_adapters needs for steps of up to `rows` rows, by count, width, slots and max_rank of the descriptor (no
 * pointers are looked at); or a negative status.  Host arithmetic only. */
int64_t spqr_adapters_workspace_bytes(const spqr_adapters_t* a, int32_t rows);

/* A step's rows through the adapters.  `plan` is one that spqr_adapter_plan filled (earlier on the same stream, or otherwise
 * before it) with the same slots; of its arrays count, tile and row are read.  Sums in binary32; A x meets B as a sum of two
 * (SPQR_F16) or three (SPQR_BF16) values of `dtype`, which hold it to 2^-22 of a row's largest element or better.  An infinity or
 * NaN in a row of x gives infinities or NaN in that row. */
int spqr_adapters(const spqr_adapters_t* a, const spqr_adapter_plan_t* plan, void* stream);

/* ---- log probabilities --------------------------------------------------------- */

#define SPQR_MAX_TOP   64
#define SPQR_MAX_GIVEN 64

/* Of a row of logits l: z = scale * l, lse = log(sum_j e^z_j), p = e^(z - lse). */
typedef struct spqr_token_logprobs_t {
  int32_t rows, vocab;           /* rows >= 0; 1 <= vocab < 2^24                                                        */
  int32_t dtype;                 /* of the logits                                                                       */
  int32_t given;                 /* tokens given for each row, 0 .. SPQR_MAX_GIVEN                                      */
  int32_t top;                   /* 0 .. SPQR_MAX_TOP                                                                   */
  float scale;                   /* one over the temperature, > 0, finite                                               */
  const void* logits;            /* [rows][vocab]                                                                       */
  int64_t stride;                /* elements between rows, >= vocab                                                     */
  const int32_t* tokens;         /* [rows][given]                                                                       */
  float* logprob;                /* [rows][given] z[token] - lse; 0 for a token that is not in [0, vocab): sums over a text
                                    leave it out                                                                        */
  float* entropy;                /* [rows] -sum_j p_j log p_j, in nats; NULL: not written                               */
  int32_t* top_token;            /* [rows][top] the most probable tokens, the lowest id first among equal logits; -1 where
                                    fewer than `top` have a logit above -infinity                                       */
  float* top_logprob;            /* [rows][top] their log probabilities; -infinity where there is none                  */
  void* workspace;               /* scratch, 256-byte aligned: written by the call's kernels; calls that may overlap need their own */
  int64_t workspace_bytes;
} spqr_token_logprobs_t;

/* Bytes of scratch that spqr_token_logprobs needs (rows, vocab and top count; no pointers are looked at; fewer rows never need
 * more than the most that any number of rows up to p->rows does); or a negative status.  Host arithmetic only. */
int64_t spqr_token_logprobs_workspace_bytes(const spqr_token_logprobs_t* p);

/* Logits of -infinity are tokens of probability 0 (log probability -infinity, nothing in the entropy); a row that has only
 * such: entropy 0.  The type's lowest finite value is a logit like others.  A row with a NaN or +infinity: its logprob (of tokens in
 * [0, vocab)), entropy and all of its top_logprob are NaN; its top_token are by value, NaN left out, -1 behind the last. */
int spqr_token_logprobs(const spqr_token_logprobs_t* p, void* stream);

#ifdef __cplusplus
}
#endif
#endif  /* SPQR_BLOCK_H_ */
