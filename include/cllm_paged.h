/*
 * cllm_paged.h -- a paged key/value cache for blocks of new tokens: block tables
 * and slot maps built on the GPU, the write of a step's keys and values with the
 * rotary embedding, and the attention of the step's tokens over the pages.
 *
 * The engine of cllm.h keeps one run of max_seq positions per sequence.  A
 * program whose requests come and go keeps pages instead: page_size positions
 * each, handed to a request as it grows and taken back when it ends.  One step
 * over a batch of B requests, request b with ctx[b] cached tokens and new_rows[b]
 * new ones (a Jacobi block of n, a chunk of a prompt, or 1 for greedy decoding):
 *
 *   cllm_page_plan         pages for every request, and where each new row goes
 *   per layer: cllm_paged_append     K, V of the new rows into their slots
 *              cllm_paged_attention  the new rows over all pages of their request
 *
 * Conventions for the calls of this header (they differ from the engine's, since
 * they are parts of a caller's own step):
 *   - Arrays are DEVICE memory owned by the caller.  Each call queues its work on
 *     cuda_stream (a cudaStream_t, NULL = the legacy default stream) and returns
 *     without waiting; nothing is allocated, so calls can be captured in a graph.
 *   - Calls on a cache use the device that it was created on, whichever is current (NULL is that
 *     device's default stream); cllm_page_plan uses the current device.
 *   - Return value: CLLM_OK or a negative CLLM_E* code for what the host can see;
 *     then nothing is queued and the outputs are left untouched.  What only the
 *     device can see (a page number outside the pool) is kept in the cache's
 *     device status word and returned by cllm_paged_status.
 *   - Lengths (B, ctx, new_rows, row_start, seq_len) that live on the device may
 *     change between replays of a captured step.
 *   - Calls on one cache, or with one pair of tables, must not overlap in time.
 *   - An attention call's results are a function of its inputs, bit for bit; the
 *     same row's last bits may differ between batches, whose work is cut in other places.
 */
#ifndef CLLM_PAGED_H
#define CLLM_PAGED_H

#include <stdint.h>

#include "cllm.h"

#ifdef __cplusplus
extern "C" {
#endif

#define CLLM_F16 2 /* fp16 pools, queries and outputs (paged calls only) */

/* ---- block tables and slot maps ------------------------------------------------- */

/* The pages of up to max_batch requests, and the free ones.  Free pages wait in
 * a ring: state[0] is the index in ring[] of the next page to hand out, state[1]
 * how many there are.  table[b][j], j < held[b], is the page of request b's
 * positions j*page_size ..; other entries are -1. */
typedef struct {
  int32_t *table; /* [max_batch][width] */
  int32_t *held;  /* [max_batch] */
  int32_t *ring;  /* [n_pages] */
  int32_t *state; /* [4]: first, count, 0, 0 (the third is used within a call) */
  int max_batch, width, n_pages, page_size;
} cllm_page_tables;

/* What a plan says about the step's rows, those of request 0 first. */
typedef struct {
  int32_t *row_start; /* [max_batch + 1] first row of each request, then the total (at most 2^31 - 1) */
  int32_t *seq_len;   /* [max_batch] tokens of the request after the step; 0 if refused */
  int32_t *granted;   /* [max_batch] 1, or 0 if refused */
  int64_t *slots;     /* [max_rows] page * page_size + offset; -1: no slot */
  int32_t *positions; /* [max_rows] position in the request; 0 where there is no slot */
  int max_rows;
} cllm_page_rows;

/*
 * Grow or shrink the pages of requests 0..B-1 to ceil((ctx + new_rows) / page_size)
 * and say where each new row goes.  A request that has ended (ctx = new_rows = 0)
 * gives all its pages back.  Requests are served in order: one is refused, and
 * keeps what it holds, when the pages it and the requests before it ask for
 * exceed the free ones; when its length is negative or more than width pages; or
 * when its rows would pass max_rows (row_start counts them all the same, past max_rows too).  Pages given back (in order of request, then of
 * position) can be handed out from the next call on.
 * in, out: the tables before and after; the same tables for an update in place,
 * or another table/held/state over the same ring to see what a step would get
 * before adopting it (the ring's live entries are not changed).  Entries of rows
 * B.. are not touched.  out->state[2] must be 0 before the first call.  rows->seq_len may
 * be ctx or new_rows.
 * Errors: EINVAL (null or misaligned pointers, sizes < 1, B outside [0, max_batch],
 * in and out of different sizes or rings, page_size not a power of two,
 * width * page_size or max_batch * width past 2^31 - 1, max_batch > 4096), ECUDA.
 */
int cllm_page_plan(const cllm_page_tables *in, const cllm_page_tables *out, const cllm_page_rows *rows, int B,
                   const int32_t *ctx, const int32_t *new_rows, void *cuda_stream);

/* ---- the cache ------------------------------------------------------------------- */

/*
 * K and V pools of the caller: element (layer, page, head, pos, d) of either is at
 * layer*stride_layer + page*stride_page + head*stride_head + pos*stride_pos + d
 * (element strides, so pages may hold one head's positions together or one
 * position's heads together, and K and V may share an allocation).
 * Constraints: head_dim 64 or 128; page_size a power of two from 8 to 256;
 * n_heads a multiple of n_kv_heads, at most 64 heads to one; pointers and strides
 * multiples of 16 bytes.
 */
typedef struct {
  void *k, *v;
  int dtype; /* CLLM_F32 | CLLM_BF16 | CLLM_F16: of the pools, new rows, queries and outputs */
  int layers, n_pages, page_size, n_kv_heads, head_dim, n_heads;
  int64_t stride_layer, stride_page, stride_head, stride_pos;
} cllm_paged_desc;

typedef struct cllm_paged cllm_paged;

/* Create a cache over the pools: checks the shape, builds their tensor maps and
 * allocates (owns) the scratch of the attention's split work on the current
 * device: 512 rows of head_dim + 2 floats per SM (40 MB at head_dim 128).  The pools stay the caller's and must outlive the cache.
 * Errors: EINVAL, EUNSUPPORTED (shape outside the constraints, not an sm_103
 * device), ENOMEM, ECUDA. */
int cllm_paged_create(const cllm_paged_desc *desc, cllm_paged **out);

/* Wait for the device, then release what the cache owns.  NULL is a no-op. */
void cllm_paged_destroy(cllm_paged *cache);

/* Wait for the stream and return (and clear) what the calls before found on the
 * device: CLLM_OK, CLLM_EDEVICE (a page or slot outside the pool, a position
 * outside the rotary table: those rows were skipped or read as zeros) or
 * CLLM_ETIMEOUT (a bounded wait ran out; the outputs of that attention call, and of those
 * after it until this one, are not valid). */
int cllm_paged_status(cllm_paged *cache, void *cuda_stream);

/*
 * Write rows of keys and values into their slots (cllm_page_plan's, or any
 * others; -1 skips a row's K and V; two rows with one slot may leave a mix of both, in pieces
 * of 16 bytes).
 * rope: K as it is when NULL (q unused).  With it K and, when q is not NULL, q are
 * rotated (pairs i, i + head_dim/2: the engine's convention) by row positions[t] in
 * fp32 and rounded once; q goes to q_out (which may be q).
 */
typedef struct {
  int layer, rows;
  const void *k, *v;        /* [rows][n_kv_heads][head_dim], heads side by side */
  const void *q;            /* [rows][n_heads][head_dim], heads side by side, or NULL */
  void *q_out;
  int64_t k_stride, v_stride, q_stride, q_out_stride; /* elements between rows */
  const int64_t *slots;     /* [rows] */
  const float *rope;        /* [max_pos][head_dim / 2][2] (cos, sin), or NULL */
  const int32_t *positions; /* [rows] */
  int max_pos;
} cllm_paged_rows;

/* Errors: EINVAL (null or misaligned pointers, strides too small or not multiples of 16
 * bytes, layer outside the pools, rows < 0, q without rope), ECUDA. */
int cllm_paged_append(cllm_paged *cache, const cllm_paged_rows *r, void *cuda_stream);

/*
 * Attention of a step.  Request b's rows are row_start[b] .. row_start[b+1]-1 of
 * q and out; the i-th is its token ctx + i of seq_len[b] = ctx + rows (whose keys
 * and values are in the cache already).  It sees key k when
 *   k < ctx, or among the new tokens k <= ctx + i (mask NULL), or bit k - ctx of
 *   the row's mask words (mask: verification of several candidates at once);
 *   and, with window > 0, (ctx + i) - k < window.  (With a mask too the window goes by the
 *   row's place i in the block, not by its depth in a candidate: a row of the second candidate
 *   sees fewer cached keys than its position's window has.)
 * out = softmax(scale q k) v in the pools' type; a row that sees nothing (its mask
 * is empty, or seq_len[b] < rows, as a plan leaves a refused request) is 0 with lse
 * -inf.  lse[row][head] = log sum exp(scale q k), natural, may be NULL.  What a row
 * does not see never reaches it, infinities and NaN included; a score that it does see and
 * that is NaN or +inf makes the row and its lse NaN.  Rows from
 * row_start[batch] on are not written.  Pages wholly before the window are not read.
 */
typedef struct {
  int layer, batch, rows; /* rows: of q and out, at least row_start[batch]; only requests of
                           * seq_len 0 may have rows past them, which are not written */
  const void *q;
  void *out; /* no element of q or of the pools (a row may be read again after others are written) */
  float *lse;
  int64_t q_stride, q_head_stride, out_stride, out_head_stride; /* elements */
  const int32_t *row_start; /* [batch + 1] */
  const int32_t *seq_len;   /* [batch] at most table_width pages, and at most 2^31 - 8192 */
  const int32_t *table;     /* [batch][table_width] */
  int table_width;
  float scale;
  int window;           /* 0: none */
  const uint32_t *mask; /* [rows][mask_words], or NULL: causal */
  int mask_words;
} cllm_paged_attn;

/* Errors: EINVAL (null or misaligned pointers, out the same as q, strides not multiples of 16 bytes,
 * sizes outside their ranges, scale not positive and finite), EUNSUPPORTED (rows x
 * table_width so large that the work may exceed 2^31 - 1 units of a few rows and 64
 * keys: cut the step), ECUDA. */
int cllm_paged_attention(cllm_paged *cache, const cllm_paged_attn *a, void *cuda_stream);

#ifdef __cplusplus
}
#endif

#endif /* CLLM_PAGED_H */
