/*
 * The operators of a decoder layer, for an executor that runs a placement of
 * the what-if simulation (gmgsim.h) on a GB300 and measures what the
 * estimators (gmgest.h) are fitted on.  They are the nodes of the layer's
 * graph: products (qkv, oproj + add, gateup + silu, down + add), rotary
 * positions (rope) written into a paged cache (kvw), and attention (attn)
 * whose requests share retained state: new instances attach to intermediates
 * that stay resident (Sec. 3.2, checkpoint metadata).
 *
 *   op_free, op_fork, op_grow, op_compact   pages of the cache
 *   op_rope, op_rope_append                 rotary positions, into the cache
 *   op_attend_plan, op_attend               attention over shared prefixes
 *   op_linear                               product with its epilogue
 *
 * All pointers are device pointers unless stated; calls are asynchronous on
 * `stream`, allocate nothing, and return 0 or a negative GMG_E* code
 * (gmgsim.h): GMG_EINVAL for arguments outside what is documented here,
 * GMG_EWS for a short or misaligned buffer, GMG_ECUDA for a failed launch.
 * Strides are in elements; the innermost dimension of a tensor is contiguous
 * and no tensor's elements overlap.  Sums, softmax statistics and angles are
 * held in 32 bits or more and rounded once, to the output's type; op_attend's
 * probabilities are rounded to the values' type before, for their product.
 */
#ifndef GMGOP_H
#define GMGOP_H

#include <stddef.h>
#include <stdint.h>

#include "gmgsim.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types. */
#define GMG_OP_F32 0
#define GMG_OP_BF16 1
#define GMG_OP_F16 2

/* A paged cache of keys and values.  Request row s holds tokens 0 ..
 * lens[s] - 1; token t is slot t % page_tokens of page table[s * max_pages +
 * t / page_tokens].  Entries beyond a request's pages are -1.  refs[p] counts
 * the rows (and any holders of the caller's) that list page p; a page with no
 * reference is free.
 *   pool [n_pages][n_layers][2 (K, V)][n_kv_heads][page_tokens][head_dim],
 *   16-byte aligned; page_tokens is 8, 16, 32, 64, 128 or 256, head_dim a
 *   multiple of 8 up to 128; bf16 or fp16.
 *   status int32[8]: [0] GMG_PAGE_* of the last page call, [1] the first entry of its
 *   lists that has a fault (of equal rows the second; GMG_PAGE_FULL: how many pages are missing), [2]
 *   pages moved (op_compact), [3] pages in use (op_compact), [4] tokens that
 *   op_rope_append had no page for, added up, [5] blocks of op_attend with a wait
 *   that gave up (0 unless the GPU is at fault: their output is not a result), added up. */
typedef struct {
  void* pool;
  int32_t* table;
  int32_t* lens;
  int32_t* refs;
  int32_t* status;
  int32_t dtype, n_pages, n_layers, n_kv_heads, page_tokens, head_dim;
  int32_t n_seq, max_pages;
} op_cache_t;

#define GMG_PAGE_OK 0
#define GMG_PAGE_FULL 1   /* fewer free pages than needed */
#define GMG_PAGE_SEQ 2    /* a request row out of range */
#define GMG_PAGE_TWICE 3  /* a request row listed twice, or forked from and into */
#define GMG_PAGE_LONG 4   /* a length that is negative or beyond max_pages (fork: beyond the source's) */
#define GMG_PAGE_USED 5   /* op_fork: the new row is not empty */

/* Bytes of the scratch of the page calls on this cache (0 on bad arguments).
 * Zero it once; calls that share it must be ordered.  256-byte aligned. */
size_t op_page_scratch_bytes(const op_cache_t* cache);

/* Page calls.  Lists are int32 of n entries (0 <= n <= n_seq).  A call whose
 * lists are not valid, or that needs more free pages than there are, changes
 * nothing but status; the later calls of a stream do not look at it.
 *
 * op_free: drop the rows' references, empty the rows.
 * op_fork: row dst[i], empty, gets the first keep[i] tokens of row src[i] (keep
 *   NULL: all) by reference.
 * op_grow: row seq[i] gets room for add[i] >= 0 more tokens and its length grows
 *   by them.  Where add[i] > 0 and its last page is partly filled and had more
 *   than one reference when the call began, the row takes a copy of that page
 *   first, in all layers (the page loses a reference, and may become free for the
 *   next call).  New pages are the free ones in increasing order, to the entries
 *   in list order (an entry's copy first).
 * op_compact: with L pages in use, the k-th used page at or beyond L moves to the
 *   k-th free page below L (increasing order), with data, references and table
 *   entries. */
int op_free(const op_cache_t* cache, const int32_t* seq, int32_t n, void* scratch, size_t scratch_bytes,
            gmg_stream_t stream);
int op_fork(const op_cache_t* cache, const int32_t* src, const int32_t* dst, const int32_t* keep, int32_t n,
            void* scratch, size_t scratch_bytes, gmg_stream_t stream);
int op_grow(const op_cache_t* cache, const int32_t* seq, const int32_t* add, int32_t n, void* scratch,
            size_t scratch_bytes, gmg_stream_t stream);
int op_compact(const op_cache_t* cache, void* scratch, size_t scratch_bytes, gmg_stream_t stream);

/* Rotary positions: with pairs (u, v) of the first `rotary` elements of a head,
 * the angle a = pos * f_i of pair i and the factor m,
 *   (u, v) -> m (u cos a - v sin a, u sin a + v cos a)
 * (backward: a -> -a, the gradient's way back); the other elements pass.
 * Pairs are (2i, 2i + 1) if interleaved, else (i, i + rotary / 2).
 *   freq [rotary / 2] uint64: f_i / (2 pi) * 2^64, rounded, for 0 <= f_i < 2 pi.
 *   An angle is reduced by the wrap of a 64-bit product, so that its error does not grow
 *   with the position beyond |pos| 2^-65 turns, from the rounding of freq; its top 32 bits
 *   are then rounded to fp32, up to 2^-26 turns (1e-7 radians). */
typedef struct {
  const uint64_t* freq;
  int32_t rotary, interleaved;
  float factor;
} op_rope_t;

/* out[t][h] = x[t][h] rotated by pos[t] (int32); head_dim >= rotary, rotary even, at most 256.
 * out may be x itself (same strides). */
int op_rope(const op_rope_t* rope, int32_t dtype, int64_t n_tokens, int32_t n_heads, int32_t head_dim, const void* x,
            int64_t x_tok, int64_t x_head, const int32_t* pos, int32_t backward, void* out, int64_t out_tok,
            int64_t out_head, gmg_stream_t stream);

/* q_out[t] = q[t] rotated by pos[t]; k[t] rotated and v[t] are written to `layer` of
 * the cache, at token pos[t] of row seq[t].  A token whose row or page does not
 * exist (a negative seq marks padding) is rotated but not written; status[4]
 * counts those with seq >= 0.  The page has to be the row's own, which op_grow
 * sees to: what other rows share would be written too.  n_heads may be 0.  Types are the cache's. */
int op_rope_append(const op_rope_t* rope, const op_cache_t* cache, int32_t layer, int64_t n_tokens, int32_t n_heads,
                   const void* q, int64_t q_tok, int64_t q_head, const void* k, int64_t k_tok, int64_t k_head,
                   const void* v, int64_t v_tok, int64_t v_head, const int32_t* pos, const int32_t* seq, void* q_out,
                   int64_t o_tok, int64_t o_head, gmg_stream_t stream);

/* Attention of a batch of requests over a paged cache.  Request b has
 * q_len[b] queries, the last of its kv_len[b] cached tokens: query i sits at
 * position kv_len[b] - q_len[b] + i and sees the keys at or before it (none, if
 * that is negative: its output is 0, its lse -inf).  Query head h reads
 * key/value head h / (n_heads / n_kv_heads).
 *   o = sum_j softmax_j(scale q . k_j) v_j,   lse = log sum_j exp(scale q . k_j)
 * Requests group_off[g] .. group_off[g + 1] share their first prefix[g] tokens:
 * where that is less work, all their queries are taken together against the
 * pages of the group's first request, each page read once for all of them.
 *
 * A plan (host memory, then copied to the device by the caller) holds the work
 * items for these lengths; one plan serves every layer of a step. */
typedef struct {
  int32_t n_batch, n_heads, n_kv_heads, head_dim, page_tokens;
  int32_t n_groups;           /* 0: no sharing (group_off and prefix not read) */
  const int32_t* q_len;       /* host [n_batch], 0 .. 2^30 */
  const int32_t* kv_len;      /* host [n_batch], 0 .. 2^30 */
  const int32_t* seq;         /* host [n_batch] table rows; NULL: b */
  const int32_t* group_off;   /* host [n_groups + 1], 0 .. n_batch increasing */
  const int32_t* prefix;      /* host [n_groups] >= 0, at most each member's kv_len - q_len */
} op_attend_desc_t;

typedef struct {
  int32_t n_batch, n_heads, n_kv_heads, head_dim, page_tokens;
  int32_t n_items, n_joins;   /* work items (per key/value head); joins of partial results */
  int32_t max_seq, max_kv;    /* what table rows and lengths the plan reaches */
  int32_t join_tokens;        /* queries of the largest join */
  int64_t n_tokens;           /* queries in all */
  int64_t part_rows;          /* rows of partial results per key/value head */
  size_t plan_bytes;          /* of the plan's array */
  size_t work_bytes;          /* of op_attend's workspace */
} op_attend_plan_t;

/* Fills *plan and, if items is not NULL, items[plan->plan_bytes / 4] (host
 * int32, on the device 16-byte aligned; item_bytes is what it holds).  n_sm: SMs to spread the work over. */
int op_attend_plan(const op_attend_desc_t* desc, int32_t n_sm, op_attend_plan_t* plan, int32_t* items,
                   size_t item_bytes);

/* q, out [n_tokens][n_heads][head_dim] (requests one after another; strides
 * multiples of 8 elements, 16-byte aligned; out contiguous heads), lse
 * [n_tokens][n_heads] fp32 or NULL.  d_items: the plan's array on the device;
 * work: 256-byte aligned.  Types are the cache's.  A table entry that is no page of
 * the pool reads as zeros. */
int op_attend(const op_attend_plan_t* plan, const int32_t* d_items, const op_cache_t* cache, int32_t layer,
              const void* q, int64_t q_tok, int64_t q_head, float scale, void* out, int64_t out_tok, int64_t out_head,
              float* lse, void* work, size_t work_bytes, gmg_stream_t stream);

/* y = act(x w^T + bias) + residual, or, with a gate,
 * y = act(x gate^T + gate_bias) * (x w^T + bias) + residual.
 * x [m][k], w and gate [n][k], residual and y [m][n], bias and gate_bias [n], all of
 * one type (bf16 or fp16); biases and residual may be NULL, gate where gated is 0.  Products are
 * summed in fp32.  y may be residual itself (same strides).  m, n, k >= 0. */
#define GMG_OP_NONE 0
#define GMG_OP_RELU 1
#define GMG_OP_SILU 2
#define GMG_OP_GELU 3 /* v/2 (1 + erf(v / sqrt 2)) */

typedef struct {
  int32_t dtype, act, gated, reserved;
  int64_t m, n, k;
  const void *x, *w, *gate, *bias, *gate_bias, *residual;
  void* y;
  int64_t x_row, w_row, gate_row, residual_row, y_row; /* row strides, >= the row's length */
} op_linear_t;

/* Bytes of the workspace (256-byte aligned; its first 4 KB zeroed once; calls that
 * share it must be ordered, replays of captured ones among them).  Its first int32 counts blocks
 * of op_linear with a wait that gave up (0 unless the GPU is at fault: a call with such a block
 * has returned 0, and what it wrote is not its result).  0 on bad arguments. */
size_t op_linear_work_bytes(const op_linear_t* args);
int op_linear(const op_linear_t* args, void* work, size_t work_bytes, gmg_stream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* GMGOP_H */
