/*
 * pasta_kv8.h -- C ABI of the 8-bit paged KV cache: its places, its rows, its attention.
 *
 * The cache serves the same step as pasta_attn.h (several decoding streams of a
 * request over one pool of interleaved rows), with two differences.  K and V are
 * held in 8 bits, which halves what a step has to read.  And everything that
 * changes from step to step -- lengths, page tables, slots, the split of the work
 * -- is made on the GPU from device arrays, so that a captured step can be
 * replayed token after token without the host.
 *
 * A step is   pasta_kv8_slots     places of the new rows (once per step)
 *             pasta_kv8_plan      split of the attention's work (once per step)
 *             pasta_kv8_append    the new rows of a layer, as codes (per layer)
 *             pasta_kv8_attend    the attention of a layer (per layer)
 *
 * Conventions are those of pasta_attn.h: status codes, nothing throws or aborts,
 * DEVICE pointers are the caller's, the library allocates no device memory, all
 * work is enqueued on the handle's stream, whose device has to be the current one.
 * The calls make no HIP call but kernel launches, so all four may be captured into
 * a graph.  A caller that uses a buffer on another stream orders the two itself.
 * Calls on one handle are not thread-safe.
 *
 * DEVICE arrays cannot be checked on the host.  The kernels check what they read
 * from them before they use it as an address: lengths and offsets are clamped to
 * the sizes given here, and a page number outside [0, n_phys_pages) is no page
 * (rows that would go there are dropped, tokens there are seen by nobody).
 */
#ifndef PASTA_KV8_H
#define PASTA_KV8_H

#include <stdint.h>

#include "pasta_attn.h" /* status codes */

#ifdef __cplusplus
extern "C" {
#endif

typedef struct pasta_kv8 pasta_kv8; /* opaque */

/* How a code stands for a number, in units of its block's scale. */
enum {
  PASTA_KV8_E4M3 = 0, /* sign, 4 bits of exponent, 3 of mantissa; largest 448, no infinity */
  PASTA_KV8_INT8 = 1  /* -127 .. 127 */
};

/* Types of rows (PASTA_F32 and PASTA_BF16 of pasta_attn.h, and fp16). */
enum { PASTA_F16 = 2 };

/* The cache.
 *
 * A SLOT is a place for one token: slot = page * page_tokens + offset.  16
 * consecutive slots are a BLOCK: block b of page p is slots
 * p * page_tokens + 16 b .. + 15.  For each layer, block and kv head g there is one
 * K scale and one V scale, fp32 powers of two (or NaN, see pasta_kv8_append):
 *
 *   scale index  (p * Hkv + g) * (page_tokens / 16) + b
 *
 * and 16 * D bytes of codes for each, at that index times 16 * D, in the order in
 * which the attention's matrix instructions take them:
 *
 *   K   [D / 16][16 tokens][16 dims]
 *   V   [D][16 tokens]
 *
 * Layer l starts at l * n_phys_pages * Hkv * (page_tokens / 16) scales.          */
typedef struct {
  uint32_t struct_size;      /* sizeof(pasta_kv8_config) */
  int32_t codes;             /* PASTA_KV8_E4M3 | PASTA_KV8_INT8 */
  int32_t dtype;             /* PASTA_BF16 | PASTA_F16: q and out */
  int32_t n_q_heads;         /* Hq */
  int32_t n_kv_heads;        /* Hkv <= 256; Hq / Hkv in {1, 2, 4, 8}; head h reads kv head h / (Hq / Hkv) */
  int32_t head_dim;          /* D in {64, 128} */
  int32_t n_layers;
  int32_t max_requests;      /* rows of page_table */
  int32_t max_rows;          /* most rows of one step, all requests together */
  int32_t page_tokens;       /* a power of two, 16 .. 4096 */
  int32_t n_phys_pages;      /* n_phys_pages * page_tokens < 2^31 */
  int32_t pages_per_request; /* columns of page_table; * page_tokens <= 2^27 */
  float softmax_scale;       /* finite; applied to q.k */
  void *k_codes, *v_codes;   /* DEVICE, 16-byte aligned.  Any of the DEVICE pointers from here on may be */
  float *k_scale, *v_scale;  /* DEVICE                     NULL if no call is made that needs it.         */
  int32_t *page_table;       /* DEVICE [max_requests][pages_per_request] */
  int32_t *free_pages;       /* DEVICE [n_phys_pages]: a stack of free pages (slots) */
  uint8_t *slot_tag;         /* DEVICE [n_phys_pages * page_tokens], 16-byte aligned: who wrote the slot (slots, attend) */
  int32_t *slot_position;    /* DEVICE [n_phys_pages * page_tokens], 16-byte aligned: its position id (slots, attend) */
  void *workspace;           /* DEVICE, 256-byte aligned, used by slots, plan and attend */
  uint64_t workspace_bytes;  /* in: bytes provided; query mode writes bytes needed */
  void *hip_stream;
} pasta_kv8_config;

/* Creates a handle (out == NULL: checks cfg but for its pointers and writes the
 * workspace's size).  Makes no HIP call.
 * Errors: E_INVAL, E_CAPACITY (workspace too small), E_NOMEM.                    */
int32_t pasta_kv8_create(pasta_kv8_config *cfg, pasta_kv8 **out);
int32_t pasta_kv8_destroy(pasta_kv8 *h);

/* Places of a step's rows.  Request r holds length[r] tokens.  Of these it keeps
 * kept = min(length[r], keep[r]) (drafts taken back; 0 releases it) and gets
 * n = row_offsets[r + 1] - row_offsets[r] new rows behind them; it needs
 * ceil((kept + n) / page_tokens) pages and has ceil(length[r] / page_tokens).
 *
 *   pages no longer needed go onto the stack, requests ascending, pages of a
 *   request ascending; then pages that are needed come off its top, in the same
 *   order (the k-th page taken is the k-th from the top).
 *   A request is REFUSED, and nothing of it changes, if it would outgrow its row of
 *   the page table, or if it needs pages and the needs of the requests up to and
 *   including it (those that would outgrow their table not counted) exceed the stack.
 *
 * Writes page_table (entries of taken pages; an entry past a request's pages keeps
 * its old value), free_pages, length_out[r] (kept + n; of a refused request,
 * length[r]), *free_out (pages left), slot[i] of every row i < n_rows (-1: of a
 * refused request, behind row_offsets[n_requests], or where a page number is bad),
 * and for every row with a slot slot_tag[slot] = row_tag[i],
 * slot_position[slot] = row_position[i] (where given).
 * length_out may be length, and free_out free_count: then a captured call advances
 * by itself.  Needs page_table, free_pages, workspace.
 * Errors: E_INVAL, E_CAPACITY (n_requests, n_rows), E_DEVICE, E_STATE.           */
typedef struct {
  uint32_t struct_size, flags;    /* flags: 0 */
  int32_t n_requests, n_rows;
  const int32_t *length;          /* DEVICE [n_requests] */
  const int32_t *keep;            /* DEVICE [n_requests], or NULL: everything */
  const int32_t *row_offsets;     /* DEVICE [n_requests + 1], ascending from 0 */
  const uint8_t *row_tag;         /* DEVICE [n_rows], or NULL */
  const int32_t *row_position;    /* DEVICE [n_rows], or NULL */
  const int32_t *free_count;      /* DEVICE [1]: pages on the stack */
  int32_t *slot;                  /* DEVICE [n_rows] out */
  int32_t *length_out;            /* DEVICE [n_requests] out */
  int32_t *free_out;              /* DEVICE [1] out */
} pasta_kv8_slots_args;
int32_t pasta_kv8_slots(pasta_kv8 *h, const pasta_kv8_slots_args *a);

/* New rows of one layer into the cache, k_new and v_new [n_rows][Hkv][D].  Rows of
 * one block have to be neighbours with ascending slots, as pasta_kv8_slots gives
 * them out; rows whose slot is not in [0, n_phys_pages * page_tokens) are skipped.
 *
 * Scales.  Q = 448 (E4M3) or 127 (INT8).  For the rows that a call brings into a
 * block, per kv head and for K and V apart, e = the least whole number with
 * max|x| <= Q * 2^e, held within [-100, 119].
 *   A run that starts at the block's first slot starts the block anew: its scale
 *   is 2^e, and its slots behind the run read as 0.
 *   A run that goes on in a block raises its scale 2^f to 2^max(e, f); if that is
 *   more than 2^f, the codes ahead of the run are rounded again, x -> x * 2^(f-e).
 *   (E4M3: exact but for its subnormals.  INT8: since scales at least double, all
 *   roundings of a value together are off by less than one step of the last scale.)
 *   code = the nearest to x * 2^-e, ties to even; beyond Q (only past 2^119 Q) it is Q.
 *   If any of the new values is infinite or NaN, the scale becomes NaN: the whole
 *   block reads as NaN for this head from then on, until it is started anew.  The
 *   codes of rows that go into such a block are 0: no code stands for NaN.
 *
 * Needs the codes and scales.  k_new, v_new 16-byte aligned.
 * Errors: E_INVAL, E_CAPACITY, E_DEVICE, E_STATE.                                */
typedef struct {
  uint32_t struct_size, flags;    /* flags: 0 */
  int32_t layer, n_rows;
  int32_t dtype;                  /* of the rows: PASTA_F32 | PASTA_BF16 | PASTA_F16 */
  const int32_t *slot;            /* DEVICE [n_rows] */
  const void *k_new, *v_new;      /* DEVICE */
} pasta_kv8_append_args;
int32_t pasta_kv8_append(pasta_kv8 *h, const pasta_kv8_append_args *a);

/* Split of the attention's work of one step, kept in the workspace until the next
 * pasta_kv8_plan of the handle: which tokens each work-group reads.  length[] counts
 * the step's own rows, which are a request's last n (length_out of pasta_kv8_slots).
 * slot (optional): a request whose first row has no slot was refused; its rows get
 * the result of a row that sees nothing.
 * Needs page_table and the workspace.  Errors: E_INVAL, E_CAPACITY, E_DEVICE,
 * E_STATE.                                                                       */
typedef struct {
  uint32_t struct_size, flags;    /* flags: 0 */
  int32_t n_requests, n_rows;
  int32_t max_request_rows;       /* no request has more rows than this (it decides which kernels run; rows
                                     beyond it are still right) */
  const int32_t *length;          /* DEVICE [n_requests] */
  const int32_t *row_offsets;     /* DEVICE [n_requests + 1] */
  const int32_t *prefix_len;      /* DEVICE [n_requests], or NULL: none */
  const int32_t *slot;            /* DEVICE [n_rows], or NULL */
} pasta_kv8_plan_args;
int32_t pasta_kv8_plan(pasta_kv8 *h, const pasta_kv8_plan_args *a);

/* Attention of the planned rows over one layer.  q, out [n_rows][Hq][D].  Row i of
 * request r is its token p = length[r] - n + i.  For head h, over the tokens j of r:
 *
 *   s_j = softmax_scale * <q, K_j>
 *   s_j = logit_cap * tanh(s_j / logit_cap)                     if logit_cap > 0
 *   s_j = s_j - slopes[h] * |position of the row - position of j|   if slopes
 *   visible:  j < length[r]  and  ( j < prefix_len[r]
 *             or  j <= p  and  (no row_see  or  bit slot_tag[slot of j] of row_see[row]) )
 *   out = sum_j softmax(s)_j V_j      lse = log sum_j exp(s_j)
 *
 * over the visible j; a row that sees nothing gets out = 0, lse = -inf.  Positions
 * are slot_position and row_position if row_position is given, else j and p.  Tags
 * are 0 .. 63 (taken modulo 64).  With a tag per stream, row_see is the set of the
 * streams whose rows a row's stream descends from; once all streams of a request
 * have joined, prefix_len covers them and their tags are free again.
 *
 * Sums, maxima and the output are held in fp32.  The softmax weights, each times
 * its block's V scale and in units of the row's largest such product, enter the
 * product with V as fp16: what is 2^-25 of the largest or less adds to the sums, but
 * nothing to out.  Rows that no request has (behind row_offsets[n_requests]) get
 * out = 0, lse = -inf.
 * Needs everything but free_pages; slot_tag with row_see, slot_position with
 * row_position.  n_rows is that of the last plan (E_STATE otherwise, or without one).
 * Errors: E_INVAL, E_DEVICE, E_STATE.                                            */
typedef struct {
  uint32_t struct_size, flags;    /* flags: 0 */
  int32_t layer, n_rows;
  float logit_cap;                /* 0: none; else > 0 and finite */
  const void *q;                  /* DEVICE, 16-byte aligned */
  void *out;                      /* DEVICE, 16-byte aligned */
  float *lse;                     /* DEVICE [n_rows][Hq], or NULL */
  const float *slopes;            /* DEVICE [Hq], or NULL */
  const uint64_t *row_see;        /* DEVICE [n_rows], or NULL */
  const int32_t *row_position;    /* DEVICE [n_rows], or NULL; only with slopes */
} pasta_kv8_attend_args;
int32_t pasta_kv8_attend(pasta_kv8 *h, const pasta_kv8_attend_args *a);

#ifdef __cplusplus
}
#endif
#endif /* PASTA_KV8_H */
