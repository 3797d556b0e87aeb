/*
 * pasta_rows.h -- C ABI of what a step does to its rows beside the cache: rotary
 * positions on their way in, drafted tokens against the target's probabilities on
 * their way out.
 *
 * Both caches (pasta_kv8.h, pasta_kv4.h) take keys and queries that are turned already,
 * by position ids that need not be consecutive.  And pasta_kv8_slots takes drafts back
 * by keep[]: pasta_rows_verify writes it.  So a captured step
 *
 *   slots (keep, no rows) -> slots -> plan -> per layer: rotate, append, attend -> verify
 *
 * goes on by as many tokens as were accepted, without the host.  Drafts are taken back by
 * a call of their own, ahead of the one that places the step's rows: a request that this one
 * refuses stays as it is, so that with keep[] its rejected drafts would stay in the cache.
 *
 * Conventions are those of pasta_kv8.h: status codes, nothing throws or aborts, DEVICE
 * pointers are the caller's, all work is enqueued on the handle's stream, whose device
 * has to be the current one, no call makes a HIP call but kernel launches, so all may be
 * captured, what comes from DEVICE arrays is checked by the kernels before it is used
 * as an address, calls on one handle are not thread-safe.
 */
#ifndef PASTA_ROWS_H
#define PASTA_ROWS_H

#include <stdint.h>

#include "pasta_kv8.h" /* status codes, types of rows */

#ifdef __cplusplus
extern "C" {
#endif

typedef struct pasta_rows pasta_rows; /* opaque */

/* Which dims make up a plane of the rotation: f and f + rope_dims / 2, or 2f and 2f + 1. */
enum { PASTA_ROPE_HALF = 0, PASTA_ROPE_INTERLEAVED = 1 };

/* A handle for rotate has rope_dims > 0, one for verify vocab > 0; the fields of the other
 * are then 0.                                                                     */
typedef struct {
  uint32_t struct_size;      /* sizeof(pasta_rows_config) */
  int32_t max_rows;          /* most rows of one call, < 2^24 */
  /* rotate */
  int32_t n_q_heads, n_kv_heads; /* >= 1, together <= 1024 */
  int32_t head_dim;          /* a multiple of 8, <= 256 */
  int32_t rope_dims;         /* even, 2 .. head_dim: the first dims of a head are turned, the others stay */
  int32_t rope_layout;       /* PASTA_ROPE_HALF | PASTA_ROPE_INTERLEAVED */
  float rope_magnitude;      /* of what is turned, finite; 1 unless a scaling for long contexts asks for another */
  const double *rope_frequency; /* DEVICE [rope_dims / 2]: radians a position, of each plane */
  /* verify */
  int32_t vocab;             /* <= 2^22 */
  int32_t max_sequences;
  void *workspace;           /* DEVICE, 256-byte aligned, used by verify; NULL if that needs none */
  uint64_t workspace_bytes;  /* in: bytes provided; query mode writes bytes needed */
  void *hip_stream;
} pasta_rows_config;

/* Creates a handle (out == NULL: checks cfg but for its pointers and writes the
 * workspace's size).  Makes no HIP call.
 * Errors: E_INVAL, E_CAPACITY (workspace too small), E_NOMEM.                    */
int32_t pasta_rows_create(pasta_rows_config *cfg, pasta_rows **out);
int32_t pasta_rows_destroy(pasta_rows *h);

/* Turns rows of q [n_rows][Hq][D] and k [n_rows][Hkv][D] by their positions: with
 * a = position * rope_frequency[f], a plane (x, y) becomes
 *
 *   rope_magnitude * (x cos a - y sin a,  y cos a + x sin a)
 *
 * PASTA_ROWS_BACKWARD: a is -a, which is the gradient's way back (and, with a magnitude
 * of 1, the inverse).  Angles are computed in 64 bits, the rest in fp32, rounded once.
 * q_out may be q, and k_out k, with the same stride; else they do not overlap.  q or k
 * may be NULL, with its out.  Row i lies at i * stride values (0: side by side): rows can
 * be parts of a projection's.
 * Pointers 16-byte aligned; strides whole numbers of 16 bytes, no less than a row.
 * Errors: E_INVAL, E_CAPACITY (n_rows), E_DEVICE, E_STATE.                       */
enum { PASTA_ROWS_BACKWARD = 1 };
typedef struct {
  uint32_t struct_size, flags;    /* flags: 0 | PASTA_ROWS_BACKWARD */
  int32_t n_rows;
  int32_t dtype;                  /* PASTA_F32 | PASTA_BF16 | PASTA_F16 */
  const int32_t *position;        /* DEVICE [n_rows] */
  const void *q, *k;              /* DEVICE */
  void *q_out, *k_out;            /* DEVICE */
  int64_t q_stride, k_stride, q_out_stride, k_out_stride; /* in values */
} pasta_rows_rotate_args;
int32_t pasta_rows_rotate(pasta_rows *h, const pasta_rows_rotate_args *a);

/* Drafted tokens against the target.  Sequence s has the step's rows
 * o = row_offsets[s] .. row_offsets[s + 1] - 1, n of them: the last token that was kept
 * and n - 1 drafts.  Row i of target is the distribution p_i of what follows row i; row i
 * of draft the distribution q_i that token[i] was drawn from (row o of it is not read).
 * Without draft, tokens were not drawn but chosen: q_i is 1 at token[i] and 0 elsewhere.
 *
 *   draft i is accepted if all ahead of it are and draw[i] * q_i[token[i]] < p_{i-1}[token[i]]
 *   a = number of accepted drafts, j = o + a the last row that stays
 *   w = max(p_j - q_{j+1}, 0) if a draft was rejected, else (and if that is 0 throughout) p_j
 *   next_token = the least t with  w_0 + .. + w_t > last_draw[s] * (w_0 + .. + w_{vocab-1})
 *
 * Products, differences and sums are those of 64 bits.  Weights that are not finite and above 0
 * count as 0, draws are held within [0, 1 - 2^-24], a token outside of the vocabulary is rejected;
 * next_token is -1 if no weight is left, or n is 0.
 *
 *   accepted[s] = a      keep[s] = length[s] - n + 1 + a (of length[s] tokens, the step's
 *   rows among them; length[s] if n is 0): pasta_kv8_slots's keep for the next step
 *   position_out[i] = row_position[i] + 1 + a for the sequence's rows: their positions in
 *   the next step.  It may be row_position.
 *
 * slot (optional): the rows' places, as pasta_kv8_slots gave them.  A sequence whose first
 * row has none was refused: a is 0, next_token -1, keep[s] = length[s] (what of it was to be
 * taken back has been, ahead of the step), and its positions stay.
 *
 * Rows behind row_offsets[n_sequences] are left alone.  Strides are at least vocab, in values.
 * Needs the workspace.  Errors: E_INVAL, E_CAPACITY, E_DEVICE, E_STATE.          */
typedef struct {
  uint32_t struct_size, flags;    /* flags: 0 */
  int32_t n_sequences, n_rows;
  int32_t dtype;                  /* of the probabilities: PASTA_F32 | PASTA_BF16 | PASTA_F16 */
  const int32_t *row_offsets;     /* DEVICE [n_sequences + 1] */
  const int32_t *token;           /* DEVICE [n_rows] */
  const int32_t *slot;            /* DEVICE [n_rows], or NULL */
  const void *target;             /* DEVICE [n_rows][vocab] */
  const void *draft;              /* DEVICE [n_rows][vocab], or NULL */
  int64_t target_stride, draft_stride; /* in values; 0: vocab */
  const float *draw;              /* DEVICE [n_rows] */
  const float *last_draw;         /* DEVICE [n_sequences] */
  const int32_t *length;          /* DEVICE [n_sequences], or NULL (with keep) */
  const int32_t *row_position;    /* DEVICE [n_rows], or NULL (with position_out) */
  int32_t *accepted;              /* DEVICE [n_sequences] out */
  int32_t *next_token;            /* DEVICE [n_sequences] out */
  int32_t *keep;                  /* DEVICE [n_sequences] out, or NULL */
  int32_t *position_out;          /* DEVICE [n_rows] out, or NULL */
} pasta_rows_verify_args;
int32_t pasta_rows_verify(pasta_rows *h, const pasta_rows_verify_args *a);

#ifdef __cplusplus
}
#endif
#endif /* PASTA_ROWS_H */
