/*
 * pasta_kv4.h -- C ABI of the 4-bit paged KV cache: its rows, in and out, and its attention.
 *
 * The cache of pasta_kv8.h with half its bytes: the same pages, slots, tables, tags
 * and positions, the same plan and the same attention, over codes of 4 bits.  The
 * places of a step's rows are pasta_kv8_slots's, by a pasta_kv8 handle over the same
 * page table (it needs neither codes nor scales).  A step is
 *
 *                     pasta_kv8_slots     places of the new rows (once per step)
 *                     pasta_kv4_plan      split of the attention's work (once per step)
 *                     pasta_kv4_append    the new rows of a layer, as codes (per layer)
 *                     pasta_kv4_attend    the attention of a layer (per layer)
 *
 * Conventions are those of pasta_kv8.h: status codes, nothing throws or aborts, DEVICE
 * pointers are the caller's, all work is enqueued on the handle's stream, whose device
 * has to be the current one, no call makes a HIP call but kernel launches, so all may be
 * captured, what comes from DEVICE arrays is checked by the kernels before it is used
 * as an address, calls on one handle are not thread-safe, handles share no memory but
 * what they are given, and two handles of one workspace exclude each other.
 */
#ifndef PASTA_KV4_H
#define PASTA_KV4_H

#include <stdint.h>

#include "pasta_kv8.h" /* status codes, types of rows, arguments of plan and attend */

#ifdef __cplusplus
extern "C" {
#endif

typedef struct pasta_kv4 pasta_kv4; /* opaque */

/* The cache.
 *
 * A code is a sign, two bits of exponent and one of mantissa: 0, 1/2, 1, 3/2, 2, 3, 4, 6
 * are the codes 0 .. 7, their negatives 8 .. 15.  Every row of K has a scale per kv head
 * and 32 dims, every row of V one per kv head: a power of two 2^e, -100 <= e <= 119, held
 * as the byte e + 127, or the byte 255, under which the values read as NaN.  (Of bytes that
 * are none of these pasta_kv4_read makes 2^(byte - 127); what pasta_kv4_attend makes of them
 * is not said.)
 *
 * Slots and blocks are those of pasta_kv8.h.  A block of 16 tokens of page p, kv head g is
 *
 *   block index  i = (p * Hkv + g) * (page_tokens / 16) + b
 *   K codes   at i * 8 D        [D / 32][16 tokens][32 dims]    two codes to a byte, the
 *   V codes   at i * 8 D        [D][16 tokens]                  first in its lower half
 *   K scales  at i * 16 (D/32)  [16 tokens][D / 32]
 *   V scales  at i * 16         [16 tokens]
 *
 * Layer l starts at block l * n_phys_pages * Hkv * (page_tokens / 16).                   */
typedef struct {
  uint32_t struct_size;      /* sizeof(pasta_kv4_config) */
  int32_t dtype;             /* PASTA_BF16 | PASTA_F16: q and out */
  int32_t n_q_heads;         /* as in pasta_kv8_config, to softmax_scale */
  int32_t n_kv_heads;
  int32_t head_dim;          /* D in {64, 128} */
  int32_t n_layers;
  int32_t max_requests;
  int32_t max_rows;
  int32_t page_tokens;
  int32_t n_phys_pages;
  int32_t pages_per_request;
  float softmax_scale;
  void *k_codes, *v_codes;   /* DEVICE, 16-byte aligned.  Any of the DEVICE pointers from here on may be */
  uint8_t *k_scale, *v_scale;/* DEVICE, 16-byte aligned   NULL if no call is made that needs it.         */
  const int32_t *page_table; /* DEVICE [max_requests][pages_per_request] (plan, attend) */
  const uint8_t *slot_tag;   /* DEVICE [n_phys_pages * page_tokens], 16-byte aligned (attend) */
  const int32_t *slot_position; /* DEVICE [n_phys_pages * page_tokens], 16-byte aligned (attend) */
  void *workspace;           /* DEVICE, 256-byte aligned, used by plan and attend */
  uint64_t workspace_bytes;  /* in: bytes provided; query mode writes bytes needed */
  void *hip_stream;
} pasta_kv4_config;

/* Creates a handle (out == NULL: checks cfg but for its pointers and writes the
 * workspace's size).  Makes no HIP call.
 * Errors: E_INVAL, E_CAPACITY (workspace too small), E_NOMEM.                    */
int32_t pasta_kv4_create(pasta_kv4_config *cfg, pasta_kv4 **out);
int32_t pasta_kv4_destroy(pasta_kv4 *h);

/* New rows of one layer into the cache: k_new, v_new [n_rows][Hkv][D], row i at
 * i * k_stride, i * v_stride values (0: rows side by side).  A row goes to slot[i];
 * rows whose slot is not in [0, n_phys_pages * page_tokens) are skipped.  Rows of one
 * block have to be neighbours (no skipped row between them, either) with ascending slots,
 * which may leave some out (those of pasta_kv8_slots do not), and no slot may stand in a
 * call twice: bytes that two tokens share are put back by who writes one of them.  What no
 * row is written to keeps its bytes.
 *
 * Per row, kv head and, of K, 32 dims: e = the least whole number with
 * max|x| <= 7 * 2^e, held within [-100, 119]; code = the nearest to x * 2^-e, ties to the
 * even code, beyond 6 it is 6.  So nothing up to 7 * 2^119 is off by more than 2^e.  If
 * any of the values is infinite or NaN, the scale's byte is 255 and the codes are 0.
 *
 * Needs the codes and scales.  k_new, v_new 16-byte aligned, strides whole numbers of 16
 * bytes and no less than Hkv * D values.
 * Errors: E_INVAL, E_CAPACITY, E_DEVICE, E_STATE.                                */
typedef struct {
  uint32_t struct_size, flags;    /* flags: 0 */
  int32_t layer, n_rows;
  int32_t dtype;                  /* of the rows: PASTA_F32 | PASTA_BF16 | PASTA_F16 */
  const int32_t *slot;            /* DEVICE [n_rows] */
  const void *k_new, *v_new;      /* DEVICE */
  int64_t k_stride, v_stride;     /* in values */
} pasta_kv4_append_args;
int32_t pasta_kv4_append(pasta_kv4 *h, const pasta_kv4_append_args *a);

/* Rows of one layer back out of the cache, the values that their codes stand for:
 * fp32 and bf16 hold them exactly, fp16 rounds them (beyond its range: infinite).
 * slot[] may name slots in any order and more than once (rows in neighbouring slots side
 * by side read fastest); rows whose slot is not in range are left as they were.
 * k_out or v_out may be NULL.  Alignment and strides as above.  n_rows is not bounded by
 * max_rows, but by 2^27.
 * Needs the codes and scales that are read.
 * Errors: E_INVAL, E_CAPACITY, E_DEVICE, E_STATE.                                */
typedef struct {
  uint32_t struct_size, flags;    /* flags: 0 */
  int32_t layer, n_rows;
  int32_t dtype;                  /* PASTA_F32 | PASTA_BF16 | PASTA_F16 */
  const int32_t *slot;            /* DEVICE [n_rows] */
  void *k_out, *v_out;            /* DEVICE, or one of them NULL */
  int64_t k_stride, v_stride;     /* in values */
} pasta_kv4_read_args;
int32_t pasta_kv4_read(pasta_kv4 *h, const pasta_kv4_read_args *a);

/* pasta_kv8_plan and pasta_kv8_attend over this cache, argument for argument.  Of what
 * is said there: a token whose K reads as NaN for a head gives NaN to the rows that see it,
 * one whose V does, too (out, not lse).  K enters the products exactly; q does, too; the
 * softmax weights, each times its token's V scale and in units of the row's largest such product,
 * enter the product with V as fp16: what is 2^-24 of the largest or less adds to the sums,
 * but nothing to out.  Scores are held in fp32, which tells those beyond 2^22 in magnitude
 * no longer apart by what matters: there out is still a mean of the values of tokens whose
 * scores are the largest within 2^-18 of that magnitude, and out and lse are finite as long
 * as the scores are (but where a block's V scales are more than 2^8 apart, or beyond 2^100,
 * they can be anything).                                                                 */
int32_t pasta_kv4_plan(pasta_kv4 *h, const pasta_kv8_plan_args *a);
int32_t pasta_kv4_attend(pasta_kv4 *h, const pasta_kv8_attend_args *a);

#ifdef __cplusplus
}
#endif
#endif /* PASTA_KV4_H */
