/* Decoding over a paged KV cache held in 8 bits (libvfm.so): appending rotated
 * keys and values to it, attention of new tokens over it, and one backbone
 * layer with both.
 *
 * A token's K and V take half the bytes of a bf16 cache's: twice the tokens in
 * the same memory for the long-lived decode iterations of token-based FMs
 * (paper Section 4.2), and half the bytes that a decode step streams.  The
 * calls follow vfm_decode.h in everything that is not said here: batches,
 * plans, row order, windows and sinks, page tables, alignment, errors.
 */
#ifndef VFM_KV8_H
#define VFM_KV8_H

#include "vfm_decode.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Positions that share a scale: an aligned run of 16 of a page. */
#define VFM_KV8_RUN 16

/* The cache.  pages.k and pages.v are codes, device uint8
 * [n_kv_heads][n_pages * page_size][head_dim]: e4m3 numbers (sign, 4 exponent
 * bits of bias 7, 3 mantissa bits; up to 448; codes 0x7F and 0xFF are NaN, no
 * infinities).  exps, device uint8 [n_pages * page_size / 16][n_kv_heads][2],
 * holds a byte e for K and one for V of each run and key head: a slot's element
 * is its code's number times 2^(e - 127), 1 <= e <= 247.  exps needs no
 * initial contents, nor do the pools: the first row that a sequence writes to a
 * run sets its scale, whatever lies there. */
typedef struct vfm_kv_pages_q8 {
  vfm_kv_pages pages;
  void* exps;                 /* 16-byte aligned, as pages.k and pages.v */
} vfm_kv_pages_q8;

/* vfm_kv_append to that cache.  A new row's rotated key (its value) y is taken
 * in 64 bits, magnitudes above 1.875 * 2^127 as that, infinities as NaN.  For
 * each run, key head and pool, with a the largest |y| of the call's new rows in
 * the run (NaN apart; 0 if there is none):
 *   e = the least e >= 1 with a <= 448 * 2^(e - 127), no less than the run's
 *       byte so far if rows of the sequence are in the run already;
 *   code = y * 2^(127 - e) rounded once to e4m3, to the nearest, ties to even.
 * Where e grows, the codes of the rows that are there are multiplied by
 * 2^(old e - e), rounded the same way (only what becomes subnormal changes).
 * "Rows of the sequence" are the positions before ctx; slots behind the last
 * new row keep what they hold.  q_out gets the rotated queries, rounded once
 * to their type (bf16 ones below 2^-126 from a number up to 2^-149 off).  New
 * rows of two requests that a page table sends to one run leave either's scale
 * and codes of either there.  Errors as vfm_kv_append. */
int vfm_kv_append_q8(const vfm_attn* attn, const vfm_batch* batch, const void* qkv, int64_t ld,
                     void* q_out, const vfm_kv_pages_q8* kv, void* stream);

/* vfm_attention_paged over that cache: attn->dtype is the type of queries and
 * outputs.  With VFM_BF16 the products are of bf16 numbers (which hold every
 * code times its scale exactly), with VFM_F32 of fp32 ones.  A NaN code counts
 * as a NaN; what unseen slots hold, and scales of runs that no row sees, does
 * not reach any output.  The sums of weights times values are fp32 before they
 * are divided: a row's largest |value| times its visible keys times 2^8 stays
 * below 2^128.  Errors as vfm_attention_paged, workspace as
 * vfm_attention_workspace_q8 says. */
int vfm_attention_workspace_q8(const vfm_attn* attn, const vfm_batch* batch, size_t* bytes);
int vfm_attention_paged_q8(const vfm_attn* attn, const vfm_batch* batch, const void* q, int64_t ldq,
                           const vfm_kv_pages_q8* kv, void* out, int64_t ldo, void* workspace,
                           size_t ws_bytes, void* stream);

/* vfm_layer_forward_windowed over that cache (window 0: rows see every earlier
 * key).  The layer reads its new rows' keys and values back from the cache, so
 * a prompt in chunks and a prompt at once round them alike but for the runs
 * that a chunk's border cuts, whose scale grows in two steps. */
int vfm_workspace_size_q8(const vfm_cfg* cfg, const vfm_batch* batch, const vfm_lora_table* lora,
                          int32_t window, int32_t n_sink, size_t* bytes);
int vfm_layer_forward_q8(const vfm_cfg* cfg, const vfm_layer_weights* w, const vfm_lora_table* lora,
                         const vfm_batch* batch, float* x, const vfm_kv_pages_q8* kv, int32_t window,
                         int32_t n_sink, void* workspace, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* VFM_KV8_H */
