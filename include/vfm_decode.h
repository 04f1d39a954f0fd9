/* Decoding over a bounded KV cache (libvfm.so): appending rotated keys and
 * values to a paged cache, attention of new tokens over that cache with a
 * sliding window and first tokens that stay visible, one backbone layer with
 * that attention, and drawing the next tokens from the head outputs.
 *
 * Token-based FMs are served with continuous batching and long-lived decode
 * iterations (paper Section 4.2; Section 6: a vLLM-style runtime, whose KV
 * cache is paged).  A sliding window bounds what a long-lived sequence keeps
 * and reads; the calls here work on the batches, plans and page tables of
 * vfm.h and follow its conventions (row order, ownership, streams, errors:
 * everything is checked on the host before anything is enqueued, nothing is
 * allocated, no pointer is kept).  In addition, every call here refuses a
 * stream of another device than the current one with VFM_ERR_ARG.
 *
 * All pointers to K / V, queries, outputs and workspaces must be 16-byte
 * aligned (VFM_ERR_ARG), workspaces 256-byte aligned (VFM_ERR_WORKSPACE).
 */
#ifndef VFM_DECODE_H
#define VFM_DECODE_H

#include "vfm.h"

#ifdef __cplusplus
extern "C" {
#endif

/* One attention over a paged cache: its head layout and what a row sees.
 * n_heads query heads share n_kv_heads key / value heads, n_heads / n_kv_heads
 * (1 .. 64) consecutive query heads each; n_heads <= 1024; head_dim 64 or 128.
 * The row at position j sees the key at position k iff
 *   k <= j  and  (window == 0  or  j - k < window  or  k < n_sink),
 * so a row always sees itself; with window 0 n_sink has no effect. */
typedef struct vfm_attn {
  int32_t dtype;        /* VFM_F32 | VFM_BF16: queries, cache and outputs */
  int32_t n_heads;
  int32_t n_kv_heads;
  int32_t head_dim;
  int32_t window;       /* 0: every earlier key; else 1 .. 2^30 */
  int32_t n_sink;       /* 0 .. 2^30 first tokens that stay visible */
  float scale;          /* of q . k, > 0; 0: 1 / sqrt(head_dim) */
  float rope_theta;     /* vfm_kv_append: 0 no rotation, else the RoPE base */
} vfm_attn;

/* Rotary embedding of new rows and the write of their K / V to the cache.
 *   qkv:   device [T, ld] (dtype), plan order: n_heads query heads, then
 *          n_kv_heads key heads, then n_kv_heads value heads of head_dim;
 *          ld >= (n_heads + 2 n_kv_heads) * head_dim, a multiple of 8.
 *   q_out: device [T, n_heads * head_dim]: the rotated queries (must not
 *          overlap qkv).
 *   kv:    the cache, [n_kv_heads][n_pages * page_size][head_dim] (dtype).
 * Row i of a request goes to position ctx + i; its rotation (rotate-half, as
 * in vfm_layer_forward) is by that position, the angles taken in 64 bits so
 * that far positions keep theirs, one rounding of the result.  Values are
 * copied bit for bit.  With rope_theta 0 queries and keys are, too.
 * Only the pages of the new positions are looked at.  Two new rows that a
 * page table sends to one slot leave either of them there.
 * Errors: VFM_ERR_ARG, VFM_ERR_SHAPE (head layout, ld, a request's pages
 * outside the table or [0, n_pages), ctx + len above 2^30, n_pages *
 * page_size of 2^31 or more), VFM_ERR_UNSUPPORTED (head_dim, group, a step of
 * 2^24 rows and more). */
int vfm_kv_append(const vfm_attn* attn, const vfm_batch* batch, const void* qkv, int64_t ld,
                  void* q_out, const vfm_kv_pages* kv, void* stream);

/* Attention of the batch's rows over their requests' pages; the rows' own K / V
 * are in the cache already (vfm_kv_append, or any earlier write).
 *   q:   device [T, ldq] (dtype), plan order, heads of head_dim from column 0;
 *        ldq >= n_heads * head_dim, a multiple of 8 (rows of a larger matrix).
 *   out: device [T, ldo] (dtype), ldo as ldq; columns past n_heads * head_dim
 *        stay as they were.  Must not overlap q.
 *   workspace: device, >= vfm_attention_workspace bytes; concurrent calls
 *        must not share one, and neither may graphs that can run at once.
 * A request has one row (decode) or many (a prompt or a chunk of one), after
 * any number of cached tokens.  Only pages with a position that one of the
 * request's rows sees are looked at: entries of pages that lie between the
 * sinks and the window may hold anything, so a sequence can give them back
 * or use them again (a ring of pages).  What unseen slots of seen pages hold
 * (NaN and infinities too) does not reach any output.
 * A row's result does not depend on the batch around its request.  The
 * softmax is taken in fp32; bf16 rounds its weights to bf16 for the product
 * with V.  The workspace holds partial results of the requests whose keys go
 * to many blocks (long contexts of few rows), of each as much as alone, up to
 * twice that or 16 MB where this is simpler; 0 bytes where there is none.
 * Errors as vfm_kv_append, plus VFM_ERR_WORKSPACE and VFM_ERR_UNSUPPORTED for
 * steps of 2^24 blocks and more: key heads times, in bf16, 16 packed queries
 * (rows x group) of requests with up to 32, 128 of others, in fp32 16. */
int vfm_attention_workspace(const vfm_attn* attn, const vfm_batch* batch, size_t* bytes);
int vfm_attention_paged(const vfm_attn* attn, const vfm_batch* batch, const void* q, int64_t ldq,
                        const vfm_kv_pages* kv, void* out, int64_t ldo, void* workspace,
                        size_t ws_bytes, void* stream);

/* vfm_layer_forward_paged with that append and attention (n_kv_heads =
 * cfg->n_heads; the rotation's angles in 64 bits):
 * one backbone layer of a causal, decode or mixed step whose rows see the
 * window and the sinks only.  Any request may be a prompt, a chunk after
 * cached tokens or a single row, in bf16 and fp32.  Pages are needed for the
 * positions that some row sees or that a new row is written to.
 * The workspace is vfm_workspace_size_windowed's.  Errors as
 * vfm_layer_forward_paged (VFM_ERR_UNSUPPORTED: VFM_ATTN_BIDIR, a
 * VFM_ATTN_DECODE request of several rows, a VFM_ATTN_CAUSAL request with
 * ctx > 0) and vfm_attention_paged. */
int vfm_workspace_size_windowed(const vfm_cfg* cfg, const vfm_batch* batch, const vfm_lora_table* lora,
                                int32_t window, int32_t n_sink, size_t* bytes);
int vfm_layer_forward_windowed(const vfm_cfg* cfg, const vfm_layer_weights* w, const vfm_lora_table* lora,
                               const vfm_batch* batch, float* x, const vfm_kv_pages* kv, int32_t window,
                               int32_t n_sink, void* workspace, size_t ws_bytes, void* stream);

/* Per-request sampling parameters: device arrays [n_req] in ORIGINAL order,
 * each may be NULL (its filter off, temperature 1).  They are read by the
 * kernel, so values out of range are given a meaning instead of an error. */
typedef struct vfm_sampling {
  const float* temperature;  /* > 0 (taken within 1e-30 .. 1e30); <= 0 or NaN: greedy */
  const int32_t* top_k;      /* >= 1: that many; <= 0: off */
  const float* top_p;        /* < 1: that share (<= 0: the first alone); >= 1 or NaN: off */
  const float* min_p;        /* > 0: at least that share of the largest; <= 0 or NaN: off */
} vfm_sampling;

/* The next token of each request, drawn from its head outputs.
 *   out: device float32 head outputs (vfm_head_forward's layout: request i's
 *     n_i outputs l_j from out_off[i], original order).
 *   u:   device float32 [n_req], original order: one uniform number in [0, 1)
 *     per request (below 0 or NaN: 0; 1 and more: the last token with any
 *     weight).
 *   ids: device int32 [n_req]; logprob: device float32 [n_req] or NULL.
 * With M the largest l, w_j = exp((l_j - M) / T), 1 where l_j = M (also where
 * M is infinite) and 0 for a NaN.  The outputs in the order of l, ties by
 * lowest index first: top-k keeps the first k; top-p keeps of those the
 * shortest run from the start whose weights reach top_p times the sum of
 * those k; min-p keeps of those the ones with w_j >= min_p.  The first is
 * always kept.  The token is the first kept one, by index, at which the
 * running sum of kept weights exceeds u times their sum S, and logprob
 * log(w_j / S).  Greedy (temperature <= 0): the largest output, ties to the
 * lowest index, logprob 0.  A request with no non-NaN output: -1, logprob NaN.
 * Weights are computed in fp64, rounded to s-bit fixed point (s = 44 up to
 * 2^19 outputs, then 63 - ceil(log2 n): 43 up to 2^20, 33 at 2^30, as many as
 * a 64-bit sum holds) and summed exactly, in any order: a weight below
 * 2^-(s + 1) of the largest counts as 0, and the result does not depend on
 * how the work is split.
 * VFM_ERR_SHAPE: a request of more than 2^30 outputs.  VFM_ERR_UNSUPPORTED:
 * 2^24 requests and more, 2^22 where one has more than 1024 outputs. */
int vfm_sample_tokens(const vfm_batch* batch, const float* out, const vfm_sampling* sampling,
                      const float* u, int32_t* ids, float* logprob, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* VFM_DECODE_H */
