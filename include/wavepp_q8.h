/*
 * wavepp_q8.h -- C ABI of the 8-bit paged cache of libwavepp_attn.so: the append of a wave's K/V into pages of 8-bit
 * values, the way back to bf16 rows, and attention over such pages -- causal, or with capped scores, a bias on the
 * distance and an interval of keys for each query -- for chunks of any length from a single token (decoding) up, for
 * AMD gfx950 (MI355X).
 *
 * Format.  The 16 slots [16 i, 16 i + 16) of a page share a scale for each KV head: a value is an 8-bit e4m3 code (a
 * sign bit, four bits of exponent, three of mantissa; magnitudes 0, 2^-9 to 448, no infinities) times the block's power
 * of two 2^(e - 127), e being its scale byte.  The page of one KV head is one run of
 *     page_size * head_dim  code bytes, row by row, then
 *     16                    bytes, of which the first page_size / 16 are the scale bytes, block by block,
 * 1 + 1/512 (pages of 64, head dim 128) to 1 + 1/64 bytes a value against the 2 of bf16 pages.  Pools are
 * [num_pages][num_kv_heads][that run].
 *
 * Rounding (wavepp_q8_append_kv).  With amax the largest magnitude among a block's new values, the scale s is the
 * smallest power of two with amax <= 448 s, e not under 8, or the block's scale if it holds earlier tokens and theirs is
 * larger.  Every value is rounded to the nearest code times s, ties to the even code.  Where the scale of a block that
 * holds earlier tokens grows, their codes are rounded again to the new one: what stays normal (2^-6 s and more) keeps its
 * value, and what falls below is off by at most 2^-10 s more.  So a stored value depends on how a block was cut into
 * appends only by that.  Magnitudes over 1.75 * 2^127, infinities and NaN count as 1.75 * 2^127 of their sign, so e is at
 * most 246, and every value that the append stores is exactly a bf16 number.  They reach only the queries that see their
 * row, but take the precision of their block.
 *
 * Everything else -- spans, block tables, which page may appear where, the workspace and its upload, ownership, streams
 * and errors -- is as in wavepp_attn.h.  A plan made here is a wavepp_plan: wavepp_plan_workspace_bytes,
 * wavepp_plan_get_info, wavepp_plan_get_items, wavepp_attn_plan_upload and wavepp_plan_destroy take it, and the entry
 * points of the other caches, whose pages are of another size, refuse it (WAVEPP_EINVAL), as those below refuse theirs.
 *
 * Call order on one stream, per wave: wavepp_q8_plan (host only) -> wavepp_attn_plan_upload -> wavepp_q8_append_kv ->
 * wavepp_q8_chunked_prefill (the last two once per layer, each with its own pools).  The launches of both may be captured
 * into a graph after the upload; its replays run on whatever the buffers then hold.  Calls whose plans have splits write
 * partials into their workspace, so calls that may overlap need a workspace each.  The scores are part of the plan: a model
 * whose layers differ in theirs, a window here and the whole past there, has a plan, a workspace and an upload a wave for
 * each kind, and any of them will do for the append.
 */
#ifndef WAVEPP_Q8_H
#define WAVEPP_Q8_H

#include "wavepp_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* What a layer's scores are, beyond the causal softmax_scale q.k of wavepp_attn.h; all HOST memory, copied by
 * wavepp_q8_plan.  Of query t of the wave (packed), at position i of its request, and key j, in this order:
 *     s = softmax_scale q.k
 *     s = cap tanh(s / cap)            where cap > 0 (1e-3 to 1e6)
 *     s = s - slopes[head] |i - j|     where slopes is not NULL (num_q_heads numbers within [-1024, 1024])
 *     key j has weight exp(s) where key_begin[t] <= j < key_end[t], and none elsewhere.
 * key_begin NULL is 0 and key_end NULL is i + 1 for every query, which is the causal rule.  Both arrays have one entry for
 * each new token, in [0, p_r + c_r]: a window of w keys is key_begin = max(0, i + 1 - w), a document's tokens begin at its
 * first position, and a prefix that all of a request sees ends no earlier than its last position.  A query whose interval
 * is empty sees nothing: its output is zero and its lse -infinity.
 * A tile is up to 256 rows of neighbouring queries of a request, the heads of a KV head's group being rows of their own.  Its
 * keys are read from the first that one of its queries sees to the last: what lies before or behind may hold any bytes, so
 * that any page of the pool may stand in the block table for those that every window has left.  Keys between that lie in
 * none of its queries' intervals are read and have no weight, so they have to be rows that an append stored. */
typedef struct {
  float cap;
  const float* slopes;
  const int32_t* key_begin;
  const int32_t* key_end;
} wavepp_q8_scores;

/* Bytes of one page of one KV head; 0 unless head_dim is 64 or 128 and page_size 16 or 64. */
size_t wavepp_q8_page_bytes(int32_t head_dim, int32_t page_size);

/* wavepp_attn_plan for an 8-bit cache.  Supported: (head_dim_qk, head_dim_v) in {(64, 64), (128, 128)}, kv_shared = 0, any
 * num_q_heads % num_kv_heads == 0, page_size in {16, 64}; a latent cache is WAVEPP_EUNSUPPORTED.  scores may be NULL; one
 * out of the ranges above is WAVEPP_EINVAL, as is a softmax_scale over 1e30 times a cap or under 1e-20 beside slopes.
 * Arguments and errors otherwise as there. */
int wavepp_q8_plan(const wavepp_attn_shape* shape, const wavepp_batch* batch, const wavepp_q8_scores* scores,
                   int32_t max_splits, wavepp_plan** out);

/* Round the wave's new rows into the pages reserved for them.  Device pointers, contiguous:
 *   k_new [T][num_kv_heads][head_dim], v_new likewise, bf16, 16-byte aligned;
 *   k_pool, v_pool [num_pages][num_kv_heads][wavepp_q8_page_bytes], 16-byte aligned.
 * Written are the codes of the wave's new tokens, the scale bytes of their blocks and, where such a scale grows, the codes
 * of the block's earlier tokens.  Enqueued again on the same rows it leaves the same bytes.  A wave whose blocks of 16 slots
 * come to 2^25 or more, times num_kv_heads and in whole fours, is WAVEPP_EUNSUPPORTED, here and in wavepp_q8_read_kv.  Errors
 * otherwise as for wavepp_attn_append_kv. */
int wavepp_q8_append_kv(const wavepp_plan* plan, const void* k_new, const void* v_new, void* k_pool, void* v_pool,
                        void* workspace, size_t ws_bytes, hipStream_t stream);

/* The way back: the bf16 rows of the wave's new tokens [p_r, p_r + c_r) as the pages hold them, exactly (a code of NaN or
 * a scale byte over 246, which no append writes, may give NaN or infinity, one under 3 zero).  To read a request's whole
 * cache, plan it with p_r = 0 and c_r its length.  k_out, v_out [T][num_kv_heads][head_dim] bf16, 16-byte aligned. */
int wavepp_q8_read_kv(const wavepp_plan* plan, const void* k_pool, const void* v_pool, void* k_out, void* v_out,
                      void* workspace, size_t ws_bytes, hipStream_t stream);

/* Attention of the wave's queries over the cached values with the plan's scores, K and V read from 8-bit pages: bf16 q and
 * out, fp32 natural-log lse (or NULL).  bf16 products of the exact cached values with fp32 accumulation, scores and
 * softmax; the weights are rounded to bf16 for their products with V, their sum in the lse is of the weights themselves.
 * A row whose softmax sum is not a number (a NaN in its query, a largest score that overflows or lies beyond
 * 2^28 ln 2, where fp32 cannot place its exponential) has NaN as its output and its lse, whole or joined from splits.
 * Scores under -2^28 ln 2 have no weight; an lse of -infinity says that no key had any, and the output is then zero.  A
 * capped score is off by at most 2^-20 of itself plus, for a cap of 128 or less, 2^-21 of the cap.  With a cap of 50 or
 * less and no slopes, weights of 2^-80 to 2^65 are summed, so values of V over 2^40 may overflow to infinity where scores
 * lie near the cap, and those under 2^-40 may lose bits where all of a row's scores lie near -cap.
 * Deterministic: repeated calls give bit-identical results.  A plan with 2^24 items or more (wavepp_plan_get_info) of requests
 * of up to 32 rows a KV head, or 2^23 or more of longer ones, is WAVEPP_EUNSUPPORTED.  Errors otherwise as for
 * wavepp_attn_chunked_prefill. */
int wavepp_q8_chunked_prefill(const wavepp_plan* plan, const void* q, const void* k_pool, const void* v_pool, void* out,
                              float* lse, void* workspace, size_t ws_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* WAVEPP_Q8_H */
