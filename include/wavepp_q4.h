/*
 * wavepp_q4.h -- C ABI of the 4-bit paged cache of libwavepp_attn.so: the append of a wave's K/V into
 * pages of 4-bit values, the way back to bf16 rows, and attention over such pages, for chunks of any
 * length from a single token (decoding) up, for AMD gfx950 (MI355X).
 *
 * Format.  Along the head dim, blocks of 32 values share a scale: a value is a 4-bit code, one sign
 * bit (8) over the magnitudes {0, 1/2, 1, 3/2, 2, 3, 4, 6}, times the block's power of two 2^(e - 127),
 * e being its scale byte.  The page of one KV head is one run of
 *     page_size * head_dim / 2   code bytes: row by row, value 2i of a row in the low four bits of its
 *                                byte i and value 2i + 1 in the high four, then
 *     page_size * head_dim / 32  scale bytes: row by row, block by block,
 * 17/32 bytes a value against the 2 of bf16 pages.  Pools are [num_pages][num_kv_heads][that run].
 *
 * Rounding (wavepp_q4_append_kv).  With amax the block's largest magnitude, the scale is the smallest
 * power of two s with amax <= 7 s, e clamped to [8, 252].  Every value is rounded to the nearest code
 * times s, ties to the even code, magnitudes over 6 s to 6 s; so with e inside its clamps no value is
 * off by more than s.  The format has no infinities and no NaN: they count as the largest finite
 * magnitude of their sign and reach only the queries that see their row.  A V row that had one shows there as
 * outputs of order 1e38 times its weight, or infinite.  A K row that had one shows as NaN in outputs and LSE where it makes a
 * logit too large, and has no weight, so leaves no trace, where it makes it as far below zero.
 * Every value that the append stores is exactly a bf16 number.
 *
 * Everything else -- spans, block tables, which page may appear where, the workspace and its upload,
 * ownership, streams and errors -- is as in wavepp_attn.h.  A plan made here is a wavepp_plan:
 * wavepp_plan_workspace_bytes, wavepp_plan_get_info, wavepp_plan_get_items, wavepp_attn_plan_upload and
 * wavepp_plan_destroy take it, and the other entry points of wavepp_attn.h, whose pages are of
 * another size, refuse it (WAVEPP_EINVAL), as those below refuse a plan of wavepp_attn_plan.
 *
 * Call order on one stream, per wave: wavepp_q4_plan (host only) -> wavepp_attn_plan_upload ->
 * wavepp_q4_append_kv -> wavepp_q4_chunked_prefill (the last two once per layer, each with its own
 * pools).  The launches of both may be captured into a graph after the upload; its replays run on
 * whatever the buffers then hold.  Calls whose plans have splits write partials into their
 * workspace, so calls that may overlap need a workspace each.
 */
#ifndef WAVEPP_Q4_H
#define WAVEPP_Q4_H

#include "wavepp_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Bytes of one page of one KV head; 0 unless head_dim is 64 or 128 and page_size 16 or 64. */
size_t wavepp_q4_page_bytes(int32_t head_dim, int32_t page_size);

/* wavepp_attn_plan for a 4-bit cache.  Supported: (head_dim_qk, head_dim_v) in {(64, 64), (128, 128)},
 * kv_shared = 0, any num_q_heads % num_kv_heads == 0, page_size in {16, 64}; a latent cache is
 * WAVEPP_EUNSUPPORTED.  Arguments and errors otherwise as there. */
int wavepp_q4_plan(const wavepp_attn_shape* shape, const wavepp_batch* batch, int32_t max_splits, wavepp_plan** out);

/* Quantise the wave's new rows into the pages reserved for them.  Device pointers, contiguous:
 *   k_new [T][num_kv_heads][head_dim], v_new likewise, bf16, 16-byte aligned;
 *   k_pool, v_pool [num_pages][num_kv_heads][wavepp_q4_page_bytes], 16-byte aligned.
 * Only the codes and scales of the wave's new tokens are written.  Errors as for wavepp_attn_append_kv. */
int wavepp_q4_append_kv(const wavepp_plan* plan, const void* k_new, const void* v_new, void* k_pool, void* v_pool,
                        void* workspace, size_t ws_bytes, hipStream_t stream);

/* The way back: the bf16 rows of the wave's new tokens [p_r, p_r + c_r) as the pages hold them, exactly (a scale
 * byte under 8 or over 252, which no append writes, may give zero or infinity).  To read a request's whole
 * cache, plan it with p_r = 0 and c_r its length.  k_out, v_out [T][num_kv_heads][head_dim] bf16, 16-byte aligned. */
int wavepp_q4_read_kv(const wavepp_plan* plan, const void* k_pool, const void* v_pool, void* k_out, void* v_out,
                      void* workspace, size_t ws_bytes, hipStream_t stream);

/* Attention of the wave's queries over the cached values, as defined in wavepp_attn.h with K and V read
 * from 4-bit pages: bf16 q and out, fp32 natural-log lse (or NULL).  bf16 products of the exact cached
 * values with fp32 accumulation and softmax.  A row whose softmax sum is not a number (a NaN in its query, a largest
 * logit that overflows or lies beyond 2^28 ln 2, where fp32 cannot place its exponential) has NaN as its output and
 * its lse, whole or joined from splits.  Logits under -2^28 ln 2 have no weight; an lse of -infinity says that no key
 * had any, and the output then says nothing.
 * Deterministic: repeated calls give bit-identical results.  Errors as for wavepp_attn_chunked_prefill. */
int wavepp_q4_chunked_prefill(const wavepp_plan* plan, const void* q, const void* k_pool, const void* v_pool, void* out,
                              float* lse, void* workspace, size_t ws_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* WAVEPP_Q4_H */
