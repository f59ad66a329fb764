/*
 * wavepp_lin.h -- C ABI of the linear-attention part of libwavepp_attn.so: layers whose state decays by one
 * factor for each head, for chunks of any length from a single token (decoding) up, resuming from and
 * leaving recurrent-state snapshots, for AMD gfx950 (MI355X).
 *
 * The operation (Preliminaries, "Transformer Architectures", Eq. 1, with the update of such layers): per
 * head, with a decay alpha_t in [0, 1], key k_t, value v_t and query q_t,
 *     S_t = alpha_t S_{t-1} + k_t v_t^T,     o_t = scale S_t^T q_t.
 * alpha_t = 0 forgets the prefix.  Heads may share keys and queries: head h uses those of head
 * h / (num_heads / num_qk_heads).  The decay is given per token and head, or once per head.
 * Resume semantics are those of wavepp_kda.h: request r starts from the snapshot in slot state_in[r] (or from
 * the zero state), runs its c_r tokens and leaves its state in slot state_out[r].
 *
 * Layouts (row-major, contiguous; tokens packed by request in order):
 *   q, k      [T][num_qk_heads][head_dim_k]   bf16
 *   v, out    [T][num_heads][head_dim_v]      bf16
 *   alpha     [T][num_heads] or [num_heads]   fp32
 *   state_pool[num_state_slots][num_heads][head_dim_k][head_dim_v]   fp32
 *
 * Numerics: the state is carried and stored in fp32.  Chunks of at most 10 tokens run token by token
 * in fp32; longer ones in blocks of 64 tokens on bf16 matrix instructions with fp32 accumulation.  What
 * enters the state there, values times decays, keeps its 24 bits as three bf16 parts; the weights inside a
 * block, and the state as the block's queries read it, are rounded to bf16 (2^-8), which is what the bf16
 * outputs are rounded to.  A token's output depends on no later token's numbers, NaN and infinities
 * included; a state that an infinity has entered in a block holds NaN where it did.
 *
 * Call order on one stream, per wave: wavepp_lin_plan (host only) -> wavepp_lin_upload -> wavepp_lin_chunked_prefill
 * (once per layer, each with its own tensors and state pool).  A plan of single tokens that resume in place serves every
 * decoding step of its batch.  The launches may be captured into a graph after the upload.  Plans of long chunks keep
 * partial states in their workspace, so calls that may overlap need a workspace each.
 *
 * Ownership, streams and errors: as in wavepp_kda.h.
 */
#ifndef WAVEPP_LIN_H
#define WAVEPP_LIN_H

#include "wavepp_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Static shape of one layer.  Supported: head_dim_k and head_dim_v each 64 or 128, num_heads a multiple of
 * num_qk_heads, scale finite. */
typedef struct {
  int32_t num_heads;         /* heads of v, alpha, out and the state */
  int32_t num_qk_heads;      /* heads of q and k */
  int32_t head_dim_k;
  int32_t head_dim_v;
  int32_t num_state_slots;   /* slots in the snapshot pool */
  int32_t alpha_per_token;   /* 1: alpha is [T][num_heads]; 0: [num_heads] */
  float scale;
} wavepp_lin_shape;

/* One wave, HOST memory, copied by wavepp_lin_plan; rules for slots as for wavepp_kda_batch. */
typedef struct {
  int32_t num_requests;
  const int32_t* chunk_lens;
  const int32_t* state_in;
  const int32_t* state_out;
} wavepp_lin_batch;

typedef struct wavepp_lin_plan_s wavepp_lin_plan_t;

typedef struct {
  int64_t total_tokens;      /* T */
  int32_t num_step_items;    /* requests that run token by token */
  int32_t num_segments;      /* pieces that the other requests' chunks are cut into */
  int32_t num_partials;      /* partial states in the workspace, per head */
  int32_t block_tokens;      /* 64 */
  int64_t metadata_bytes;
  int64_t workspace_bytes;
} wavepp_lin_info;

/* Validate the wave and build its work list; where it has fewer chains (request, head) than the chip has room
 * for, or a chunk so long that it would run on after the others, long chunks are cut into segments: each segment's own
 * state first, then the states between them, then all outputs at once.  Host only.  Errors as for wavepp_kda_plan. */
int wavepp_lin_plan(const wavepp_lin_shape* shape, const wavepp_lin_batch* batch, wavepp_lin_plan_t** out);

/* Device workspace the plan needs (metadata and partial states), 256-byte aligned. */
size_t wavepp_lin_workspace_bytes(const wavepp_lin_plan_t* plan);

int wavepp_lin_get_info(const wavepp_lin_plan_t* plan, wavepp_lin_info* info);

/* As wavepp_kda_upload. */
int wavepp_lin_upload(const wavepp_lin_plan_t* plan, void* workspace, size_t ws_bytes, hipStream_t stream);

/* One layer of the wave.  Device pointers with the layouts above, 16-byte aligned (alpha 4-byte).  Reads the
 * snapshots named by state_in and writes out and the snapshots named by state_out; every other slot and byte is
 * left untouched.  Requires that the last upload into `workspace` was of `plan` (else WAVEPP_EINVAL, nothing
 * enqueued).  Deterministic: repeated calls on the same inputs give bit-identical results. */
int wavepp_lin_chunked_prefill(const wavepp_lin_plan_t* plan, const void* q, const void* k, const void* v,
                               const float* alpha, float* state_pool, void* out, void* workspace, size_t ws_bytes,
                               hipStream_t stream);

void wavepp_lin_destroy(wavepp_lin_plan_t* plan);

#ifdef __cplusplus
}
#endif

#endif /* WAVEPP_LIN_H */
