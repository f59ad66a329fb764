/*
 * wavepp_rope.h -- C ABI of the rotary positions of libwavepp_attn.so: the query and key rows of a wave's new tokens are
 * turned by their positions, before wavepp_*_append_kv and wavepp_*_chunked_prefill, whatever cache the wave's plan is of
 * (bf16, latent, 4-bit or 8-bit), for AMD gfx950 (MI355X).
 *
 * With n = rot_dim / 2 pairs a head, pair i of the row of a token at position t becomes
 *     (a, b) -> magnitude (a cos(t f_i) - b sin(t f_i), a sin(t f_i) + b cos(t f_i)),
 * a and b being the head's values
 *     rot_offset + i and rot_offset + n + i        (interleaved = 0: halves), or
 *     rot_offset + 2 i and rot_offset + 2 i + 1    (interleaved = 1: pairs),
 * and the head's other values stay.  Products and sums are in fp32 and rounded to bf16 once.  The angle t f_i is taken in
 * fp64 and brought into one turn there, so at any position it is off by no more than 2^-52 of itself and 2^-22.
 *
 * Frequencies, in radians a token: f_i = base^(-2 i / rot_dim), or, for contexts longer than the trained original_length,
 * with scaling
 *     WAVEPP_ROPE_LINEAR  f_i / factor;
 *     WAVEPP_ROPE_TURNS   w f_i + (1 - w) f_i / factor with w growing from 0 to 1 with the turns that the pair makes in
 *                         original_length, u_i = original_length f_i / 2 pi: w = (u_i - slow_turns) / (fast_turns -
 *                         slow_turns), kept within [0, 1];
 *     WAVEPP_ROPE_INDEX   the same with w falling from 1 to 0 with the pair's index: w = 1 - (i - lo) / (hi - lo), kept
 *                         within [0, 1], lo = max(0, floor(at(fast_turns))), hi = min(rot_dim - 1, ceil(at(slow_turns))),
 *                         at(u) = rot_dim ln(original_length / 2 pi u) / (2 ln base); hi - lo is taken as 0.001 at least;
 * or the caller's own.  No frequency may lie outside [-1e30, 1e30].
 */
#ifndef WAVEPP_ROPE_H
#define WAVEPP_ROPE_H

#include "wavepp_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  WAVEPP_ROPE_PLAIN = 0,
  WAVEPP_ROPE_LINEAR = 1,
  WAVEPP_ROPE_TURNS = 2,
  WAVEPP_ROPE_INDEX = 3
} wavepp_rope_scaling;

typedef struct {
  int32_t rot_dim;               /* even, 2 to 256 */
  int32_t rot_offset;            /* >= 0 */
  int32_t interleaved;           /* 0 or 1 */
  int32_t scaling;               /* a wavepp_rope_scaling */
  double base;                   /* over 1 */
  double factor;                 /* over 0; read unless PLAIN */
  double original_length;        /* over 0; read by TURNS and INDEX, as are the next two */
  double slow_turns, fast_turns; /* 0 < slow_turns < fast_turns */
  double magnitude;              /* over 0 */
  const double* frequencies;     /* NULL, or rot_dim / 2 numbers (HOST, copied) in place of base and scaling */
} wavepp_rope_spec;

typedef struct wavepp_rope wavepp_rope;

/* Check the spec and take its frequencies.  Host only.  On error (WAVEPP_EINVAL; WAVEPP_EUNSUPPORTED for a rot_dim over
 * 256) *out is NULL.  The object is read only afterwards, so any number of calls and threads may share it. */
int wavepp_rope_create(const wavepp_rope_spec* spec, wavepp_rope** out);

/* The frequencies in use: writes min(capacity, rot_dim / 2) of them and returns that number, or a negative status. */
int wavepp_rope_frequencies(const wavepp_rope* rope, double* out, int32_t capacity);

/* Turn the rows of the plan's new tokens.  Device pointers, bf16, 16-byte aligned, rows of a token contiguous:
 *   q, q_out [T][num_q_heads][head_dim_qk], k, k_out [T][num_kv_heads][head_dim_qk];
 * either pair may be NULL as a whole.  A stride is the number of elements from one token to the next: a multiple of 8, at
 * least a token's row and at most 2^30.  So q and k may be slices of one packed projection.  An output is the input itself
 * (same address and stride: in place) or shares no element with any other buffer of the call, the positions and what the
 * workspace holds of the plan among them (else WAVEPP_EALIAS).  A token's position is p_r + i, or positions[its packed index] (device, int32, 4-byte aligned, any value) where positions is not
 * NULL.  rot_offset + rot_dim must not exceed the plan's head_dim_qk.  The workspace holds the plan's upload, as for the
 * other entry points, and is only read.  One launch; it may be captured.  The rope may be destroyed once this returned.
 * A wave of 2^24 tokens or more is WAVEPP_EUNSUPPORTED.
 * Errors: WAVEPP_EINVAL, WAVEPP_EUNSUPPORTED, WAVEPP_EALIAS, WAVEPP_ENOSPACE, WAVEPP_EHIP.  A wave with T = 0 is a no-op. */
int wavepp_rope_apply(const wavepp_rope* rope, const wavepp_plan* plan, const void* q, int64_t q_stride, const void* k,
                      int64_t k_stride, void* q_out, int64_t q_out_stride, void* k_out, int64_t k_out_stride,
                      const int32_t* positions, void* workspace, size_t ws_bytes, hipStream_t stream);

void wavepp_rope_destroy(wavepp_rope* rope);

#ifdef __cplusplus
}
#endif

#endif /* WAVEPP_ROPE_H */
