"""fp64 reference for linear attention with a decay for each head, with resume from and snapshot to state slots.

TEST INFRASTRUCTURE ONLY (see the package docstring).

Per head (Preliminaries, "Transformer Architectures", Eq. 1: a state of fixed size, updated by a linear map plus an
additive term and read after the update):

    S_t = alpha_t S_{t-1} + k_t v_t^T,    o_t = scale S_t^T q_t,

with alpha_t a number in [0, 1] per token and head or per head, and head h using the queries and keys of head
h // (H / Hqk).  Token by token, exactly as written.  q, k, v are bf16 bit patterns, alpha and states fp32.
"""
from __future__ import annotations

import numpy as np

from .attention import bf16_bits_to_f64


def token(S, q, k, v, alpha, scale):
    """One token of all heads: S [H, d_k, d_v]; q, k [H, d_k]; v [H, d_v]; alpha [H]."""
    S = alpha[:, None, None] * S + k[:, :, None] * v[:, None, :]
    return S, scale * np.einsum("hij,hi->hj", S, q)


def chunked_prefill(q, k, v, alpha, state_pool, chunk_lens, state_in, state_out, scale):
    """One wave: (o [T, H, d_v] fp64, the pool after it [slots, H, d_k, d_v] fp64)."""
    q, k, v = (bf16_bits_to_f64(x) for x in (q, k, v))
    T, H, dv = v.shape
    G = H // q.shape[1]
    q, k = np.repeat(q, G, axis=1), np.repeat(k, G, axis=1)
    alpha = np.broadcast_to(np.asarray(alpha, dtype=np.float64), (T, H))
    before = np.asarray(state_pool, dtype=np.float64)
    after = before.copy()
    o = np.zeros((T, H, dv))
    t = 0
    for r, c in enumerate(np.asarray(chunk_lens).tolist()):
        if c == 0:
            continue
        S = before[state_in[r]].copy() if state_in[r] >= 0 else np.zeros(before.shape[1:])
        for _ in range(c):
            S, o[t] = token(S, q[t], k[t], v[t], alpha[t], scale)
            t += 1
        after[state_out[r]] = S
    return o, after


def sizes(q, k, v, alpha, state_pool, chunk_lens, state_in, state_out, scale):
    """The same recurrence over absolute values: what roundings of its terms scale with."""
    a = [np.asarray(x, dtype=np.uint16) & np.uint16(0x7FFF) for x in (q, k, v)]
    return chunked_prefill(*a, alpha, np.abs(np.asarray(state_pool, dtype=np.float64)), chunk_lens, state_in, state_out, abs(scale))
