"""fp64 reference for the 4-bit paged cache: the rounding of rows into codes and scale bytes, the page
layout, and the way back.

TEST INFRASTRUCTURE ONLY (see the package docstring).

The format, from its definition: along the head dim, 32 values share a power-of-two scale 2^(e - 127), e a byte; a
value is one of the magnitudes {0, 1/2, 1, 3/2, 2, 3, 4, 6} with a sign, times the scale.  The scale of a block is
the smallest power of two s with amax <= 7 s (e kept within [8, 252]); a value is rounded to the nearest
magnitude times s, ties to the even code, larger ones to 6 s.  Infinities and NaN count as the largest finite bf16 of
their sign.  Rounding here is a search over all eight magnitudes, and the scale a search over all exponents.

A page of one head: code bytes row by row (value 2i in the low half of byte i), then scale bytes row by row.
"""
from __future__ import annotations

import numpy as np

from .attention import bf16_bits_to_f64

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = 32
LARGEST = bf16_bits_to_f64(np.array([0x7F7F], dtype=np.uint16))[0]


def finite(bits):
    """bf16 bit patterns as fp64, with infinities and NaN as the largest finite number of their sign."""
    bits = np.asarray(bits, dtype=np.uint16)
    with np.errstate(invalid="ignore"):
        x = bf16_bits_to_f64(bits)
    sign = np.where(bits >> 15, -1.0, 1.0)
    return np.where(np.isfinite(x), x, sign * LARGEST)


def quantise(bits):
    """Rows of bf16 bits [..., d] as codes [..., d] (0..15) and scale bytes [..., d / 32]."""
    bits = np.asarray(bits, dtype=np.uint16)
    x = finite(bits).reshape(*bits.shape[:-1], -1, BLOCK)
    amax = np.abs(x).max(axis=-1)
    e = np.full(amax.shape, 252)
    for c in range(251, 7, -1):                                   # the smallest that still holds amax
        e = np.where(amax <= 7.0 * 2.0 ** (c - 127), c, e)
    a = np.abs(x) / np.exp2(e - 127.0)[..., None]
    code = np.zeros(a.shape, dtype=np.uint8)
    near = a.copy()                                                 # distance to magnitude 0
    for c in (2, 4, 6, 1, 3, 5, 7):                                 # even codes first: they keep a tie
        d = np.abs(a - MAGNITUDES[c])
        code = np.where(d < near, np.uint8(c), code)
        near = np.minimum(d, near)
    code = code.reshape(bits.shape) | ((bits >> 15).astype(np.uint8) << 3)
    return code, e.astype(np.uint8)


def values(codes, scales):
    """fp64 values [..., d] of codes [..., d] and scale bytes [..., d / 32]."""
    codes = np.asarray(codes)
    v = np.where(codes & 8, -1.0, 1.0) * MAGNITUDES[codes & 7]
    s = np.exp2(np.asarray(scales, dtype=np.float64) - 127.0)
    return (v.reshape(*codes.shape[:-1], -1, BLOCK) * s[..., None]).reshape(codes.shape)


def page_bytes(head_dim, page_size):
    return page_size * (head_dim // 2 + head_dim // BLOCK)


def split_pool(pool, head_dim, page_size):
    """Pool bytes [P, H, bytes] as codes [P, H, B, d] and scales [P, H, B, d / 32]."""
    pool = np.asarray(pool, dtype=np.uint8)
    n = page_size * head_dim // 2
    b = pool[..., :n].reshape(*pool.shape[:2], page_size, head_dim // 2)
    codes = np.stack((b & 15, b >> 4), axis=-1).reshape(*pool.shape[:2], page_size, head_dim)
    return codes, pool[..., n:].reshape(*pool.shape[:2], page_size, head_dim // BLOCK)


def join_pool(codes, scales):
    P, H = codes.shape[:2]
    b = codes[..., 0::2] | (codes[..., 1::2] << 4)
    return np.concatenate((b.reshape(P, H, -1), scales.reshape(P, H, -1)), axis=-1).astype(np.uint8)


def pool_values(pool, head_dim, page_size):
    """fp64 values [P, H, B, d] of every slot of a pool."""
    return values(*split_pool(pool, head_dim, page_size))


def append(pool, new_bits, prefix_lens, chunk_lens, block_table, head_dim, page_size):
    """A copy of the pool bytes with the wave's new rows [T, H, d] rounded into their pages."""
    codes, scales = split_pool(np.array(pool, copy=True), head_dim, page_size)
    c_new, s_new = quantise(new_bits)
    cu = 0
    for r in range(len(prefix_lens)):
        for i in range(int(chunk_lens[r])):
            pos = int(prefix_lens[r]) + i
            page, slot = int(block_table[r][pos // page_size]), pos % page_size
            codes[page, :, slot] = c_new[cu + i]
            scales[page, :, slot] = s_new[cu + i]
        cu += int(chunk_lens[r])
    return join_pool(codes, scales)


def attention(q_bits, k_values, v_values, prefix_lens, chunk_lens, block_table, page_size, softmax_scale):
    """Causal softmax attention of the wave's queries over fp64 cache values [P, H, B, d].

    Returns (o [T, Hq, d], lse [T, Hq], size [T, Hq, d]) with size the same sums over |V|: what roundings of the
    probabilities scale with.
    """
    q = bf16_bits_to_f64(q_bits)
    T, Hq, d = q.shape
    Hkv = k_values.shape[1]
    G = Hq // Hkv
    o, size, lse = np.zeros(q.shape), np.zeros(q.shape), np.zeros((T, Hq))
    t = 0
    for r in range(len(prefix_lens)):
        p, c = int(prefix_lens[r]), int(chunk_lens[r])
        pos = np.arange(p + c)
        pages = np.asarray(block_table[r], dtype=np.int64)[pos // page_size]
        for h in range(Hq):
            K, V = k_values[pages, h // G, pos % page_size], v_values[pages, h // G, pos % page_size]
            for i in range(c):
                n = p + i + 1
                s = softmax_scale * (K[:n] @ q[t + i, h])
                e = np.exp(s - s.max())
                w = e / e.sum()
                o[t + i, h], size[t + i, h] = w @ V[:n], w @ np.abs(V[:n])
                lse[t + i, h] = s.max() + np.log(e.sum())
        t += c
    return o, lse, size
