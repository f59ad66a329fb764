"""fp64 reference for the 8-bit paged cache: the rounding of blocks of rows into codes and scale bytes, the page layout,
the way back, and attention with other scores than the causal ones.

TEST INFRASTRUCTURE ONLY (see the package docstring).

The format, from its definition: 16 slots of a page share a power-of-two scale 2^(e - 127) for each head, e a byte; a value
is an e4m3 number (sign, four bits of exponent of bias 7, three of mantissa, the largest exponent with the largest mantissa
is not a number) times the scale.  The scale of a block is the smallest power of two s with amax <= 448 s over the new
values, e at least 8, and no smaller than the block's if it holds earlier tokens, which are then rounded again.  A value is
rounded to the nearest number of the grid, ties to the even code; larger magnitudes than 1.75 * 2^127, infinities and NaN
count as that.  Rounding here is a search among the 127 magnitudes, and the scale a search over all exponents.

A page of one head: code bytes row by row, then 16 bytes, the first of which are the blocks' exponents.
"""
from __future__ import annotations

import numpy as np

from .attention import bf16_bits_to_f64

BLOCK = 16
SCALE_BYTES = 16
LARGEST = 1.75 * 2.0 ** 127


def _magnitude(code):
    e, m = code >> 3, code & 7
    return m / 8.0 * 2.0 ** -6 if e == 0 else (1.0 + m / 8.0) * 2.0 ** (e - 7)


MAGNITUDES = np.array([_magnitude(c) for c in range(127)])


def finite(bits):
    """bf16 bit patterns as fp64, with infinities, NaN and all magnitudes over LARGEST as LARGEST of their sign."""
    bits = np.asarray(bits, dtype=np.uint16)
    with np.errstate(invalid="ignore"):
        x = bf16_bits_to_f64(bits)
    sign = np.where(bits >> 15, -1.0, 1.0)
    return np.where(np.abs(x) <= LARGEST, x, sign * LARGEST)


def needed(amax):
    """Exponent bytes of the smallest scales that hold magnitudes of `amax`."""
    e = np.full(np.shape(amax), 246)
    for c in range(245, 7, -1):
        e = np.where(amax <= 448.0 * 2.0 ** (c - 127), c, e)
    return e


def round_codes(x, e):
    """Codes of fp64 values x, which may have a negative zero, with exponent bytes e that broadcast against them."""
    a = np.abs(x) / np.exp2(np.asarray(e, dtype=np.float64) - 127.0)
    above = np.clip(np.searchsorted(MAGNITUDES, a), 1, 126)
    below = above - 1
    d_lo, d_hi = a - MAGNITUDES[below], MAGNITUDES[above] - a
    up = (d_hi < d_lo) | ((d_hi == d_lo) & (above % 2 == 0))
    return (np.where(up, above, below) | (np.signbit(x).astype(np.int64) << 7)).astype(np.uint8)


def values(codes, e):
    """fp64 values of codes with exponent bytes that broadcast against them."""
    codes = np.asarray(codes)
    v = np.append(MAGNITUDES, np.nan)[codes & 127]
    return np.where(codes & 128, -v, v) * np.exp2(np.asarray(e, dtype=np.float64) - 127.0)


def page_bytes(head_dim, page_size):
    return page_size * head_dim + SCALE_BYTES


def split_pool(pool, head_dim, page_size):
    """Pool bytes [P, H, bytes] as codes [P, H, B, d], exponent bytes [P, H, B / 16] and padding."""
    pool = np.asarray(pool, dtype=np.uint8)
    n = page_size * head_dim
    return (pool[..., :n].reshape(*pool.shape[:2], page_size, head_dim), pool[..., n:n + page_size // BLOCK],
            pool[..., n + page_size // BLOCK:])


def join_pool(codes, e, padding=None):
    P, H, B, _ = codes.shape
    if padding is None:
        padding = np.zeros((P, H, SCALE_BYTES - B // BLOCK), dtype=np.uint8)
    return np.concatenate((codes.reshape(P, H, -1), e, padding), axis=-1).astype(np.uint8)


def quantise_pool(x):
    """Pool bytes of fp64 rows [P, H, B, d]."""
    P, H, B, d = x.shape
    blocks = x.reshape(P, H, B // BLOCK, BLOCK * d)
    e = needed(np.abs(blocks).max(-1))
    return join_pool(round_codes(blocks, e[..., None]).reshape(x.shape), e.astype(np.uint8))


def pool_values(pool, head_dim, page_size):
    """fp64 values [P, H, B, d] of every slot of a pool."""
    codes, e, _ = split_pool(pool, head_dim, page_size)
    return values(codes, np.repeat(e, BLOCK, axis=-1)[..., None])


def append(pool, new_bits, prefix_lens, chunk_lens, block_table, head_dim, page_size):
    """A copy of the pool bytes with the wave's new rows [T, H, d] rounded into their pages."""
    codes, e, padding = (np.array(a, copy=True) for a in split_pool(pool, head_dim, page_size))
    new = finite(new_bits)
    cu = 0
    for p, c, row in zip(prefix_lens, chunk_lens, block_table):
        p, c = int(p), int(c)
        for start in range(p // BLOCK * BLOCK, p + c, BLOCK):
            if c == 0:
                break
            page, slot = int(row[start // page_size]), start % page_size
            old = max(p - start, 0)
            end = min(p + c - start, BLOCK)
            rows = new[cu + start + old - p:cu + start + end - p].transpose(1, 0, 2)          # [H, n, d]
            scale = needed(np.abs(rows).max((1, 2)))
            if old:
                was = e[page, :, slot // BLOCK].astype(np.int64)
                scale = np.maximum(scale, was)
                held = values(codes[page, :, slot:slot + old], was[:, None, None])
                codes[page, :, slot:slot + old] = round_codes(held, scale[:, None, None])
            codes[page, :, slot + old:slot + end] = round_codes(rows, scale[:, None, None])
            e[page, :, slot // BLOCK] = scale
        cu += c
    return join_pool(codes, e, padding)


def attention(q_bits, k_values, v_values, prefix_lens, chunk_lens, block_table, page_size, softmax_scale, cap=0.0,
              slopes=None, key_begin=None, key_end=None):
    """Softmax attention of the wave's queries over fp64 cache values [P, H, B, d], one query and head after another.

    Returns (o [T, Hq, d], lse [T, Hq], size [T, Hq, d]) with size the same sums over |V|: what roundings of the
    probabilities scale with.
    """
    q = bf16_bits_to_f64(q_bits)
    T, Hq, d = q.shape
    G = Hq // k_values.shape[1]
    o, size, lse = np.zeros(q.shape), np.zeros(q.shape), np.full((T, Hq), -np.inf)
    t = 0
    for r in range(len(prefix_lens)):
        p, c = int(prefix_lens[r]), int(chunk_lens[r])
        pos = np.arange(p + c)
        pages = np.asarray(block_table[r], dtype=np.int64)[pos // page_size]
        for h in range(Hq):
            K, V = k_values[pages, h // G, pos % page_size], v_values[pages, h // G, pos % page_size]
            for i in range(c):
                a = 0 if key_begin is None else int(key_begin[t + i])
                b = p + i + 1 if key_end is None else int(key_end[t + i])
                if a >= b:
                    continue
                s = softmax_scale * (K[a:b] @ q[t + i, h])
                if cap:
                    s = cap * np.tanh(s / cap)
                if slopes is not None:
                    s = s - float(slopes[h]) * np.abs(p + i - pos[a:b])
                e = np.exp(s - s.max())
                w = e / e.sum()
                o[t + i, h], size[t + i, h] = w @ V[a:b], w @ np.abs(V[a:b])
                lse[t + i, h] = s.max() + np.log(e.sum())
        t += c
    return o, lse, size
