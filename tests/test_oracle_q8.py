"""Pins of the 8-bit cache's oracle: hand-made blocks, the definition's inequalities, the page layout and the scores."""
import numpy as np
import pytest
import torch

from oracle import bf16_bits_to_f64, q4, q8, rope


def bits(x):
    return torch.as_tensor(np.asarray(x, dtype=np.float32)).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)


def store(rows, prefix=0, pool=None, d=64, page=16):
    rows = np.asarray(rows, dtype=np.float64)
    x = np.zeros((len(rows), 1, d))
    x[:, 0, :rows.shape[1]] = rows
    pool = np.zeros((1, 1, q8.page_bytes(d, page)), np.uint8) if pool is None else pool
    return q8.append(pool, bits(x), [prefix], [len(rows)], [[0]], d, page)


def test_the_grid_is_torchs_e4m3():
    every = torch.arange(256, dtype=torch.uint8)
    want = every.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(q8.values(every.numpy(), np.int64(127)), want, equal_nan=True)


def test_rounding_is_torchs_over_many_values():
    rng = np.random.default_rng(0)
    x = np.clip(rng.standard_normal(50000) * np.exp2(rng.integers(-14, 9, 50000)), -448, 448).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(q8.round_codes(x.astype(np.float64), np.int64(127)), want)


def test_ties_go_to_the_even_code():
    x = np.array([1.0625, 1.1875, -1.0625, 2.0 ** -10, 3 * 2.0 ** -10, -2.0 ** -10, 432.0, 416.0, 0.0, -0.0])
    v = q8.values(q8.round_codes(x, np.int64(127)), np.int64(127))
    assert v.tolist() == [1.0, 1.25, -1.0, 0.0, 2.0 ** -8, 0.0, 448.0, 416.0, 0.0, 0.0]
    assert np.signbit(v).tolist() == [False, False, True, False, False, True, False, False, False, True]


@pytest.mark.parametrize("amax,e", [(448.0, 127), (450.0, 128), (224.0, 126), (1.75, 119), (1.7578125, 120), (1.0, 119), (0.0, 8)])
def test_scale_is_the_smallest_that_holds_the_block(amax, e):
    assert store([[amax, 0.001 * amax]])[0, 0, 16 * 64] == e


def test_extremes():
    x = np.zeros((1, 1, 64), dtype=np.uint16)
    x[0, 0, :6] = [0x7F80, 0xFF80, 0x7FC1, 0xFFFF, 0x7F7F, 0x3F80]            # infinities, NaN, the largest, 1
    pool = q8.append(np.zeros((1, 1, q8.page_bytes(64, 16)), np.uint8), x, [0], [1], [[0]], 64, 16)
    assert pool[0, 0, 16 * 64] == 246
    big = 1.75 * 2.0 ** 127
    assert q8.pool_values(pool, 64, 16)[0, 0, 0, :6].tolist() == [big, -big, big, -big, big, 0.0]


def test_a_block_grows_its_scale_and_rounds_what_it_holds_again():
    pool = store([[1.0, 2.0 ** -9, 1.125]])
    assert pool[0, 0, 16 * 64] == 119
    pool = store([[300.0]], 1, pool)                                           # needs 2^0: the small value falls to a step of 2^-9
    assert pool[0, 0, 16 * 64] == 127
    assert q8.pool_values(pool, 64, 16)[0, 0, :2, :3].tolist() == [[1.0, 2.0 ** -9, 1.125], [288.0, 0.0, 0.0]]
    pool = store([[448.0 * 64]], 2, pool)
    assert q8.pool_values(pool, 64, 16)[0, 0, :3, :3].tolist() == [[1.0, 0.0, 1.125], [288.0, 0.0, 0.0], [448.0 * 64, 0, 0]]
    pool = store([[1.0]], 3, pool)                                             # and does not shrink it
    assert pool[0, 0, 16 * 64] == 133
    again = store([[5.0]], 0, pool)                                            # a block begun anew forgets it
    assert again[0, 0, 16 * 64] == 121


def test_error_of_a_block_and_appends_in_pieces():
    rng = np.random.default_rng(1)
    x = bits(rng.standard_normal((16, 1, 64)) * np.exp2(rng.integers(-6, 6, (16, 1, 1))))
    zero = np.zeros((1, 1, q8.page_bytes(64, 16)), np.uint8)
    whole = q8.append(zero, x, [0], [16], [[0]], 64, 16)
    v, f = q8.pool_values(whole, 64, 16)[0, 0], bf16_bits_to_f64(x)[:, 0]
    s = 2.0 ** (whole[0, 0, 16 * 64] - 127.0)
    assert (np.abs(v - f) <= np.maximum(2.0 ** -4 * np.abs(f), 2.0 ** -10 * s)).all()
    parts = zero
    for i in range(16):
        parts = q8.append(parts, x[i:i + 1], [i], [1], [[0]], 64, 16)
    w = q8.pool_values(parts, 64, 16)[0, 0]
    assert parts[0, 0, 16 * 64] == whole[0, 0, 16 * 64] and (np.abs(w - v) <= 2.0 ** -9 * s).all()
    normal = np.abs(f) >= 2.0 ** -6 * s
    assert np.array_equal(w[normal], v[normal])


@pytest.mark.parametrize("dim,page", [(64, 16), (128, 64)])
def test_page_layout(dim, page):
    rng = np.random.default_rng(5)
    pool = rng.integers(0, 256, (3, 2, q8.page_bytes(dim, page))).astype(np.uint8)
    codes, e, padding = q8.split_pool(pool, dim, page)
    assert np.array_equal(q8.join_pool(codes, e, padding), pool)
    assert codes[1, 1, 5, 7] == pool[1, 1, 5 * dim + 7] and e[2, 0, page // 16 - 1] == pool[2, 0, page * dim + page // 16 - 1]


def wave(rng, Hq=4, Hkv=2, d=8, page=16):
    prefix, chunk = [20, 0], [3, 5]
    bt = np.array([[2, 0], [1, -1]])
    q = bits(rng.standard_normal((8, Hq, d)))
    k, v = (rng.standard_normal((3, Hkv, page, d)) for _ in range(2))
    return q, k, v, prefix, chunk, bt, page, 0.4


def test_scores_that_change_nothing_are_the_causal_attention():
    a = wave(np.random.default_rng(6))
    o, lse, size = q4.attention(*a)
    pos = np.concatenate([20 + np.arange(3), np.arange(5)])
    for s in ({}, {"cap": 1e6}, {"slopes": np.zeros(4)}, {"key_begin": pos * 0, "key_end": pos + 1}):
        o2, lse2, size2 = q8.attention(*a, **s)
        assert np.allclose(o, o2, atol=1e-9) and np.allclose(lse, lse2, atol=1e-9) and np.allclose(size, size2, atol=1e-9)


def test_scores_by_hand():
    q, k, v, prefix, chunk, bt, page, scale = wave(np.random.default_rng(7))
    lo, hi = np.array([5, 5, 30, 0, 0, 1, 4, 2]), np.array([23, 4, 23, 1, 5, 5, 5, 3])
    hi[2], lo[2] = 23, 22
    slopes = np.array([0.5, -0.25, 0.0, 1.0])
    o, lse, _ = q8.attention(q, k, v, prefix, chunk, bt, page, scale, cap=1.5, slopes=slopes, key_begin=lo, key_end=hi)
    assert (o[1] == 0).all() and np.isneginf(lse[1]).all()
    x = bf16_bits_to_f64(q)
    for t, (r, i) in enumerate([(0, 20), (0, 21), (0, 22), (1, 0), (1, 1), (1, 2), (1, 3), (1, 4)]):
        for h in range(4):
            w, total = 0.0, 0.0
            for j in range(lo[t], hi[t]):
                K, V = (a[bt[r][j // page], h // 2, j % page] for a in (k, v))
                s = 1.5 * np.tanh(scale * float(K @ x[t, h]) / 1.5) - slopes[h] * abs(i - j)
                w, total = w + np.exp(s) * V, total + np.exp(s)
            if total:
                assert np.allclose(o[t, h], w / total) and np.isclose(lse[t, h], np.log(total))


def test_turning_keeps_lengths_and_makes_products_relative():
    rng = np.random.default_rng(8)
    f = rope.frequencies(16)
    assert f[0] == 1.0 and np.isclose(f[4], 0.01)
    for interleaved in (False, True):
        a, b = rng.standard_normal((2, 40, 1, 24))
        a[:], b[:] = a[:1], b[:1]
        pos = np.arange(40)
        x, y = rope.turn(a, pos, f, 8, interleaved), rope.turn(b, pos + 11, f, 8, interleaved)
        assert np.allclose((x * y).sum(-1), (x * y).sum(-1)[0]) and np.allclose((x ** 2).sum(-1), (a ** 2).sum(-1))
        assert np.array_equal(x[..., :8], a[..., :8]) and np.array_equal(x[0], a[0])
    one = rope.turn(np.array([[[1.0, 0.0, 5.0, 6.0]]]), [np.pi / 2], np.array([1.0]), 0, True)
    assert np.allclose(one, [[[0.0, 1.0, 5.0, 6.0]]])
    one = rope.turn(np.array([[[1.0, 9.0, 0.0, 6.0]]]), [np.pi / 2], np.array([1.0, 0.0]), 0, False, 2.0)
    assert np.allclose(one, [[[0.0, 18.0, 2.0, 12.0]]])


def test_frequencies_of_the_scalings():
    f = rope.frequencies(8, 1e4)
    assert np.allclose(rope.frequencies(8, 1e4, "linear", 4.0), f / 4)
    kw = dict(factor=8.0, original_length=2 * np.pi * 100, slow_turns=1.0, fast_turns=10.0)
    # turns of the pairs: 100, 10, 1, 0.1
    assert np.allclose(rope.frequencies(8, 1e4, "turns", **kw), [1.0, 0.1, 0.01 / 8, 0.001 / 8])
    # index 1 at 10 turns, 2 at 1 turn
    assert np.allclose(rope.frequencies(8, 1e4, "index", **kw), [1.0, 0.1, 0.01 / 8, 0.001 / 8])
    mid = rope.frequencies(8, 1e4, "turns", **{**kw, "fast_turns": 19.0})
    assert np.isclose(mid[1], 0.1 * (0.5 + 0.5 / 8))
