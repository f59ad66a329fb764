"""Pins of the 4-bit cache's oracle: hand-made blocks, the definition's inequalities, and the page layout."""
import numpy as np
import pytest
import torch

from oracle import q4


def bits(x):
    return torch.as_tensor(np.asarray(x, dtype=np.float32)).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)


def block(*first):
    return np.array(list(first) + [0.0] * (32 - len(first)))


def test_ties_go_to_the_even_code_and_large_values_to_six():
    # amax 7 with scale 1: 7 is a step over 6 and saturates; the others are halfway between two magnitudes
    x = block(7.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -5.0, 6.5)
    codes, e = q4.quantise(bits(x))
    assert e.tolist() == [127]
    got = q4.values(codes, e)[:11]
    assert got.tolist() == [6.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, -0.0, -4.0, 6.0]
    assert codes[8] == 8                                    # the sign of what rounds to zero is kept


@pytest.mark.parametrize("amax,e", [(7.0, 127), (7.03125, 128), (3.5, 126), (3.515625, 127), (4.0, 127), (1.0, 125)])
def test_scale_is_the_smallest_that_holds_the_block(amax, e):
    assert q4.quantise(bits(block(amax)))[1].tolist() == [e]


def test_extremes():
    zero, e = q4.quantise(bits(block()))
    assert not zero.any() and e.tolist() == [8]
    big = np.array([0x7F80, 0xFF80, 0x7FC1, 0xFFFF, 0x7F7F, 0x3F80] + [0] * 26, dtype=np.uint16)   # inf, NaN, largest, 1
    codes, e = q4.quantise(big)
    assert e.tolist() == [252]
    assert q4.values(codes, e)[:6].tolist() == [6 * 2.0 ** 125, -6 * 2.0 ** 125, 6 * 2.0 ** 125, -6 * 2.0 ** 125,
                                                 6 * 2.0 ** 125, 0.0]
    tiny, e = q4.quantise(bits(block(2.0 ** -120)))
    assert e.tolist() == [8] and q4.values(tiny, e)[0] == 2.0 ** -120       # half of 2^-119


def test_no_value_is_off_by_more_than_the_scale_and_rounding_twice_changes_nothing():
    rng = np.random.default_rng(3)
    x = bits(rng.standard_normal((200, 128)) * np.exp2(rng.integers(-20, 20, (200, 1))))
    codes, e = q4.quantise(x)
    v = q4.values(codes, e)
    s = np.repeat(np.exp2(e - 127.0), 32, axis=-1)
    assert (np.abs(v - q4.finite(x)) <= s).all()
    small = np.abs(q4.finite(x)) <= 2 * s
    assert (np.abs(v - q4.finite(x))[small] <= 0.25 * s[small]).all()
    again, e2 = q4.quantise(bits(v))
    assert np.array_equal(q4.values(again, e2), v)


@pytest.mark.parametrize("dim,page", [(64, 16), (128, 64)])
def test_page_layout(dim, page):
    rng = np.random.default_rng(5)
    codes = rng.integers(0, 16, (3, 2, page, dim)).astype(np.uint8)
    scales = rng.integers(8, 253, (3, 2, page, dim // 32)).astype(np.uint8)
    pool = q4.join_pool(codes, scales)
    assert pool.shape == (3, 2, q4.page_bytes(dim, page))
    c, s = q4.split_pool(pool, dim, page)
    assert np.array_equal(c, codes) and np.array_equal(s, scales)
    # value 5 of row 7: the high half of byte 2 of that row; its scale byte is the row's first
    assert pool[2, 1, 7 * dim // 2 + 2] >> 4 == codes[2, 1, 7, 5]
    assert pool[2, 1, page * dim // 2 + 7 * dim // 32] == scales[2, 1, 7, 0]


def test_append_touches_only_the_new_slots():
    rng = np.random.default_rng(6)
    pool = rng.integers(0, 256, (6, 2, q4.page_bytes(64, 16))).astype(np.uint8)
    new = bits(rng.standard_normal((5, 2, 64)))
    table = np.array([[4, 1], [5, 0]])
    after = q4.append(pool, new, [14, 3], [4, 1], table, 64, 16)
    codes, scales = q4.split_pool(after, 64, 16)
    want = q4.quantise(new)
    for t, (page, slot) in enumerate([(4, 14), (4, 15), (1, 0), (1, 1), (5, 3)]):
        assert np.array_equal(codes[page, :, slot], want[0][t]) and np.array_equal(scales[page, :, slot], want[1][t])
    before = q4.split_pool(pool, 64, 16)
    keep = np.ones((6, 16), dtype=bool)
    keep[[4, 4, 1, 1, 5], [14, 15, 0, 1, 3]] = False
    assert np.array_equal(codes.transpose(0, 2, 1, 3)[keep], before[0].transpose(0, 2, 1, 3)[keep])
    assert np.array_equal(scales.transpose(0, 2, 1, 3)[keep], before[1].transpose(0, 2, 1, 3)[keep])


def test_attention_is_softmax_over_the_visible_values():
    rng = np.random.default_rng(7)
    k, v = rng.standard_normal((4, 1, 16, 64)), rng.standard_normal((4, 1, 16, 64))
    q = bits(rng.standard_normal((3, 2, 64)))
    o, lse, size = q4.attention(q, k, v, [17], [3], [[2, 0, 3]], 16, 0.125)
    K = torch.as_tensor(np.concatenate((k[2, 0], k[0, 0])))[:20]
    V = torch.as_tensor(np.concatenate((v[2, 0], v[0, 0])))[:20]
    Q = torch.as_tensor(q.view(np.int16)).view(torch.bfloat16).double()
    mask = torch.arange(20)[None, :] <= 17 + torch.arange(3)[:, None]
    for h in range(2):
        want = torch.nn.functional.scaled_dot_product_attention(Q[:, h], K, V, attn_mask=mask, scale=0.125)
        assert np.abs(o[:, h] - want.numpy()).max() < 1e-12
        s = torch.where(mask, 0.125 * Q[:, h] @ K.T, -torch.inf)
        assert np.abs(lse[:, h] - torch.logsumexp(s, -1).numpy()).max() < 1e-12
    assert (size >= np.abs(o)).all()
