"""Pins of the linear-attention oracle: closed forms of the recurrence, resume, shared heads."""
import numpy as np
import torch

from oracle import lin
from oracle.attention import bf16_bits_to_f64


def draw(T, H, Hqk, dk, dv, seed):
    rng = np.random.default_rng(seed)

    def bits(*shape):
        x = torch.as_tensor(rng.standard_normal(shape).astype(np.float32)).to(torch.bfloat16)
        return x.view(torch.int16).numpy().view(np.uint16)

    return bits(T, Hqk, dk), bits(T, Hqk, dk), bits(T, H, dv), rng.random((T, H)).astype(np.float32)


def test_without_decay_it_is_causal_linear_attention():
    q, k, v, _ = draw(9, 2, 2, 8, 4, 1)
    o, pool = lin.chunked_prefill(q, k, v, np.ones(2), np.zeros((1, 2, 8, 4)), [9], [-1], [0], 0.5)
    Q, K, V = (bf16_bits_to_f64(x) for x in (q, k, v))
    for h in range(2):
        assert np.abs(o[:, h] - 0.5 * np.tril(Q[:, h] @ K[:, h].T) @ V[:, h]).max() < 1e-12
        assert np.abs(pool[0, h] - K[:, h].T @ V[:, h]).max() < 1e-12


def test_decays_weigh_by_their_products_and_zero_forgets():
    q, k, v, a = draw(7, 1, 1, 4, 4, 2)
    a[3] = 0.0
    S0 = np.random.default_rng(3).standard_normal((1, 1, 4, 4))
    o, pool = lin.chunked_prefill(q, k, v, a, S0, [7], [0], [0], 1.0)
    K, V, Q = (bf16_bits_to_f64(x)[:, 0] for x in (k, v, q))
    for t in range(7):
        S = S0[0, 0] * np.prod(a[:t + 1].astype(np.float64))
        for s in range(t + 1):
            S = S + np.prod(a[s + 1:t + 1].astype(np.float64)) * np.outer(K[s], V[s])
        assert np.abs(o[t, 0] - Q[t] @ S).max() < 1e-12
    again, _ = lin.chunked_prefill(q[3:], k[3:], v[3:], a[3:], np.zeros_like(S0), [4], [-1], [0], 1.0)
    assert np.abs(again - o[3:]).max() < 1e-12


def test_resume_equals_one_run_and_slots_keep():
    q, k, v, a = draw(12, 4, 2, 4, 8, 4)
    pool = np.random.default_rng(5).standard_normal((3, 4, 4, 8))
    o, after = lin.chunked_prefill(q, k, v, a, pool, [12], [1], [2], 1.0)
    o1, p1 = lin.chunked_prefill(q[:5], k[:5], v[:5], a[:5], pool, [5], [1], [0], 1.0)
    o2, p2 = lin.chunked_prefill(q[5:], k[5:], v[5:], a[5:], p1, [7], [0], [2], 1.0)
    assert np.abs(np.concatenate((o1, o2)) - o).max() < 1e-12 and np.abs(p2[2] - after[2]).max() < 1e-12
    assert np.array_equal(after[:2], pool[:2])


def test_shared_heads_equal_repeated_ones():
    q, k, v, a = draw(6, 6, 2, 4, 4, 6)
    pool = np.zeros((1, 6, 4, 4))
    o, _ = lin.chunked_prefill(q, k, v, a, pool, [6], [-1], [0], 1.0)
    o2, _ = lin.chunked_prefill(np.repeat(q, 3, 1), np.repeat(k, 3, 1), v, a, pool, [6], [-1], [0], 1.0)
    assert np.array_equal(o, o2)
    size, _ = lin.sizes(q, k, v, a, pool, [6], [-1], [0], 1.0)
    assert (size >= np.abs(o) - 1e-12).all()
