"""The 4-bit cache and linear attention where byte offsets pass 32 bits: pools, states and token rows of more than 4 GiB.

The last requests of a large wave are compared bit for bit with the same requests alone, in small buffers.
"""
import numpy as np
import pytest
import torch

import paper_2609_35263_amd as wp

pytestmark = pytest.mark.gpu


def test_q4_pools_and_token_rows():
    Hq, Hkv, dim, page, pages = 64, 8, 128, 64, 130_000
    requests, prefix, chunk = 2050, 40, 128                      # 262,400 tokens of 16 KiB; three pages each
    need = (prefix + chunk + page - 1) // page
    table = (pages - 1 - np.arange(requests * need)).reshape(requests, need)[::-1].astype(np.int32)
    assert pages * Hkv * wp.q4_page_bytes(dim, page) > 1 << 32 and requests * chunk * Hq * dim * 2 > 1 << 32
    g = torch.Generator(device="cuda").manual_seed(1)

    def rows(*shape):
        return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=g)

    def wave(n, num_pages, bt):
        p = wp.q4_plan(num_q_heads=Hq, num_kv_heads=Hkv, head_dim_qk=dim, head_dim_v=dim, page_size=page, num_pages=num_pages,
                       softmax_scale=dim ** -0.5, prefix_lens=[prefix] * n, chunk_lens=[chunk] * n, block_table=bt, max_splits=1)
        ws = wp.new_workspace(p)
        wp.plan_upload(p, ws)
        return p, ws

    def run(p, ws, q, k_new, v_new, k_pool, v_pool):
        out, lse = torch.full_like(q, float("nan")), torch.empty(q.shape[:2], device="cuda")
        back = torch.empty_like(k_new), torch.empty_like(v_new)
        wp.q4_append_kv(p, k_new, v_new, k_pool, v_pool, ws)
        wp.q4_chunked_prefill(p, q, k_pool, v_pool, out, lse, ws)
        wp.q4_read_kv(p, k_pool, v_pool, *back, ws)
        return out, lse, *back

    T = requests * chunk
    q, k_new, v_new = rows(T, Hq, dim), rows(T, Hkv, dim), rows(T, Hkv, dim)
    pools = [wp.q4_new_pool(pages, Hkv, dim, page) for _ in range(2)]
    for x in pools:                                                # codes anyhow, scales of ones; only those of used pages
        used = x[pages - requests * need:]
        used[..., :page * dim // 2].random_(0, 256, generator=g)
        used[..., page * dim // 2:] = 127
    for r in (0, requests - 1):
        at = slice(r * chunk, (r + 1) * chunk)
        small = [x[torch.from_numpy(table[r].astype(np.int64)).cuda()].clone() for x in pools]
        alone = wave(1, need, np.arange(need, dtype=np.int32)[None])
        one = run(*alone, q[at].clone(), k_new[at].clone(), v_new[at].clone(), *small)
        if r == 0:
            first = one
    both = run(*wave(requests, pages, table), q, k_new, v_new, *pools)
    torch.cuda.synchronize()
    for a, b, c in zip(both, first, one):
        assert torch.equal(a[:chunk], b) and torch.equal(a[-chunk:], c)
    assert torch.isfinite(both[0]).all()


def test_lin_states_and_token_rows():
    H, dk, dv, slots = 64, 128, 128, 1100
    lens, s_in, s_out = [262_144, 8, 60], [-1, slots - 1, slots - 2], [0, slots - 1, slots - 3]
    T = sum(lens)
    assert T * H * dv * 2 > 1 << 32 and (slots - 3) * H * dk * dv * 4 > 1 << 32
    g = torch.Generator(device="cuda").manual_seed(2)

    def rows():
        return torch.empty((T, H, dk), dtype=torch.bfloat16, device="cuda").normal_(generator=g)

    def run(lens, s_in, s_out, slots, q, k, v, alpha, pool):
        p = wp.lin_plan(num_heads=H, num_qk_heads=H, head_dim_k=dk, head_dim_v=dv, num_state_slots=slots, chunk_lens=lens,
                        state_in=s_in, state_out=s_out, scale=dk ** -0.5)
        ws = wp.new_workspace(p)
        wp.lin_upload(p, ws)
        out = torch.full_like(v, float("nan"))
        wp.lin_chunked_prefill(p, q, k, v, alpha, pool, out, ws)
        return out

    x = [rows(), rows(), rows(), torch.full((T, H), 0.5, device="cuda")]
    pool = torch.zeros((slots, H, dk, dv), device="cuda")
    pool[slots - 2:].normal_(generator=g)
    few = pool[slots - 3:].clone()
    out = run(lens, s_in, s_out, slots, *x, pool)
    short = run(lens[1:], [2, 1], [2, 0], 3, *(t[lens[0]:].clone() for t in x), few)
    assert torch.equal(out[lens[0]:], short) and torch.equal(pool[slots - 3:], few)
    # decays of 1/2 forget within 200 tokens: the end of the long request, by itself
    n, state = 1000, torch.zeros((1, H, dk, dv), device="cuda")
    tail = run([n], [-1], [0], 1, *(t[lens[0] - n:lens[0]].clone() for t in x), state)
    err = (out[lens[0] - 500:lens[0]].float() - tail[-500:].float()).abs()
    # Each run is within 1.1 * 2^-7 of the sum of its terms' sizes: |q| . |k| / sqrt(128), about 7.2 and under 9, times 2^-j |v|
    # summed, about 1.6 and under 10.  States: 2^-15 each of a sum under 2 * 5.5 * 5.5.
    assert err.mean() <= 2 * 1.1 * 2.0 ** -7 * 7.2 * 1.6 and err.max() <= 2 * 1.1 * 2.0 ** -7 * 9 * 10
    assert (pool[0] - state[0]).abs().max() <= 2 * 2.0 ** -15 * 2 * 5.5 * 5.5
    assert torch.isfinite(out).all()
