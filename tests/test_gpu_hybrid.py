"""A hybrid stack served as a user would: three requests through a softmax layer over 4-bit pages and a linear-attention
layer with snapshots, prompts in ragged waves, one of them waiting at times, then single tokens on a kept plan of the
linear layer.  Every row of every wave is compared with the fp64 oracles run over the whole requests.

Tolerances: those of test_gpu_q4.py and test_gpu_lin.py.
"""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_35263_amd as wp
import workloads as wl

pytestmark = pytest.mark.gpu

HQ, HKV, D, PAGE = 16, 2, 128, 16           # the softmax layer
H, HQK, DK, DV = 8, 4, 128, 64              # the linear layer
WAVES = [[40, 0, 130], [33, 70, 0], [5, 1, 64]] + [[1, 1, 1]] * 6


def test_prompts_then_tokens_through_both_layers():
    g = torch.Generator().manual_seed(61)
    lens = np.array(WAVES)
    R, total = lens.shape[1], lens.sum(0)

    def bf(*shape):
        return torch.randn(shape, generator=g).to(torch.bfloat16)

    x = [{"q": bf(n, HQ, D), "k": bf(n, HKV, D), "v": bf(n, HKV, D), "lq": bf(n, HQK, DK), "lk": bf(n, HQK, DK),
          "lv": bf(n, H, DV), "alpha": torch.rand((n, H), generator=g) * 0.2 + 0.8} for n in total]
    pages = -(-total // PAGE)
    table = np.zeros((R, pages.max()), dtype=np.int32)
    order = np.random.default_rng(62).permutation(pages.sum())
    for r in range(R):
        table[r, :pages[r]] = order[pages[:r].sum():pages[:r + 1].sum()]
    k_pool, v_pool = (wp.q4_new_pool(int(pages.sum()), HKV, D, PAGE) for _ in range(2))
    states = torch.full((R, H, DK, DV), float("nan"), device="cuda")
    attn = dict(num_q_heads=HQ, num_kv_heads=HKV, head_dim_qk=D, head_dim_v=D, page_size=PAGE,
                num_pages=int(pages.sum()), softmax_scale=D ** -0.5, block_table=table)
    lin = dict(num_heads=H, num_qk_heads=HQK, head_dim_k=DK, head_dim_v=DV, num_state_slots=R,
               state_out=list(range(R)), scale=DK ** -0.5)
    done = np.zeros(R, dtype=np.int64)
    got = [{"out": [], "lse": [], "lin": []} for _ in range(R)]
    tokens = None
    for c in lens:
        part = {n: torch.cat([x[r][n][done[r]:done[r] + c[r]] for r in range(R)]).cuda() for n in x[0]}
        p = wp.q4_plan(prefix_lens=done, chunk_lens=c, **attn)
        ws = wp.new_workspace(p)
        wp.plan_upload(p, ws)
        out = torch.empty(c.sum(), HQ, D, dtype=torch.bfloat16, device="cuda")
        lse = torch.empty(c.sum(), HQ, device="cuda")
        wp.q4_append_kv(p, part["k"], part["v"], k_pool, v_pool, ws)
        wp.q4_chunked_prefill(p, part["q"], k_pool, v_pool, out, lse, ws)
        if (c == 1).all() and tokens is not None:
            lp, lws = tokens
        else:
            lp = wp.lin_plan(chunk_lens=c, state_in=[r if done[r] else -1 for r in range(R)], **lin)
            lws = wp.new_workspace(lp)
            wp.lin_upload(lp, lws)
            if (c == 1).all():
                tokens = lp, lws
        lo = torch.empty(c.sum(), H, DV, dtype=torch.bfloat16, device="cuda")
        wp.lin_chunked_prefill(lp, part["lq"], part["lk"], part["lv"], part["alpha"], states, lo, lws)
        for r in range(R):
            at = slice(c[:r].sum(), c[:r + 1].sum())
            for name, t in (("out", out), ("lse", lse), ("lin", lo)):
                got[r][name].append(t[at].float().cpu().numpy().astype(np.float64))
        done += c
    kv = [oracle.q4.pool_values(pool.cpu().numpy(), D, PAGE) for pool in (k_pool, v_pool)]
    for r in range(R):
        for pool, name in zip(kv, "kv"):                  # the cache holds the rounded rows
            pos = np.arange(total[r])
            want = oracle.q4.values(*oracle.q4.quantise(wl.to_bits(x[r][name])))
            assert np.array_equal(pool[table[r, pos // PAGE], :, pos % PAGE], want)
        o, lse, size = oracle.q4.attention(wl.to_bits(x[r]["q"]), *kv, [0], [total[r]], table[r:r + 1], PAGE, D ** -0.5)
        err = np.abs(np.concatenate(got[r]["out"]) - o)
        assert (err <= 1.1 * 2.0 ** -7 * size).all()
        assert (np.abs(np.concatenate(got[r]["lse"]) - lse) <= 1e-4).all()
        ref = [wl.to_bits(x[r][n]) for n in ("lq", "lk", "lv")] + [x[r]["alpha"].numpy(), np.zeros((1, H, DK, DV)), [total[r]],
                                                                   [-1], [0], DK ** -0.5]
        o, pool = oracle.lin.chunked_prefill(*ref)
        size, psize = oracle.lin.sizes(*ref)
        assert (np.abs(np.concatenate(got[r]["lin"]) - o) <= 1.1 * 2.0 ** -7 * size).all()
        assert (np.abs(states[r].cpu().numpy() - pool[0]) <= 2.0 ** -15 * psize[0]).all()
