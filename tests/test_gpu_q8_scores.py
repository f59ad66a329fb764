"""Capped scores over 8-bit pages with intervals of keys, in every form of the kernels, and the bounds that a cap allows.

Tolerances, fixed before the first run.  A key's product z = softmax_scale q.k is off by at most e = (d + 4) 2^-24 softmax_scale
sum |q k|.  The cap's slope at a distance u from 0 is 1 - tanh^2(u / c), which falls with u, so c tanh(z / c) is off by no more
than e (1 - tanh^2(max(|z| - e, 0) / c)), nor by more than the 2 c that there are, and by what its header says of the tanh
itself: 2^-20 of it, and 2^-21 c for caps up to 128.  With a slope F = |slope distance| adds 2^-22 F, and 2^-20 of the score's
size for the constants.  E is the worst of that over a row's keys, and an output is then off by at most
    2^-8 size + 2^-8 |o| + (2 (E + n 2^-24) + 2^-20) size,         size = sum p |v|, n keys
(the weights as rounded to bf16, the output's rounding, the weights and their sum), an LSE by E + n 2^-24 + 2^-20.
"""
import numpy as np
import pytest
import torch

import oracle
import workloads as wl
from tests.test_gpu_q8 import WAVES, appended, make, on_gpu

pytestmark = pytest.mark.gpu

MORE = {
    # several tiles that all rows see whole, between the ends of their intervals: (q heads, KV heads, dim, page, prefix, chunk)
    "long_tokens": (32, 8, 128, 64, [900, 1100], [1, 1]),
    "long_four_waves": (16, 2, 128, 64, [900], [16]),
    "long_four_waves_small": (24, 4, 64, 16, [1000], [21]),
    "long_eight_waves": (8, 2, 128, 64, [1300], [70]),
    "long_eight_waves_small": (8, 2, 64, 16, [1100, 3], [80, 2]),
}
ALL = {**{n: WAVES[n] for n in ("tokens", "tokens_small", "two_tiles_of_rows", "few_rows_mixed", "odd_group", "four_waves", "four_waves_small",
                                "eight_waves", "eight_waves_small", "chunks_beside_tokens")}, **MORE}


def wave(name, seed):
    q, kv, dim, page, prefix, chunk = ALL[name]
    return wl.custom_wave(q, kv, dim, dim, page, prefix, chunk, seed=seed, name=name)


def reference(spec, t, pools, cap, slopes=None, key_begin=None, key_end=None):
    """(o, lse, size, E, n) of the module's text, the worst product of a row found key by key."""
    d, B = spec.head_dim_qk, spec.page_size
    kv, vv = (oracle.q8.pool_values(p, d, B) for p in pools)
    bits = wl.to_bits(t["q"])
    o, lse, size = oracle.q8.attention(bits, kv, vv, spec.prefix_lens, spec.chunk_lens, spec.block_table, B, spec.softmax_scale,
                                       cap=cap, slopes=slopes, key_begin=key_begin, key_end=key_end)
    q = oracle.bf16_bits_to_f64(bits)
    E, N = np.zeros(lse.shape), np.ones(lse.shape)
    at = 0
    for r in range(spec.num_requests):
        p, c = int(spec.prefix_lens[r]), int(spec.chunk_lens[r])
        pos = np.arange(p + c)
        pages = np.asarray(spec.block_table[r], dtype=np.int64)[pos // B]
        for i in range(c):
            a = 0 if key_begin is None else int(key_begin[at + i])
            b = p + i + 1 if key_end is None else int(key_end[at + i])
            if a >= b:
                continue
            for h in range(spec.num_q_heads):
                K = kv[pages[a:b], h // spec.group_size, pos[a:b] % B]
                z = spec.softmax_scale * (K @ q[at + i, h])
                e = (d + 4) * 2.0 ** -24 * spec.softmax_scale * (np.abs(K) @ np.abs(q[at + i, h]))
                F = 0.0 if slopes is None else abs(float(slopes[h])) * np.abs(p + i - pos[a:b])
                s = np.abs(z)
                if cap:
                    e = np.minimum(e * (1.0 - np.tanh(np.maximum(s - e, 0.0) / cap) ** 2), 2 * cap)
                    s = cap * np.tanh(s / cap)
                worst = e + 2.0 ** -20 * (s + F) + (2.0 ** -21 * cap if cap <= 128 else 0.0) + 2.0 ** -22 * F
                E[at + i, h], N[at + i, h] = worst.max(), b - a
        at += c
    return o, lse, size, E, N


def compare(g, ref, what=""):
    o, lse, size, E, n = ref
    got, got_lse = g["out"].float().cpu().numpy().astype(np.float64), g["lse"].cpu().numpy().astype(np.float64)
    blind = np.isneginf(lse)
    assert np.isneginf(got_lse[blind]).all() and (got[blind] == 0).all(), "rows that see nothing"
    off = E + n * 2.0 ** -24
    bound = 2.0 ** -8 * (size + np.abs(o)) + (2 * off + 2.0 ** -20)[..., None] * size
    err, lerr = np.abs(got - o), np.abs(np.where(blind, 0.0, got_lse) - np.where(blind, 0.0, lse))
    print(f"[q8 scores] {what}: out {(err / np.maximum(bound, 1e-300)).max():.2f} of its bound, lse "
          f"{(lerr / (off + 2.0 ** -20)).max():.2f} of its, E up to {E.max():.1e}", flush=True)
    assert (err <= bound).all() and (lerr <= off + 2.0 ** -20).all()


def intervals(spec, rng):
    pos = np.concatenate([p + np.arange(c) for p, c in zip(spec.prefix_lens, spec.chunk_lens)]).astype(np.int64)
    n = np.repeat(spec.prefix_lens + spec.chunk_lens, spec.chunk_lens).astype(np.int64)
    start = np.maximum(0, pos - pos % 37)
    far = np.maximum(0, pos - pos % 433)
    return {
        "none": {}, "window": {"key_begin": np.maximum(0, pos + 1 - 20)}, "wide_window": {"key_begin": np.maximum(0, pos + 1 - 600)},
        "documents": {"key_begin": start}, "prefix": {"key_begin": start, "key_end": np.minimum(n, np.maximum(pos + 1, start + 15))},
        "long_documents": {"key_begin": far, "key_end": np.minimum(n, np.maximum(pos + 1, far + 400))}, "all_keys": {"key_end": n},
        "any": {"key_begin": rng.integers(0, n + 1), "key_end": rng.integers(0, n + 1)}, "nothing": {"key_begin": pos + 1},
        "nothing_at_all": {"key_end": pos * 0}, "first_key_alone": {"key_end": np.minimum(n, 1)},
        "last_key_alone": {"key_begin": n - 1, "key_end": n},
    }


SPANS = sorted(intervals(wl.custom_wave(2, 1, 64, 64, 16, [1], [1], seed=0), np.random.default_rng(0)))


@pytest.mark.parametrize("span", SPANS)
@pytest.mark.parametrize("name", sorted(ALL))
def test_capped_scores_with_intervals(name, span):
    """Caps that the fixed reference takes, over scores that reach them."""
    spec = wave(name, 101)
    t = make(spec, 102)
    t["q"] = (t["q"].float() * 4.0).to(torch.bfloat16)
    s = intervals(spec, np.random.default_rng(103))[span]
    pools = appended(spec, t)
    for cap in (3.0, 50.0):
        ref = reference(spec, t, pools, cap, **s)
        for splits in (0, 3):
            compare(on_gpu(spec, t, max_splits=splits, score_cap=cap, **s), ref, f"{name} {span} cap {cap} splits {splits}")


@pytest.mark.parametrize("cap,sloped", [(50.5, False), (30.0, True), (500.0, False), (500.0, True), (0.0, True), (0.0, False)])
@pytest.mark.parametrize("name", ["four_waves_small"] + sorted(MORE))
def test_other_scores_with_intervals(name, cap, sloped):
    """Forms with a running maximum, in the waves that have whole tiles between their ends."""
    spec = wave(name, 111)
    t = make(spec, 112)
    pools = appended(spec, t)
    slopes = np.exp2(-8.0 * (1 + np.arange(spec.num_q_heads)) / spec.num_q_heads).astype(np.float32) if sloped else None
    for span, s in intervals(spec, np.random.default_rng(113)).items():
        if span in ("prefix", "nothing", "first_key_alone", "last_key_alone"):
            continue
        s = {**s, **({"slopes": slopes} if sloped else {})}
        ref = reference(spec, t, pools, cap, **s)
        for splits in (0, 3):
            compare(on_gpu(spec, t, max_splits=splits, score_cap=cap, **s), ref,
                    f"{name} {span} cap {cap} slopes {sloped} splits {splits}")


@pytest.mark.parametrize("name", sorted(ALL))
@pytest.mark.parametrize("cap", [4.0, 50.0, 80.0])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_scores_all_at_their_cap_give_the_values_mean(name, cap, sign):
    """Every product is over 20 caps, so every score is the cap to 2^-50 of it: an LSE of the cap and ln n, and a plain mean."""
    spec = wave(name, 121)
    t = make(spec, 122, garbage=False)
    t["q"] = ((t["q"].float().abs() + 0.5) * 4000.0 * sign).to(torch.bfloat16)
    t["k_new"] = t["k_new"].abs() + 0.5
    d, B = spec.head_dim_qk, spec.page_size
    t["k_pool"] = torch.from_numpy(oracle.q8.quantise_pool(np.abs(oracle.q8.pool_values(t["k_pool"].numpy(), d, B)) + 0.5))
    vv = oracle.q8.pool_values(appended(spec, t)[1], d, B)
    shape = (spec.total_tokens, spec.num_q_heads)
    o, size, n = np.zeros((*shape, d)), np.zeros((*shape, d)), np.zeros(shape)
    at = 0
    for r in range(spec.num_requests):
        p, c = int(spec.prefix_lens[r]), int(spec.chunk_lens[r])
        pos = np.arange(p + c)
        V = vv[np.asarray(spec.block_table[r], dtype=np.int64)[pos // B], :, pos % B]                 # [n, H, d]
        for i in range(c):
            seen = V[:p + i + 1].repeat(spec.group_size, axis=1)
            o[at + i], size[at + i], n[at + i] = seen.mean(0), np.abs(seen).mean(0), p + i + 1
        at += c
    E = np.full(shape, (2.0 ** -20 + 2.0 ** -21) * cap)
    for splits in (0, 3):
        compare(on_gpu(spec, t, max_splits=splits, score_cap=cap), (o, sign * cap + np.log(n), size, E, n), f"{name} {sign} x {cap}")


@pytest.mark.parametrize("name", sorted(ALL))
def test_a_product_that_overflows_is_a_score_at_the_cap(name):
    """A key of the largest magnitude everywhere: its score is the cap, and every other key counts as without it."""
    spec = wave(name, 131)
    t = make(spec, 132)
    t["q"] = t["q"].abs()
    t["k_new"][0] = float("inf")
    pools = appended(spec, t)
    for cap in (4.0, 50.0, 200.0):
        ref = reference(spec, t, pools, cap)
        for splits in (1, 3):
            compare(on_gpu(spec, t, max_splits=splits, score_cap=cap), ref, f"{name} cap {cap} splits {splits}")


@pytest.mark.parametrize("name", sorted(ALL))
@pytest.mark.parametrize("sign,power", [(1.0, 40), (-1.0, -40)])
def test_the_largest_and_smallest_values_beside_scores_at_a_cap_of_50(name, sign, power):
    """Weights of 2^64 with values of up to 2^40, and weights of 2^-80 with values from 2^-40 on: what the header allows."""
    spec = wave(name, 141)
    t = make(spec, 142, garbage=False)
    t["q"] = ((t["q"].float().abs() + 0.5) * 4000.0 * sign).to(torch.bfloat16)
    t["k_new"] = t["k_new"].abs() + 0.5
    d, B = spec.head_dim_qk, spec.page_size
    t["k_pool"] = torch.from_numpy(oracle.q8.quantise_pool(np.abs(oracle.q8.pool_values(t["k_pool"].numpy(), d, B)) + 0.5))
    for n in ("v_new", "v_pool"):
        v = t[n].double().numpy() if n == "v_new" else oracle.q8.pool_values(t[n].numpy(), d, B)
        # magnitudes between a half and one times the power of two, or from one to two times it where that is the smallest
        v = np.where(v < 0, -1.0, 1.0) * (0.5 + 0.5 * np.minimum(np.abs(v), 1.0)) * 2.0 ** (power + (power < 0))
        t[n] = torch.from_numpy(v).to(torch.bfloat16) if n == "v_new" else torch.from_numpy(oracle.q8.quantise_pool(v))
    pools = appended(spec, t)
    ref = reference(spec, t, pools, 50.0)
    for splits in (0, 3):
        compare(on_gpu(spec, t, max_splits=splits, score_cap=50.0), ref, f"{name} 2^{power}")
