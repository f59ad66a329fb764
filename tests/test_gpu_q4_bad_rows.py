"""What the LSE of the 4-bit cache's attention says of a row whose softmax sum is not a number.

A cached K row of NaN holds the largest magnitude everywhere, so a query of positive numbers has a logit that overflows to
+infinity there and a sum that is NaN; a query of NaN has NaN logits alone.  In both the LSE has to be NaN, whole or joined
from splits: -infinity means that a row saw no key, and a finite LSE that the bad key was not there.  Rows that see
neither keep every bit.
"""
import numpy as np
import pytest
import torch

import oracle
import workloads as wl
from tests.test_gpu_q4 import LSE, MERGED, make, on_gpu, same

pytestmark = pytest.mark.gpu

WAVES = {
    # name: (q heads, KV heads, dim, page, prefix, chunk)
    "tokens": (32, 8, 128, 64, [700, 40], [1, 1]),
    "tokens_small": (24, 4, 64, 16, [300, 15], [1, 1]),
    "few_rows_many_splits": (24, 4, 64, 16, [9000, 2049], [1, 1]),
    "few_rows": (16, 2, 128, 64, [200, 333], [4, 3]),
    "four_waves": (16, 2, 128, 64, [500, 77], [9, 16]),
    "eight_waves": (8, 2, 64, 16, [600, 5], [130, 70]),
    "long_four_waves": (16, 2, 128, 64, [20000, 300], [9, 9]),
}


def run(name, splits, spoil):
    """The wave without and with spoil(tensors), and which of its tokens are the first request's."""
    q, kv, dim, page, prefix, chunk = WAVES[name]
    spec = wl.custom_wave(q, kv, dim, dim, page, prefix, chunk, seed=71, name=name)
    t = make(spec, 72)
    t["q"] = t["q"].abs()
    bad = {n: x.clone() for n, x in t.items()}
    spoil(bad)
    return on_gpu(spec, t, max_splits=splits), on_gpu(spec, bad, max_splits=splits), np.arange(spec.total_tokens) < chunk[0]


def check(clean, g, seen):
    assert torch.isfinite(clean["lse"]).all()
    lse = g["lse"][seen]
    assert torch.isnan(lse).all(), lse[~torch.isnan(lse)][:4]
    assert torch.isnan(g["out"][seen].float()).all()
    assert same(clean["out"][~seen], g["out"][~seen]) and same(clean["lse"][~seen], g["lse"][~seen])


@pytest.mark.parametrize("name", sorted(WAVES))
@pytest.mark.parametrize("splits", [0, 1, 3])
def test_a_bad_key_shows_in_the_lse_of_every_row_that_sees_it(name, splits):
    def spoil(t):
        t["k_new"][0] = float("nan")                 # the first request's first new token

    check(*run(name, splits, spoil))


@pytest.mark.parametrize("name", sorted(WAVES))
@pytest.mark.parametrize("splits", [0, 3])
def test_a_query_of_nan_has_an_lse_of_nan(name, splits):
    def spoil(t):
        t["q"][0] = float("nan")

    clean, g, _ = run(name, splits, spoil)
    check(clean, g, np.arange(len(g["out"])) < 1)


def test_a_row_whose_keys_all_weigh_nothing_still_says_so():
    """A logit of -infinity for the only key, or for all of them: no weight, an LSE of -infinity."""
    spec = wl.custom_wave(16, 2, 128, 128, 64, [0], [1], seed=73, name="nothing")
    t = make(spec, 74)
    t["q"], t["k_new"] = -t["q"].abs(), torch.full_like(t["k_new"], float("inf"))
    g = on_gpu(spec, t)
    assert (g["lse"] == -float("inf")).all()


@pytest.mark.parametrize("name", sorted(WAVES))
@pytest.mark.parametrize("splits", [0, 3])
def test_one_bad_number_of_a_key_with_a_finite_logit(name, splits):
    """A logit of order 1e37 is finite, but fp32 cannot place its exponential: where it is the largest, out and LSE are NaN.
    Where it is as far below zero the key weighs nothing, as it should."""
    def spoil(sign):
        def do(t):
            t["k_new"][0, :, 5] = float("nan")       # cached as 6 * 2^125, the rest of its block as zeros
            c = WAVES[name][5][0]
            t["q"][:c, :, 5] = (sign * (0.25 + 0.5 * torch.rand(t["q"][:c, :, 5].shape, generator=gen))).to(torch.bfloat16)
        return do

    gen = torch.Generator().manual_seed(75)
    check(*run(name, splits, spoil(1.0)))
    clean, g, seen = run(name, splits, spoil(-1.0))
    assert same(clean["out"][~seen], g["out"][~seen]) and same(clean["lse"][~seen], g["lse"][~seen])
    q, kv, dim, page, prefix, chunk = WAVES[name]
    right(wl.custom_wave(q, kv, dim, dim, page, prefix, chunk, seed=71, name=name), g)


def right(spec, g):
    """Whether the outputs are the oracle's over the values that the cache holds."""
    k, v = (oracle.q4.pool_values(g[n].cpu().numpy(), spec.head_dim_qk, spec.page_size) for n in ("k_pool", "v_pool"))
    with np.errstate(over="ignore", invalid="ignore"):
        o, lse, size = oracle.q4.attention(wl.to_bits(g["q"].cpu()), k, v, spec.prefix_lens, spec.chunk_lens, spec.block_table,
                                           spec.page_size, spec.softmax_scale)
    assert (np.abs(g["out"].float().cpu().numpy() - o) <= MERGED * size).all()
    assert (np.abs(g["lse"].cpu().numpy() - lse) <= LSE).all()


@pytest.mark.parametrize("dim,page", [(128, 64), (64, 16)])
@pytest.mark.parametrize("chunk", [1, 9, 40])
@pytest.mark.parametrize("splits", [1, 9, 17])
def test_a_key_far_below_zero_alone_in_its_split(dim, page, chunk, splits):
    """The first new token begins a tile, and a split where a tile is one: its row sees no other key there."""
    spec = wl.custom_wave(16, 2, dim, dim, page, [1024, 70], [chunk, 1], seed=76, name="alone")
    t = make(spec, 77)
    t["k_new"][0, :, 5] = float("nan")
    t["q"][:chunk, :, 5] = -t["q"][:chunk, :, 5].abs() - 0.25
    right(spec, on_gpu(spec, t, max_splits=splits))
