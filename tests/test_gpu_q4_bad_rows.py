"""What the LSE of the 4-bit cache's attention says of a row whose softmax sum is not a number.

A cached K row of NaN holds the largest magnitude everywhere, so a query of positive numbers has a logit that overflows to
+infinity there and a sum that is NaN; a query of NaN has NaN logits alone.  In both the LSE has to be NaN, whole or joined
from splits: -infinity means that a row saw no key, and a finite LSE that the bad key was not there.  Rows that see
neither keep every bit.
"""
import numpy as np
import pytest
import torch

import workloads as wl
from tests.test_gpu_q4 import make, on_gpu, same

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
