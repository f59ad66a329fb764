"""What the LSE of the 8-bit cache's attention says of a row whose softmax sum is not a number.

A cached K row of NaN holds the largest magnitude everywhere, so a query of both signs has products of +infinity and of
-infinity with it, and a score that is NaN.  That key has no place in a running maximum: where a part of the work sees no
other key, its maximum is -infinity and its sum NaN.  The output and the LSE of the row have to be NaN all the same, whole or
joined from splits, and rows that do not see the key keep every bit.
"""
import numpy as np
import pytest
import torch

import workloads as wl
from tests.test_gpu_q8 import make, on_gpu, same

pytestmark = pytest.mark.gpu

WAVES = {
    # name: (q heads, KV heads, dim, page, prefix, chunk); the first request's first new token is the bad one, and where 32
    # divides its prefix it begins a block of 32 keys
    "alone_behind_32": (32, 8, 128, 64, [32, 40], [1, 1]),
    "alone_behind_64": (24, 4, 64, 16, [64, 15], [1, 1]),
    "alone_behind_96": (16, 2, 128, 16, [96, 7], [1, 1]),
    "alone_behind_many": (16, 2, 128, 64, [2048, 7], [1, 1]),
    "within_a_block": (16, 2, 128, 64, [45, 7], [1, 1]),
    "first_key": (16, 2, 64, 64, [0, 7], [1, 1]),
    "few_rows": (16, 2, 128, 64, [64, 333], [4, 3]),
    "two_tiles_of_rows": (32, 1, 64, 64, [32, 400], [1, 1]),
    "four_waves": (16, 2, 128, 64, [64, 77], [9, 16]),
    "eight_waves": (8, 2, 64, 16, [128, 5], [130, 70]),
}
SCORES = {"causal": {}, "cap": {"score_cap": 30.0}, "wide_cap": {"score_cap": 200.0}, "slopes": {"slopes": 0.05}}


def signs(heads, dim):
    """Signs of a query's values: halves in the even heads, eights in turn in the odd ones, so that some product sums of either
    order of the head dim are all of one sign."""
    at = np.arange(dim)
    return torch.from_numpy(np.stack([np.where((at < dim // 2) if h % 2 == 0 else (at // 8 % 2 == 0), 1.0, -1.0) for h in range(heads)]))


@pytest.mark.parametrize("form", sorted(SCORES))
@pytest.mark.parametrize("name", sorted(WAVES))
def test_a_key_whose_score_is_nan_shows_in_out_and_lse_of_every_row_that_sees_it(name, form):
    q, kv, dim, page, prefix, chunk = WAVES[name]
    spec = wl.custom_wave(q, kv, dim, dim, page, prefix, chunk, seed=81, name=name)
    t = make(spec, 82)
    # products of at least 2^9 * 1.75 * 2^127: infinite wherever a partial sum is of one sign
    t["q"] = ((1.0 + t["q"].float().abs()) * 512.0 * signs(q, dim)).to(torch.bfloat16)
    bad = {n: x.clone() for n, x in t.items()}
    bad["k_new"][0] = float("nan")
    kw = dict(SCORES[form])
    if "slopes" in kw:
        kw["slopes"] = np.full(q, kw["slopes"])
    seen = np.arange(spec.total_tokens) < chunk[0]
    for splits in (0, 1, 3):
        clean, g = on_gpu(spec, t, max_splits=splits, **kw), on_gpu(spec, bad, max_splits=splits, **kw)
        nan = torch.isnan(g["out"].float())
        assert torch.equal(nan.all(-1), nan.any(-1)) and torch.equal(nan.all(-1), torch.isnan(g["lse"])), splits
        # one pattern of signs or the other has whole products of one sign, however a kernel orders the head dim
        assert torch.isnan(g["lse"])[seen].view(chunk[0], q // 2, 2).all(1).any(-1).all(), splits
        assert same(clean["out"][~seen], g["out"][~seen]) and same(clean["lse"][~seen], g["lse"][~seen])
