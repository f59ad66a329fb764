"""Keys that no query sees leave no trace: pages, codes and scale bytes before the first and behind the last key of a request's
intervals may hold anything, codes of NaN and scales of infinity among them, and every answer keeps its bits."""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_35263_amd as wp
import workloads as wl
from tests.test_gpu_q8 import check, make, on_gpu, same

pytestmark = pytest.mark.gpu

WAVES = {
    # name: (q heads, KV heads, dim, page, prefix, chunk)
    "tokens": (32, 8, 128, 64, [700, 240, 333], [1, 1, 1]),
    "tokens_small": (24, 4, 64, 16, [300, 95, 1100], [1, 1, 1]),
    "tokens_small_pages": (16, 2, 128, 16, [257, 161], [1, 1]),
    "two_tiles_of_rows": (32, 1, 64, 64, [190, 400], [1, 1]),
    "few_rows": (16, 2, 128, 64, [200, 131, 333], [4, 2, 3]),
    "four_waves": (16, 2, 128, 64, [300, 177], [9, 16]),
    "four_waves_small": (24, 4, 64, 16, [250, 333], [17, 21]),
    "eight_waves": (8, 2, 128, 64, [470, 300], [150, 65]),
    "eight_waves_small": (8, 2, 64, 16, [433, 205], [130, 70]),
}
# first key that is seen, and how many keys before the request's cached end are not (both within every prefix above)
CUTS = [(1, 0), (15, 1), (16, 16), (17, 30), (31, 33), (33, 0), (64, 14), (70, 5), (79, 3), (80, 15), (47, 47)]
FORMS = {"plain": {}, "cap": {"score_cap": 30.0}, "cap_and_slopes": {"score_cap": 4.0, "slopes": 0.02}}


def spoiled(spec, t, first, end):
    """The tensors with all cached slots of request r outside [first[r], end[r]) as bad as bytes can be, and the block table with
    one such page in the place of every page that lies outside as a whole."""
    d, B = spec.head_dim_qk, spec.page_size
    table = spec.block_table.copy()
    used = set(table[table >= 0].tolist())
    spare = next(p for p in range(spec.num_pages) if p not in used)
    out = dict(t)
    for n in ("k_pool", "v_pool"):
        codes, e, padding = (np.array(a) for a in oracle.q8.split_pool(t[n].numpy(), d, B))
        codes[spare], e[spare] = 0x7F, 255
        for r in range(spec.num_requests):
            p = int(spec.prefix_lens[r])
            for j in list(range(first[r])) + list(range(end[r], p)):
                page, slot = spec.block_table[r, j // B], j % B
                codes[page, :, slot] = 0xFF if j & 1 else 0x7F
            for j in range(0, p // 16 * 16, 16):              # (the block of the new tokens keeps its scale)
                if j + 16 <= first[r] or j >= end[r]:
                    e[spec.block_table[r, j // B], :, j % B // 16] = 255
            for b in range(p // B):
                if (b + 1) * B <= first[r] or b * B >= end[r]:
                    table[r, b] = spare
        out[n] = torch.from_numpy(oracle.q8.join_pool(codes, e, padding))
    return out, table


def scores_of(spec, form):
    s = dict(FORMS[form])
    if "slopes" in s:
        s["slopes"] = np.full(spec.num_q_heads, s["slopes"], dtype=np.float32)
    return s


def compare(spec, form, begin, end, first, last):
    t = make(spec, 92)
    s = {**scores_of(spec, form), "key_begin": begin, "key_end": end}
    bad, table = spoiled(spec, t, first, last)
    for splits in (0, 3):
        clean = on_gpu(spec, t, max_splits=splits, **s)
        check(spec, t, clean, f"{form} splits {splits}", **{("cap" if n == "score_cap" else n): x for n, x in s.items()})
        held, spec.block_table = spec.block_table, table
        try:
            g = on_gpu(spec, bad, max_splits=splits, **s)
        finally:
            spec.block_table = held
        assert same(clean["out"], g["out"]) and same(clean["lse"], g["lse"]), splits


@pytest.mark.parametrize("form", sorted(FORMS))
@pytest.mark.parametrize("name", sorted(WAVES))
def test_keys_outside_the_intervals_leave_no_trace(name, form):
    """Every token of a request sees the same cached keys."""
    q, kv, dim, page, prefix, chunk = WAVES[name]
    for cut, (a, z) in enumerate(CUTS):
        spec = wl.custom_wave(q, kv, dim, dim, page, prefix, chunk, seed=91 + cut, name=name, pool_slack=0.2)
        first, last = np.full(len(prefix), a), np.array(prefix) - z
        compare(spec, form, np.repeat(first, chunk), np.repeat(last, chunk), first, last)


@pytest.mark.parametrize("form", sorted(FORMS))
@pytest.mark.parametrize("name", sorted(WAVES))
def test_what_a_window_has_left_behind_leaves_no_trace(name, form):
    q, kv, dim, page, prefix, chunk = WAVES[name]
    pos = np.concatenate([p + np.arange(c) for p, c in zip(prefix, chunk)])
    for window in (1, 16, 50, 77):
        spec = wl.custom_wave(q, kv, dim, dim, page, prefix, chunk, seed=93, name=name, pool_slack=0.2)
        first = np.maximum(0, np.array(prefix) + 1 - window)
        compare(spec, form, np.maximum(0, pos + 1 - window), pos + 1, first, np.array(prefix))


def test_a_tile_reads_none_of_the_keys_that_only_later_tiles_see():
    """Causal chunks too: a tile of a long chunk ends with its own last token."""
    spec = wl.custom_wave(8, 2, 128, 128, 64, [100], [150], seed=95, name="own_end")
    p = wp.q8_plan_for(spec)
    t = make(spec, 96)
    g = on_gpu(spec, t, plan=p)
    k, v = g["k_pool"].clone(), g["v_pool"].clone()
    rows = p.info()["rows_per_item"] // spec.group_size           # tokens of a tile
    end = 100 + rows                                              # keys that the first tile sees
    page, slot = (end + 16) // 64, (end + 15) // 16 * 16 % 64
    for pool in (k, v):
        at = pool[int(spec.block_table[0, page])]
        at[:, slot * 128:64 * 128] = 0x7F
    out, lse = torch.empty_like(g["out"]), torch.empty_like(g["lse"])
    wp.q8_chunked_prefill(p, g["q"], k, v, out, lse, g["ws"])
    assert same(out[:rows], g["out"][:rows]) and same(lse[:rows], g["lse"][:rows])
