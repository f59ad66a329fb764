"""How the plans of linear attention cut a long chunk that runs beside many short ones (no GPU)."""
import time

import numpy as np
import pytest

import paper_2609_35263_amd as wp


def plan(lens, H=64, Hqk=64, dk=128, dv=128):
    n = len(lens)
    return wp.lin_plan(num_heads=H, num_qk_heads=Hqk, head_dim_k=dk, head_dim_v=dv, num_state_slots=n, chunk_lens=lens,
                       state_in=[-1] * n, state_out=list(range(n)))


@pytest.mark.parametrize("short", [1, 14, 15, 16, 40, 100])
def test_a_long_chunk_is_cut_however_many_short_ones_run_beside_it(short):
    """64 heads leave a whole chunk of 16,384 tokens on 64 of 256 CUs for 256 blocks; the short ones take none of them long."""
    i = plan([16384] + [64] * short).info()
    assert i["num_partials"] >= 3 and i["num_segments"] == short + 1 + i["num_partials"]


@pytest.mark.parametrize("short", [29, 30, 31, 32, 200])
def test_the_same_for_heads_that_share_q_and_k(short):
    i = plan([9000] + [64] * short, 32, 8, 128, 64).info()
    assert i["num_partials"] >= 3


def test_single_tokens_beside_it_change_nothing():
    alone, beside = plan([16384]).info(), plan([16384] + [1] * 500).info()
    assert alone["num_segments"] == beside["num_segments"] > 1


@pytest.mark.parametrize("lens", [[4096] * 16, [64] * 500, [2000] * 64, list(range(1500, 2500, 20))])
def test_chunks_of_like_lengths_that_fill_the_chip_stay_whole(lens):
    i = plan(lens).info()
    assert i["num_partials"] == 0 and i["num_segments"] == len(lens)


def test_where_the_others_fill_the_chip_for_as_long_a_chunk_stays_whole():
    """16 chunks of 16,384 tokens, 64 heads: four rounds of the longest on 256 CUs."""
    assert plan([16384] * 16 + [64] * 200).info()["num_partials"] == 0


def test_cutting_stays_quick():
    """A plan of 64,000 chains with one long chunk takes well under a second."""
    rng = np.random.default_rng(1)
    lens = [400000] + rng.integers(11, 200, 1000).tolist()
    best = min(_seconds(lens) for _ in range(3))
    assert best < 0.5, best


def _seconds(lens):
    t = time.perf_counter()
    plan(lens)
    return time.perf_counter() - t
