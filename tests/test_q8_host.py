"""Host side of the 8-bit paged cache: plans, their scores, what they refuse, and the checks of a call's buffers (no GPU)."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2609_35263_amd as wp
import workloads as wl

FAKE = 1 << 20          # stands for a device address: nothing is launched on it


def kw(**over):
    base = dict(num_q_heads=8, num_kv_heads=2, head_dim_qk=64, head_dim_v=64, page_size=16, num_pages=16,
                softmax_scale=0.125, prefix_lens=[48], chunk_lens=[32], block_table=[[3, 7, 1, 12, 5, -1]])
    return {**base, **over}


@pytest.mark.parametrize("over,status", [
    (dict(prefix_lens=[-1]), -1), (dict(softmax_scale=0.0), -1), (dict(max_splits=-1), -1), (dict(num_q_heads=9), -1),
    (dict(head_dim_qk=96, head_dim_v=96), -2), (dict(head_dim_qk=64, head_dim_v=128), -2), (dict(page_size=32), -2),
    (dict(num_q_heads=16, num_kv_heads=1, head_dim_qk=576, head_dim_v=512, kv_shared=True), -2),
    (dict(block_table=[[3, 7, 16, 12, 5, -1]]), -3), (dict(block_table=[[3, 7, 1, 12, 12, -1]]), -4),
    (dict(block_table=[[3, 7, 1]]), -5),
])
def test_plans_refuse_what_the_bf16_cache_refuses_and_latent_caches(over, status):
    with pytest.raises(wp.WaveppError) as e:
        wp.q8_plan(**kw(**over))
    assert e.value.status == status


@pytest.mark.parametrize("scores", [
    dict(score_cap=-1.0), dict(score_cap=float("nan")), dict(score_cap=float("inf")), dict(score_cap=1e-4), dict(score_cap=2e6),
    dict(slopes=[0.0] * 7 + [float("nan")]), dict(slopes=[0.0] * 7 + [1025.0]), dict(slopes=[-float("inf")] * 8),
    dict(score_cap=1.0, softmax_scale=2e30), dict(score_cap=1e-3, softmax_scale=2e27), dict(slopes=[0.1] * 8, softmax_scale=1e-21),
    dict(key_begin=[-1] * 32), dict(key_begin=[0] * 31 + [81]), dict(key_end=[0] * 31 + [81]), dict(key_end=[80] * 31 + [-1]),
])
def test_plans_refuse_scores_out_of_range(scores):
    with pytest.raises(wp.WaveppError) as e:
        wp.q8_plan(**kw(**scores))
    assert e.value.status == -1


@pytest.mark.parametrize("scores", [dict(slopes=[1.0] * 7), dict(slopes=[[1.0] * 8]), dict(key_begin=[0] * 31),
                                    dict(key_end=np.zeros((32, 1))), dict(key_end=[0.5] * 32), dict(key_begin=[1 << 33] * 32)])
def test_the_binding_refuses_arrays_of_another_shape_or_kind(scores):
    with pytest.raises(ValueError):
        wp.q8_plan(**kw(**scores))


def test_scores_at_the_ends_of_their_ranges():
    for s in (dict(score_cap=1e-3, softmax_scale=9e26), dict(slopes=[0.1] * 8, softmax_scale=2e-20), dict(score_cap=1e-3), dict(score_cap=1e6), dict(slopes=[1024.0, -1024.0] * 4), dict(key_begin=[0, 80] * 16, key_end=[80, 0] * 16),
              dict(key_begin=[80] * 32), dict(key_end=[0] * 32)):
        assert wp.q8_plan(**kw(**s)).info()["total_tokens"] == 32


def test_page_bytes():
    assert [wp.q8_page_bytes(d, b) for d, b in ((64, 16), (64, 64), (128, 16), (128, 64))] == [1040, 4112, 2064, 8208]
    for d, b in ((96, 16), (128, 32), (0, 16), (576, 64)):
        with pytest.raises(ValueError):
            wp.q8_page_bytes(d, b)


@pytest.mark.parametrize("seed", range(24))
def test_items_cover_every_visible_key_of_every_row_once(seed):
    """With random intervals, empty ones among them: a row's items together have all of its keys, in tiles none of which is
    another's, and each row has an item even where it sees nothing."""
    rng = np.random.default_rng(seed)
    few = seed % 2 == 0
    R = int(rng.integers(1, 6))
    prefix, chunk = rng.integers(0, 6000, R), rng.integers(0, 4 if few else 200, R)
    spec = wl.custom_wave(16, 2, 128, 128, 64, prefix, chunk, seed=seed)
    n = np.repeat(prefix + chunk, chunk)
    pos = np.concatenate([p + np.arange(c) for p, c in zip(prefix, chunk)])
    begin, end = np.zeros_like(pos), pos + 1
    s = {}
    if seed % 3:
        begin = rng.integers(0, n + 1) if seed % 3 == 1 else np.maximum(0, pos - rng.integers(1, 500))
        s["key_begin"] = begin
    if seed % 4 > 1:
        end = rng.integers(0, n + 1)
        s["key_end"] = end
    p = wp.q8_plan_for(spec, max_splits=int(rng.integers(0, 6)), **s)
    info = p.info()
    seen = {}
    for req, head, row0, rows, lo, hi, part, split in p.items():
        if rows == 0:
            continue
        assert rows <= info["rows_per_item"] and lo % info["kv_tile"] == 0 and (lo < hi or (lo, hi) == (0, 0))
        seen.setdefault((req, head, row0, rows), []).append((lo, hi))
    cu = np.cumsum(chunk) - chunk
    for r in range(R):
        for head in range(2):
            tiles = sorted((k[2], k[3], sorted(v)) for k, v in seen.items() if k[:2] == (r, head))
            assert sum(t[1] for t in tiles) == chunk[r] * 8
            row = 0
            for row0, rows, parts in tiles:
                assert row0 == row
                tok = cu[r] + np.arange(row0 // 8, (row0 + rows - 1) // 8 + 1)
                real = begin[tok] < end[tok]
                if real.any():
                    assert parts[0][0] <= begin[tok][real].min() < parts[0][0] + info["kv_tile"] and parts[-1][1] == end[tok][real].max()
                else:
                    assert parts == [(0, 0)]
                assert all(a[1] == b[0] for a, b in zip(parts, parts[1:]))
                row += rows


def test_a_window_reads_its_window_alone():
    kw2 = dict(num_q_heads=32, num_kv_heads=8, head_dim_qk=128, head_dim_v=128, page_size=64, num_pages=600, softmax_scale=1.0,
               prefix_lens=[30000], chunk_lens=[1], block_table=np.arange(600)[None])
    items = wp.q8_plan(key_begin=[30001 - 4096], **kw2).items()
    items = items[items[:, 3] > 0]
    assert items[:, 4].min() == (30001 - 4096) // 128 * 128 and items[:, 5].max() == 30001


def rows_of(requests, prefix, chunk, dim=128, page=64, **scores):
    n = -(-(prefix + chunk) // page)
    p = wp.q8_plan(num_q_heads=32, num_kv_heads=8, head_dim_qk=dim, head_dim_v=dim, page_size=page, num_pages=n * requests,
                   softmax_scale=0.1, prefix_lens=[prefix] * requests, chunk_lens=[chunk] * requests,
                   block_table=np.arange(n * requests).reshape(requests, n), **scores)
    return p.info()["rows_per_item"]


def test_items_of_few_keys_take_four_waves_where_there_are_enough_of_them():
    assert rows_of(24, 0, 500) == 128                          # short prompts
    assert rows_of(24, 0, 500, page=16) == 128
    assert rows_of(4, 2000, 2048) == 256                       # 3,000 keys an item
    assert rows_of(4, 2000, 2048, dim=64) == 128               # half of the products for each key's turn into bf16
    assert rows_of(4, 2000, 2048, score_cap=30.0) == 128       # more vector work beside it
    assert rows_of(4, 8000, 2048, score_cap=30.0) == 256
    assert rows_of(2, 0, 500) == 256                           # 256 items of 128 rows: not enough
    begin = np.tile(np.maximum(0, 2000 + np.arange(2048) - 999), 4)
    assert rows_of(4, 2000, 2048, key_begin=begin) == 128      # a window of 1,000
    assert rows_of(1, 100000, 2048, key_begin=begin[:2048] + 98000) == 128


def call(fn, plan, *bufs, ws=FAKE, size=None):
    size = plan.workspace_bytes if size is None else size
    return getattr(wp.load_library(), fn)(plan.handle, *bufs, ws, size, None)


def test_calls_check_their_plan_workspace_and_buffers_before_anything_is_enqueued():
    q8, q4, bf = wp.q8_plan(**kw()), wp.q4_plan(**kw()), wp.plan(**kw())
    lib = wp.load_library()
    for fn, n in (("wavepp_q8_append_kv", 4), ("wavepp_q8_read_kv", 4), ("wavepp_q8_chunked_prefill", 5)):
        bufs = [FAKE] * n
        assert call(fn, bf, *bufs) == -1 and b"wavepp_q8_plan" in lib.wavepp_last_error()
        assert call(fn, q4, *bufs) == -1 and b"4-bit" in lib.wavepp_last_error()
        assert call(fn, q8, *bufs, ws=None) == -1
        assert call(fn, q8, *bufs, ws=FAKE + 16) == -1
        assert call(fn, q8, *bufs, size=q8.workspace_bytes - 1) == -6
        assert call(fn, q8, *bufs) == -1 and b"wavepp_attn_plan_upload" in lib.wavepp_last_error()
        assert getattr(lib, fn)(None, *bufs, FAKE, 1 << 20, None) == -1
    for fn, n in (("wavepp_attn_append_kv", 4), ("wavepp_attn_chunked_prefill", 5), ("wavepp_q4_append_kv", 4),
                  ("wavepp_q4_read_kv", 4), ("wavepp_q4_chunked_prefill", 5)):
        assert call(fn, q8, *[FAKE] * n) == -1 and b"wavepp_q8" in lib.wavepp_last_error()
    assert lib.wavepp_attn_chunked_prefill_noalloc(q8.handle, *[FAKE] * 7, None) == -1
    out = ctypes.c_void_p(5)
    assert lib.wavepp_q8_plan(None, None, None, 0, ctypes.byref(out)) == -1


def test_an_idle_wave_needs_no_buffers():
    for s in ({}, dict(key_begin=[], key_end=[], slopes=[0.5] * 8, score_cap=3.0)):
        p = wp.q8_plan(**kw(chunk_lens=[0], **s))
        assert call("wavepp_q8_append_kv", p, None, None, None, None) == 0
        assert call("wavepp_q8_read_kv", p, None, None, None, None) == 0
        assert call("wavepp_q8_chunked_prefill", p, None, None, None, None, None) == 0


def test_the_binding_checks_shapes_types_and_kinds_of_plan():
    p, bf, q4 = wp.q8_plan(**kw()), wp.plan(**kw()), wp.q4_plan(**kw())
    pool = torch.zeros(16, 2, 1040, dtype=torch.uint8)
    q, rows = torch.zeros(32, 8, 64, dtype=torch.bfloat16), torch.zeros(32, 2, 64, dtype=torch.bfloat16)
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    for bad in (dict(k_pool=pool[:15]), dict(v_pool=pool[:, :1]), dict(q=q[:31]), dict(out=None), dict(k_pool=None)):
        a = {**dict(q=q, k_pool=pool, v_pool=pool, out=q, lse=None), **bad}
        with pytest.raises(ValueError):
            wp.q8_chunked_prefill(p, a["q"], a["k_pool"], a["v_pool"], a["out"], a["lse"], ws)
    with pytest.raises(ValueError, match="device"):
        wp.q8_append_kv(p, rows, rows, pool, pool, ws)
    for other in (bf, q4):
        with pytest.raises(ValueError, match="q8_plan"):
            wp.q8_append_kv(other, rows, rows, pool, pool, ws)
    with pytest.raises(ValueError, match="q4_plan"):
        wp.q4_append_kv(p, rows, rows, pool, pool, ws)
    with pytest.raises(ValueError):
        wp.q8_read_kv(p, pool, pool, rows, None, ws)
