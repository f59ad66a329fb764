"""Host side of the 4-bit paged cache: plans, what they refuse, and the checks of a call's buffers (no GPU)."""
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
        wp.q4_plan(**kw(**over))
    assert e.value.status == status


def test_page_bytes():
    assert [wp.q4_page_bytes(d, b) for d, b in ((64, 16), (64, 64), (128, 16), (128, 64))] == [544, 2176, 1088, 4352]
    for d, b in ((96, 16), (128, 32), (0, 16), (576, 64)):
        with pytest.raises(ValueError):
            wp.q4_page_bytes(d, b)


@pytest.mark.parametrize("chunk,heads,rows", [([1], (32, 8), 32), ([8], (32, 8), 32), ([9], (32, 8), 128), ([1], (64, 1), 128),
                                              ([1, 33], (32, 8), 256), ([32], (32, 8), 128), ([2], (16, 1), 32)])
def test_rows_of_an_item_follow_the_longest_chunk(chunk, heads, rows):
    n = len(chunk)
    p = wp.q4_plan(num_q_heads=heads[0], num_kv_heads=heads[1], head_dim_qk=128, head_dim_v=128, page_size=64, num_pages=64,
                   softmax_scale=1.0, prefix_lens=[100] * n, chunk_lens=chunk, block_table=np.arange(64).reshape(n, -1))
    assert p.info()["rows_per_item"] == rows


def test_tokens_beside_chunks_have_items_of_their_own():
    """Few-row requests come last, in tiles and splits as if alone."""
    kw = dict(num_q_heads=16, num_kv_heads=2, head_dim_qk=128, head_dim_v=128, page_size=64, num_pages=400, softmax_scale=1.0,
              block_table=np.arange(400).reshape(4, 100))
    p = wp.q4_plan(prefix_lens=[5000, 100, 3000, 64], chunk_lens=[1, 300, 2, 0], **kw)
    items = p.items()
    few = np.isin(items[:, 0], [0, 2]) & (items[:, 3] > 0)
    assert p.info()["rows_per_item"] == 256 and few.any() and items[few][:, 3].max() == 16
    first = np.flatnonzero(few)[0]
    assert not ((items[first:, 3] > 0) & ~few[first:]).any()
    alone = wp.q4_plan(prefix_lens=[5000, 100, 3000, 64], chunk_lens=[1, 0, 2, 0], **kw).items()
    assert sorted(map(tuple, alone[alone[:, 3] > 0][:, [0, 1, 2, 3, 4, 5]])) == sorted(map(tuple, items[few][:, [0, 1, 2, 3, 4, 5]]))


@pytest.mark.parametrize("seed", range(8))
def test_items_cover_every_visible_key_of_every_row_once(seed):
    rng = np.random.default_rng(seed)
    few = seed % 2 == 0
    R = int(rng.integers(1, 6))
    prefix, chunk = rng.integers(0, 6000, R), rng.integers(0, 4 if few else 200, R)
    spec = wl.custom_wave(16, 2, 128, 128, 64, prefix, chunk, seed=seed)
    p = wp.q4_plan_for(spec, max_splits=int(rng.integers(0, 6)))
    info = p.info()
    seen = {}
    for req, head, row0, rows, lo, hi, part, split in p.items():
        if rows == 0:
            continue
        assert rows <= info["rows_per_item"] and lo % info["kv_tile"] == 0 and lo < hi
        seen.setdefault((req, head, row0, rows), []).append((lo, hi))
    for r in range(R):
        for head in range(2):
            tiles = sorted((k[2], k[3], sorted(v)) for k, v in seen.items() if k[:2] == (r, head))
            assert sum(t[1] for t in tiles) == chunk[r] * 8
            row = 0
            for row0, rows, parts in tiles:
                assert row0 == row and parts[0][0] == 0 and parts[-1][1] == prefix[r] + (row0 + rows - 1) // 8 + 1
                assert all(a[1] == b[0] for a, b in zip(parts, parts[1:]))
                row += rows


def call(fn, plan, *bufs, ws=FAKE, size=None):
    size = plan.workspace_bytes if size is None else size
    return getattr(wp.load_library(), fn)(plan.handle, *bufs, ws, size, None)


def test_calls_check_their_plan_workspace_and_buffers_before_anything_is_enqueued():
    q4, bf = wp.q4_plan(**kw()), wp.plan(**kw())
    lib = wp.load_library()
    for fn, n in (("wavepp_q4_append_kv", 4), ("wavepp_q4_read_kv", 4), ("wavepp_q4_chunked_prefill", 5)):
        bufs = [FAKE] * n
        assert call(fn, bf, *bufs) == -1 and b"wavepp_q4_plan" in lib.wavepp_last_error()
        assert call(fn, q4, *bufs, ws=None) == -1
        assert call(fn, q4, *bufs, ws=FAKE + 16) == -1
        assert call(fn, q4, *bufs, size=q4.workspace_bytes - 1) == -6
        assert call(fn, q4, *bufs) == -1 and b"wavepp_attn_plan_upload" in lib.wavepp_last_error()
        assert getattr(lib, fn)(None, *bufs, FAKE, 1 << 20, None) == -1
    for fn, n in (("wavepp_attn_append_kv", 4), ("wavepp_attn_chunked_prefill", 5)):
        assert call(fn, q4, *[FAKE] * n) == -1 and b"wavepp_q4" in lib.wavepp_last_error()
    assert lib.wavepp_attn_chunked_prefill_noalloc(q4.handle, *[FAKE] * 7, None) == -1
    out = ctypes.c_void_p(5)
    assert lib.wavepp_q4_plan(None, None, 0, ctypes.byref(out)) == -1


def test_an_idle_wave_needs_no_buffers():
    p = wp.q4_plan(**kw(chunk_lens=[0]))
    assert call("wavepp_q4_append_kv", p, None, None, None, None) == 0
    assert call("wavepp_q4_chunked_prefill", p, None, None, None, None, None) == 0


def test_the_binding_checks_shapes_types_and_kinds_of_plan():
    p, bf = wp.q4_plan(**kw()), wp.plan(**kw())
    pool = torch.zeros(16, 2, 544, dtype=torch.uint8)
    q, rows = torch.zeros(32, 8, 64, dtype=torch.bfloat16), torch.zeros(32, 2, 64, dtype=torch.bfloat16)
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    for bad in (dict(k_pool=pool[:15]), dict(v_pool=pool[:, :1]), dict(q=q[:31]), dict(out=None), dict(k_pool=None)):
        a = {**dict(q=q, k_pool=pool, v_pool=pool, out=q, lse=None), **bad}
        with pytest.raises(ValueError):
            wp.q4_chunked_prefill(p, a["q"], a["k_pool"], a["v_pool"], a["out"], a["lse"], ws)
    with pytest.raises(ValueError, match="device"):
        wp.q4_append_kv(p, rows, rows, pool, pool, ws)
    with pytest.raises(ValueError, match="q4_plan"):
        wp.q4_append_kv(bf, rows, rows, pool, pool, ws)
    with pytest.raises(ValueError):
        wp.q4_read_kv(p, pool, pool, rows, None, ws)
