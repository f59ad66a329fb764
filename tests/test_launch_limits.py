"""Waves that one launch cannot have threads for: refused by name before anything is enqueued (no GPU)."""
import numpy as np
import pytest

import paper_2609_35263_amd as wp

FAKE = 1 << 20          # stands for a device address: nothing is launched on it
UNSUPPORTED, NOT_UPLOADED = -2, -1


def plan(T, kv=1, group=1):
    n = T // 64
    return wp.q8_plan(num_q_heads=kv * group, num_kv_heads=kv, head_dim_qk=64, head_dim_v=64, page_size=64, num_pages=n, softmax_scale=0.1,
                      prefix_lens=[0], chunk_lens=[T], block_table=np.arange(n)[None])


def call(fn, p, n):
    return getattr(wp.load_library(), fn)(p.handle, *[FAKE] * n, FAKE, p.workspace_bytes, None)


def turn(p):
    r = wp.Rope(rot_dim=64)
    step, rows = p.shape["num_q_heads"] * 64, 1 << 40          # (apart from the workspace)
    return wp.load_library().wavepp_rope_apply(r.handle, p.handle, rows, step, None, 0, rows, step, None, 0, None, FAKE, p.workspace_bytes, None)


@pytest.mark.parametrize("T,status", [((1 << 24) - 64, NOT_UPLOADED), (1 << 24, UNSUPPORTED), ((1 << 24) + 640, UNSUPPORTED)])
def test_rotary_positions_of_too_many_tokens(T, status):
    assert turn(plan(T)) == status
    assert (b"tokens" if status == UNSUPPORTED else b"upload") in wp.load_library().wavepp_last_error()


@pytest.mark.parametrize("T,status", [((1 << 22) - 64, NOT_UPLOADED), (1 << 22, UNSUPPORTED)])
def test_appends_and_reads_of_too_many_blocks(T, status):
    p = plan(T, kv=128)                      # T / 64 fours of blocks, 2 * 128 workgroups for each
    for fn in ("wavepp_q8_append_kv", "wavepp_q8_read_kv"):
        assert call(fn, p, 4) == status
        assert (b"blocks" if status == UNSUPPORTED else b"upload") in wp.load_library().wavepp_last_error()
    assert call("wavepp_q8_chunked_prefill", p, 5) == NOT_UPLOADED


@pytest.mark.parametrize("T,status", [((1 << 20) - 64, NOT_UPLOADED), (1 << 20, UNSUPPORTED)])
def test_attention_of_too_many_items(T, status):
    p = plan(T, kv=128, group=16)            # T / 16 items of 256 rows a KV head
    assert call("wavepp_q8_chunked_prefill", p, 5) == status
    assert (b"tiles" if status == UNSUPPORTED else b"upload") in wp.load_library().wavepp_last_error()
    assert call("wavepp_q8_append_kv", p, 4) == NOT_UPLOADED
