"""Which buffers of a rotary call overlap, byte by byte, and which only lie between each other's rows (no GPU)."""
import numpy as np
import pytest

import paper_2609_35263_amd as wp

BASE, WS = 1 << 20, 1 << 26
ALIAS, PASSED = -4, -1          # a call that passes every check ends at its plan's missing upload
HEADS, DIM = 4, 64
WIDTH = HEADS * DIM             # elements of a token's rows


def call(q, q_stride, out, out_stride, T=6, ws=WS):
    p = wp.plan(num_q_heads=HEADS, num_kv_heads=HEADS, head_dim_qk=DIM, head_dim_v=DIM, page_size=16, num_pages=4, softmax_scale=1.0,
                prefix_lens=[3], chunk_lens=[T], block_table=[[0, 1, 2, 3]])
    r = wp.Rope(rot_dim=DIM)
    lib = wp.load_library()
    st = lib.wavepp_rope_apply(r.handle, p.handle, q, q_stride, None, 0, out, out_stride, None, 0, None, ws, p.workspace_bytes, None)
    assert st != PASSED or b"upload" in lib.wavepp_last_error(), lib.wavepp_last_error()
    return st


def share(q, q_stride, out, out_stride, T):
    rows = [set(a + 2 * (i * s + n) for i in range(T) for n in range(WIDTH)) for a, s in ((q, q_stride), (out, out_stride))]
    return bool(rows[0] & rows[1])


@pytest.mark.parametrize("seed", range(40))
def test_rows_of_unlike_strides(seed):
    """Rows that lie in each other's gaps share nothing, whatever their strides."""
    rng = np.random.default_rng(seed)
    for _ in range(10):
        T = int(rng.integers(1, 7))
        q_stride, out_stride = (int(WIDTH + 8 * rng.integers(0, 200)) for _ in range(2))
        out = BASE + 16 * int(rng.integers(-300, 300))
        if out == BASE and (q_stride == out_stride or T == 1):
            continue
        assert (call(BASE, q_stride, out, out_stride, T) == ALIAS) == share(BASE, q_stride, out, out_stride, T)


def test_rows_in_each_others_gaps_are_taken():
    assert call(BASE, 4 * WIDTH, BASE + 2 * WIDTH, 8 * WIDTH) == PASSED
    assert call(BASE, 4 * WIDTH, BASE + 2 * WIDTH, 7 * WIDTH) == ALIAS           # the second row of one, the third of the other
    assert call(BASE, 4 * WIDTH, BASE, 8 * WIDTH) == ALIAS


def test_an_output_over_the_uploaded_plan_is_refused():
    """The kernels read the plan from the workspace while they write."""
    assert call(BASE, WIDTH, WS, WIDTH) == ALIAS
    assert call(WS, WIDTH, WS, WIDTH) == ALIAS                                   # in place as well
    assert call(BASE, WIDTH, WS - 2 * WIDTH, WIDTH) == ALIAS
    assert call(BASE, WIDTH, WS - 12 * WIDTH, WIDTH) == PASSED                   # ends where the workspace begins
    assert call(BASE, WIDTH, WS + (1 << 20), WIDTH) == PASSED
    assert call(BASE, WIDTH, WS - 2 * WIDTH, 64 * WIDTH) == PASSED               # rows on both sides of it
