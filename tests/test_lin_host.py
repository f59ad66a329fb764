"""Host side of linear attention: what plans refuse, how chunks are cut, and the checks of a call's buffers (no GPU)."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2609_35263_amd as wp

FAKE = 1 << 20          # stands for a device address: nothing is launched on it


def kw(**over):
    base = dict(num_heads=8, num_qk_heads=4, head_dim_k=128, head_dim_v=64, num_state_slots=6, chunk_lens=[1, 0, 70],
                state_in=[0, 9, -1], state_out=[0, 9, 2])
    return {**base, **over}


@pytest.mark.parametrize("over,status", [
    (dict(num_heads=0), -1), (dict(num_heads=65536, num_qk_heads=1), -1), (dict(num_qk_heads=3), -1), (dict(num_qk_heads=16), -1), (dict(scale=float("nan")), -1),
    (dict(scale=float("inf")), -1), (dict(chunk_lens=[1, 0, -1]), -1), (dict(head_dim_k=96), -2), (dict(head_dim_v=256), -2),
    (dict(state_in=[6, 0, -1]), -3), (dict(state_in=[-2, 0, -1]), -3), (dict(state_out=[0, 0, 6]), -3),
    (dict(state_out=[-1, 0, 2]), -3), (dict(state_out=[2, 0, 2]), -4), (dict(state_in=[2, 0, -1]), -4),
    (dict(chunk_lens=[2 ** 30, 2 ** 30, 2 ** 30], state_in=[-1] * 3, state_out=[0, 1, 2]), -1),
])
def test_plans_refuse(over, status):
    with pytest.raises(wp.WaveppError) as e:
        wp.lin_plan(**kw(**over))
    assert e.value.status == status


def test_plan_of_both_forms():
    i = wp.lin_plan(**kw()).info()
    assert (i["total_tokens"], i["num_step_items"], i["num_segments"], i["num_partials"]) == (71, 1, 1, 0)
    assert wp.lin_plan(**kw(chunk_lens=[0, 0, 0])).info()["total_tokens"] == 0
    assert wp.lin_plan(**kw(chunk_lens=[10, 0, 11])).info()["num_step_items"] == 1
    assert wp.lin_plan(**kw(chunk_lens=[], state_in=[], state_out=[])).info()["num_segments"] == 0


def test_few_chains_are_cut_into_segments():
    one = dict(chunk_lens=[16384], state_in=[-1], state_out=[1])
    cut = wp.lin_plan(**kw(**one)).info()
    assert cut["num_segments"] > 8 and cut["num_partials"] == cut["num_segments"] - 1
    # resumed in place: one more partial state, for the start
    same = wp.lin_plan(**kw(**{**one, "state_in": [1]})).info()
    assert same["num_partials"] == cut["num_partials"] + 1
    assert same["workspace_bytes"] - same["metadata_bytes"] >= same["num_partials"] * 8 * 128 * 64 * 4
    assert wp.lin_plan(**kw(num_heads=512, **one)).info()["num_segments"] == 1


def call(plan, *bufs, ws=FAKE, size=None):
    size = plan.workspace_bytes if size is None else size
    return wp.load_library().wavepp_lin_chunked_prefill(plan.handle, *bufs, ws, size, None)


def test_calls_check_their_workspace_before_anything_is_enqueued():
    p, lib = wp.lin_plan(**kw()), wp.load_library()
    bufs = [FAKE] * 6
    assert call(p, *bufs, ws=None) == -1 and call(p, *bufs, ws=FAKE + 16) == -1
    assert call(p, *bufs, size=p.workspace_bytes - 1) == -6
    assert call(p, *bufs, ws=3 * FAKE) == -1 and b"wavepp_lin_upload" in lib.wavepp_last_error()
    assert lib.wavepp_lin_chunked_prefill(None, *bufs, FAKE, 1 << 20, None) == -1
    assert call(wp.lin_plan(**kw(chunk_lens=[0, 0, 0])), *[None] * 6) == 0
    out = ctypes.c_void_p(5)
    assert lib.wavepp_lin_plan(None, None, ctypes.byref(out)) == -1


def test_the_binding_checks_shapes_and_types():
    p = wp.lin_plan(**kw())
    bf = dict(dtype=torch.bfloat16)
    good = dict(q=torch.zeros(71, 4, 128, **bf), k=torch.zeros(71, 4, 128, **bf), v=torch.zeros(71, 8, 64, **bf),
                alpha=torch.zeros(71, 8), state_pool=torch.zeros(6, 8, 128, 64), out=torch.zeros(71, 8, 64, **bf))
    ws = torch.zeros(4096, dtype=torch.uint8)
    for name in good:
        for bad in (None, good[name][:-1]):
            with pytest.raises(ValueError, match=name):
                wp.lin_chunked_prefill(p, **{**good, name: bad}, workspace=ws)
    with pytest.raises(ValueError, match="alpha"):
        wp.lin_chunked_prefill(p, **{**good, "alpha": torch.zeros(8)}, workspace=ws)
    with pytest.raises(ValueError, match="device"):
        wp.lin_chunked_prefill(p, **good, workspace=ws)
    with pytest.raises(ValueError):
        wp.lin_plan(**kw(state_in=[0]))
