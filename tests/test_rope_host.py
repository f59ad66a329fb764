"""Host side of rotary positions: frequencies, refused specs, and the checks of a call's buffers (no GPU)."""
import ctypes

import numpy as np
import pytest
import torch

import oracle
import paper_2609_35263_amd as wp

FAKE = 1 << 20          # stands for a device address: nothing is launched on it


@pytest.mark.parametrize("rot,base", [(2, 1e4), (64, 1e4), (128, 5e5), (48, 1.5), (256, 1e6)])
@pytest.mark.parametrize("scaling", [{}, {"scaling": "linear", "factor": 4.0}, {"scaling": "linear", "factor": 0.5}] + [
    {"scaling": s, "factor": f, "original_length": n, "slow_turns": a, "fast_turns": b}
    for s in ("turns", "index") for f, n, a, b in ((8.0, 8192, 1.0, 4.0), (40.0, 4096, 1.0, 32.0), (2.0, 10, 3.0, 900.0))])
def test_frequencies_against_the_oracle(rot, base, scaling):
    f = wp.Rope(rot_dim=rot, base=base, **scaling).frequencies()
    want = oracle.rope.frequencies(rot, base, **scaling)
    assert f.shape == want.shape and (np.abs(f - want) <= 1e-14 * want).all()


GOOD = dict(rot_dim=64, base=1e4, scaling="turns", factor=2.0, original_length=4096, slow_turns=1.0, fast_turns=4.0)


@pytest.mark.parametrize("over,status", [
    (dict(rot_dim=0), -1), (dict(rot_dim=63), -1), (dict(rot_dim=-2), -1), (dict(rot_dim=258), -2), (dict(rot_offset=-1), -1),
    (dict(base=1.0), -1), (dict(base=float("nan")), -1), (dict(base=float("inf")), -1), (dict(factor=0.0), -1), (dict(factor=-1.0), -1),
    (dict(original_length=0.0), -1), (dict(slow_turns=0.0), -1), (dict(slow_turns=4.0), -1), (dict(fast_turns=float("inf")), -1),
    (dict(magnitude=0.0), -1), (dict(magnitude=float("nan")), -1), (dict(magnitude=1e39), -1), (dict(magnitude=1e-60), -1),
    (dict(frequencies=[1.0] * 31 + [float("inf")]), -1),
])
def test_specs_that_are_refused(over, status):
    with pytest.raises(wp.WaveppError) as e:
        wp.Rope(**{**GOOD, **over})
    assert e.value.status == status


def test_the_binding_refuses_unknown_scalings_and_tables_of_another_length():
    for bad in (dict(scaling="dynamic"), dict(frequencies=[1.0] * 31), dict(frequencies=[[1.0] * 32])):
        with pytest.raises(ValueError):
            wp.Rope(**{**GOOD, **bad})
    out = ctypes.c_void_p(5)
    lib = wp.load_library()
    assert lib.wavepp_rope_create(None, ctypes.byref(out)) == -1
    assert lib.wavepp_rope_frequencies(None, None, 0) == -1
    r = wp.Rope(rot_dim=8)
    assert lib.wavepp_rope_frequencies(r.handle, None, 0) == 0 and lib.wavepp_rope_frequencies(r.handle, None, 3) == -1
    spec = wp._RopeSpec(8, 0, 0, 7, 1e4, 1.0, 0.0, 0.0, 0.0, 1.0, None)
    assert lib.wavepp_rope_create(ctypes.byref(spec), ctypes.byref(out)) == -1 and out.value is None
    r.destroy()
    with pytest.raises(ValueError):
        r.handle


def plan(T=4, **over):
    return wp.plan(**{**dict(num_q_heads=4, num_kv_heads=2, head_dim_qk=64, head_dim_v=64, page_size=16, num_pages=4, softmax_scale=1.0,
                             prefix_lens=[3], chunk_lens=[T], block_table=[[0, 1, 2, 3]]), **over})


Q, K = 4 * 64, 2 * 64          # elements of a token's rows


def apply(q=FAKE, qs=Q, k=FAKE + (1 << 16), ks=K, qo=FAKE + (2 << 16), qos=Q, ko=FAKE + (3 << 16), kos=K, positions=None, p=None, rope=None,
          ws=1 << 24, size=None, uploaded=True):
    """The status of a call, with WAVEPP_EHIP for one that passes every check (there is no device to launch on)."""
    p, rope = p or plan(), rope or wp.Rope(rot_dim=64)
    lib = wp.load_library()
    return lib.wavepp_rope_apply(rope.handle, p.handle, q, qs, k, ks, qo, qos, ko, kos, positions, ws, p.workspace_bytes if size is None else size, None)


def test_calls_check_the_rope_the_plan_and_the_workspace_first():
    lib = wp.load_library()
    assert apply(ws=None) == -1 and apply(ws=(1 << 24) + 16) == -1 and apply(size=100) == -6
    assert apply(rope=wp.Rope(rot_dim=64, rot_offset=1)) == -1 and b"head dim" in lib.wavepp_last_error()
    assert apply(rope=wp.Rope(rot_dim=128)) == -1
    assert apply(rope=wp.Rope(rot_dim=2, rot_offset=2 ** 31 - 1)) == -1
    assert apply() == -1 and b"wavepp_attn_plan_upload" in lib.wavepp_last_error()
    p, r = plan(), wp.Rope(rot_dim=64)
    assert lib.wavepp_rope_apply(None, p.handle, *[0] * 8, None, 1 << 24, 1 << 20, None) == -1
    assert lib.wavepp_rope_apply(r.handle, None, *[0] * 8, None, 1 << 24, 1 << 20, None) == -1
    assert apply(p=plan(T=0), q=None, k=None, qo=None, ko=None) == 0          # an idle wave needs nothing


def test_the_binding_checks_shapes_types_strides_and_pairs():
    p, r = plan(), wp.Rope(rot_dim=64)
    q, k = torch.zeros(4, 4, 64, dtype=torch.bfloat16), torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    ws = torch.zeros(1 << 14, dtype=torch.uint8)
    for a in ((q, k, None, k), (q, k, q, None), (None, k, q, k)):
        with pytest.raises(ValueError, match="together"):
            wp.rope_apply(r, p, *a, ws)
    with pytest.raises(ValueError, match="device"):
        wp.rope_apply(r, p, q, k, q, k, ws)
    rows = wp._row_args                                     # (the checks of a tensor, here of one that is on no device)
    with pytest.raises(ValueError, match="shape"):
        rows(-1, "q", q[:3], (4, 4, 64), torch.bfloat16)
    with pytest.raises(ValueError, match="bfloat16"):
        rows(-1, "q", q.float(), (4, 4, 64), torch.bfloat16)
    with pytest.raises(ValueError, match="contiguous"):
        rows(-1, "q", torch.zeros(4, 4, 128, dtype=torch.bfloat16)[..., ::2], (4, 4, 64), torch.bfloat16)
    with pytest.raises(ValueError, match="contiguous"):
        rows(-1, "q", torch.zeros(4, 8, 64, dtype=torch.bfloat16)[:, ::2], (4, 4, 64), torch.bfloat16)
    assert rows(-1, "q", torch.zeros(4, 9, 64, dtype=torch.bfloat16)[:, :4], (4, 4, 64), torch.bfloat16)[1] == 9 * 64
    assert rows(-1, "q", q[:1], (1, 4, 64), torch.bfloat16)[1] == Q
