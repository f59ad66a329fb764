"""Linear attention cut into segments, against its fp64 oracle, with decays that a state outlives: what one segment hands to the
next is most of what is there, so a carry, a decay or a start that is lost shows (``test_lin_segments.py`` plants those).

Tolerances, fixed before the first run, in units of the same sums over absolute values ("size").  States: 2^-15 as
in ``test_gpu_lin.py``, which counts one block's decays, and 2^-24 for each token of the chunk, since the product of all decays
that a number passes is rounded once a token.  Outputs: 1.1 * 2^-7 as there; that product is inside its tenth.
"""
import numpy as np
import pytest
import torch

import oracle
import workloads as wl
from tests.test_gpu_lin import DIMS, make, on_gpu, same

pytestmark = pytest.mark.gpu

# a wave: one chunk that resumes in place, one that leaves another slot, one block, single tokens, and one from nothing
LENS, S_IN, S_OUT = [900, 400, 64, 3, 330], [0, 1, 2, 3, -1], [0, 5, 2, 3, 4]
HEADS = [(4, 4), (6, 2), (8, 2)]                 # the last has two heads of 64 columns in a workgroup


def wave(dk, dv, H, Hqk, per_token, zeros=False, lens=LENS, s_in=S_IN, s_out=S_OUT, seed=81):
    """Inputs whose decays are 1, 0.9999 and 0.999, by head or by token and head, and states of thirty times a token's size."""
    args, t = make(lens, s_in, s_out, H, Hqk, dk, dv, seed=seed, per_token=per_token, decay=1.0)
    g = torch.Generator().manual_seed(seed + 1)
    kinds = torch.tensor([0.999, 1.0, 0.9999])
    if per_token:
        t["alpha"] = kinds[torch.randint(0, 3, t["alpha"].shape, generator=g)]
    else:
        t["alpha"] = kinds[torch.arange(H) % 3].clone()
    if zeros:                                    # inside a block, at its ends, and twice in one
        for at in (70, 300, 301, 447, 448, 899, 1000):
            t["alpha"][at, at % 2::2] = 0.0
    t["state_pool"] *= 30.0
    return args, t


def reference(args, t):
    """(out, pool, bounds of out, bounds of the pool's written slots)."""
    ref = [wl.to_bits(t[n]) for n in ("q", "k", "v")] + [t["alpha"].numpy(), t["state_pool"].numpy(), args["chunk_lens"],
                                                         args["state_in"], args["state_out"], args["scale"]]
    o, pool = oracle.lin.chunked_prefill(*ref)
    size, psize = oracle.lin.sizes(*ref)
    bounds = {s: (2.0 ** -15 + c * 2.0 ** -24) * psize[s] + 1e-30 for s, c in zip(args["state_out"], args["chunk_lens"])}
    return o, pool, 1.1 * 2.0 ** -7 * size + 1e-30, bounds


def check(args, t, g):
    assert g["plan"].info()["num_partials"] > 0
    o, pool, bound, bounds = reference(args, t)
    err = np.abs(g["out"].float().cpu().numpy().astype(np.float64) - o)
    assert (err <= bound).all(), (err / bound).max()
    got, worst = g["state_pool"].cpu(), 0.0
    for s in range(got.shape[0]):
        if s in bounds:
            e = np.abs(got[s].numpy().astype(np.float64) - pool[s]) / bounds[s]
            worst = max(worst, e.max())
            assert (e <= 1).all(), (s, e.max())
        else:
            assert same(got[s], t["state_pool"][s]), f"slot {s} changed"
    print(f"[lin] {g['plan'].info()['num_partials']} partial states: out {(err / bound).max():.2f}, states {worst:.2f}", flush=True)


@pytest.mark.parametrize("dk,dv", DIMS)
@pytest.mark.parametrize("H,Hqk", HEADS)
@pytest.mark.parametrize("per_token", [True, False])
def test_what_a_segment_hands_on(dk, dv, H, Hqk, per_token):
    args, t = wave(dk, dv, H, Hqk, per_token)
    check(args, t, on_gpu(args, t))


@pytest.mark.parametrize("dk,dv", DIMS)
def test_decays_of_zero_inside_segments(dk, dv):
    args, t = wave(dk, dv, 8, 2, True, zeros=True)
    check(args, t, on_gpu(args, t))


@pytest.mark.parametrize("dk,dv", DIMS)
@pytest.mark.parametrize("per_token", [True, False])
def test_hard_decays_and_chunks_of_odd_lengths(dk, dv, per_token):
    """Zeros, denormals and ones side by side, by token or by head, over segments that end in a token or lack one."""
    args, t = make([833, 449, 191], [-1, 1, 2], [0, 1, 3], 8, 4, dk, dv, seed=83, per_token=per_token, decay="hard")
    check(args, t, on_gpu(args, t))


@pytest.mark.parametrize("dv,Hqk", [(64, 4), (64, 16), (128, 16)])
def test_a_long_chunk_among_chains_that_fill_the_chip(dv, Hqk):
    n = 64
    args, t = wave(64, dv, 16, Hqk, True, lens=[1500] + [11] * (n - 1), s_in=list(range(n)), s_out=list(range(n)))
    check(args, t, on_gpu(args, t))


@pytest.mark.parametrize("name", ["k", "v", "alpha"])
@pytest.mark.parametrize("dv", [64, 128])
def test_a_bad_number_reaches_later_segments_of_its_head_alone(name, dv):
    """A number of token 500 that is not finite: earlier tokens, other requests and (of v and alpha) other heads keep their
    bits, every later token of the chunk and its state show it."""
    args, t = wave(64, dv, 8, 4, True)
    a = on_gpu(args, t)
    spoiled = {n: x.clone() for n, x in t.items()}
    spoiled[name][500, 1] = float("nan")
    b = on_gpu(args, spoiled)
    assert a["plan"].info()["num_partials"] > 0
    hit = [2, 3] if name == "k" else [1]                   # two heads share each key
    rest = [h for h in range(8) if h not in hit]
    assert same(a["out"][:, rest], b["out"][:, rest]) and same(a["state_pool"][:, rest], b["state_pool"][:, rest])
    clean = np.arange(len(a["out"])) < 500
    clean[900:] = True
    assert torch.isnan(b["out"][500:900][:, hit].float()).all() and torch.isnan(b["state_pool"][0][hit]).all()
    kept = clean.copy()
    kept[448:500] = False                                  # summed pair by pair there, so not bit by bit the same
    assert same(a["out"][kept], b["out"][kept]) and same(a["state_pool"][1:], b["state_pool"][1:])
    o, _, bound, _ = reference(args, t)
    assert (np.abs(b["out"].float().cpu().numpy() - o) <= bound)[clean].all()
