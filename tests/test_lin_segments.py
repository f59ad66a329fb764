"""The segmented waves of ``test_gpu_lin_segments.py`` are cut, and their bounds tell a wrong carry from a right one (no GPU)."""
import numpy as np
import pytest

import oracle
import paper_2609_35263_amd as wp
import workloads as wl
from tests.test_gpu_lin import DIMS, make
from tests.test_gpu_lin_segments import HEADS, reference, wave


def waves():
    for dk, dv in DIMS:
        for H, Hqk in HEADS:
            for per_token in (True, False):
                yield wave(dk, dv, H, Hqk, per_token)[0]
        yield wave(dk, dv, 8, 2, True, zeros=True)[0]
        for per_token in (True, False):
            yield make([833, 449, 191], [-1, 1, 2], [0, 1, 3], 8, 4, dk, dv, seed=83, per_token=per_token, decay="hard")[0]
    for dv, Hqk in ((64, 4), (64, 16), (128, 16)):
        yield wave(64, dv, 16, Hqk, True, lens=[1500] + [11] * 63, s_in=list(range(64)), s_out=list(range(64)))[0]


def test_every_wave_is_cut():
    for args in waves():
        assert wp.lin_plan(**args).info()["num_partials"] >= 3, args


def segments(args, t, piece, rule):
    """The wave in pieces of a chunk, each by the oracle from what `rule` makes of (its start before, the piece's own state, the
    product of its decays): (out, pool)."""
    q, k, v = (wl.to_bits(t[n]) for n in ("q", "k", "v"))
    H = v.shape[1]
    alpha = np.broadcast_to(t["alpha"].numpy().astype(np.float64), (len(v), H))
    pool = t["state_pool"].numpy().astype(np.float64)
    out, after, at = np.zeros(v.shape), pool.copy(), 0
    for c, i, o in zip(args["chunk_lens"], args["state_in"], args["state_out"]):
        start = pool[i].copy() if i >= 0 else np.zeros(pool.shape[1:])
        for lo in range(at, at + c, piece):
            p = slice(lo, min(lo + piece, at + c))
            n = p.stop - p.start
            both = np.stack((start, np.zeros_like(start)))
            out[p], end = oracle.lin.chunked_prefill(q[p], k[p], v[p], alpha[p], both, [n], [0], [0], args["scale"])
            if p.stop == at + c:
                after[o] = end[0]
            own = oracle.lin.chunked_prefill(q[p], k[p], v[p], alpha[p], both, [n], [1], [1], args["scale"])[1][1]
            start = rule(start, own, alpha[p].prod(axis=0)[:, None, None])
        at += c
    return out, after


RULES = {
    "right": lambda start, own, decay: decay * start + own,
    "no carry": lambda start, own, decay: own,
    "no decay": lambda start, own, decay: start + own,
    "no own state": lambda start, own, decay: decay * start,
}


@pytest.mark.parametrize("per_token", [True, False])
@pytest.mark.parametrize("rule", sorted(RULES))
def test_the_bounds_tell_a_wrong_carry(rule, per_token):
    args, t = wave(64, 64, 4, 4, per_token)
    o, pool, bound, bounds = reference(args, t)
    out, after = segments(args, t, 128, RULES[rule])
    err = np.abs(out - o) / bound
    states = {s: (np.abs(after[s] - pool[s]) / bounds[s]).max() for s in bounds}
    if rule == "right":
        assert err.max() < 1e-6 and max(states.values()) < 1e-6
    else:
        assert err[256:900].max() > 1 and err[900 + 256:1300].max() > 1       # behind the second piece of the long chunks
        assert err[:128].max() < 1e-6                                      # the first piece has no carry
        assert states[0] > 100 and states[5] > 100


def test_the_bounds_tell_a_lost_start():
    args, t = wave(64, 64, 4, 4, True)
    o, _, bound, _ = reference(args, t)
    lost = {**t, "state_pool": t["state_pool"].clone()}
    lost["state_pool"][0] = 0.0
    out = reference(args, lost)[0]
    assert (np.abs(out - o) / bound)[800:900].max() > 2   # 800 tokens and six segments later
