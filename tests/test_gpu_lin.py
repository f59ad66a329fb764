"""Linear attention with a decay for each head on the GPU against its fp64 oracle, through the C ABI.

Tolerances, fixed before the first run, per element and in units of the same sums over absolute values ("size"):
  * States.  Token by token, every update is an fp32 product and sum: 2^-24 a token of what it adds up, under 2^-19
    over the lengths here.  In blocks, a weighted value keeps its 24 bits, its weight is a product of up to 64 decays
    (2^-24 each, 2^-18), and the sums run over up to 64 blocks of three products of 64 in fp32 (2^-17): under 2^-16
    together.  The bound is 2^-15, and 2^-18 for token by token.
  * Outputs.  Token by token: fp32, rounded to bf16 once (2^-8 of |o| <= size).  In blocks the state as it is read and
    the weights inside a block are rounded to bf16 besides (2^-8 of their terms): 2^-7 of size, and a tenth for the rest.
"""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_35263_amd as wp
import workloads as wl

pytestmark = pytest.mark.gpu

DIMS = [(128, 128), (128, 64), (64, 128), (64, 64)]


def make(lens, s_in, s_out, H, Hqk, dk, dv, seed, per_token=True, decay="mixed", slots=None):
    g = torch.Generator().manual_seed(seed)
    T = int(sum(lens))
    slots = max([0] + [x + 1 for x in list(s_in) + list(s_out)]) if slots is None else slots

    def bf(*shape):
        return torch.randn(shape, generator=g).to(torch.bfloat16)

    shape = (T, H) if per_token else (H,)
    if decay == "mixed":                            # from 0.998 to 0.5 a token, by head
        rate = torch.exp(torch.empty(H).uniform_(np.log(1 / 256), np.log(0.5), generator=g))
        alpha = torch.exp(-rate * torch.nn.functional.softplus(torch.randn(shape, generator=g)))
    elif decay == "hard":                           # zeros, denormals, ones, tiny and ordinary decays side by side
        kinds = torch.tensor([0.0, 1e-40, 1e-30, 1e-4, 0.5, 0.999, 1.0, 1.0])
        alpha = kinds[torch.randint(0, 8, shape, generator=g)]
        alpha = torch.where(torch.rand(shape, generator=g) < 0.7, torch.tensor(0.99), alpha)
    else:
        alpha = torch.full(shape, float(decay))
    pool = torch.full((slots, H, dk, dv), float("nan"))
    for r, c in enumerate(lens):
        if c and s_in[r] >= 0:
            pool[s_in[r]] = torch.randn((H, dk, dv), generator=g)
    t = {"q": bf(T, Hqk, dk), "k": bf(T, Hqk, dk), "v": bf(T, H, dv), "alpha": alpha, "state_pool": pool}
    args = dict(num_heads=H, num_qk_heads=Hqk, head_dim_k=dk, head_dim_v=dv, num_state_slots=slots, chunk_lens=lens,
                state_in=s_in, state_out=s_out, scale=dk ** -0.5, alpha_per_token=per_token)
    return args, t


def on_gpu(args, t, plan=None, ws=None):
    d = {n: x.cuda() for n, x in t.items()}
    p = plan or wp.lin_plan(**args)
    if ws is None:
        ws = wp.new_workspace(p)
        wp.lin_upload(p, ws)
    out = torch.full_like(d["v"], float("nan"))
    wp.lin_chunked_prefill(p, d["q"], d["k"], d["v"], d["alpha"], d["state_pool"], out, ws)
    torch.cuda.synchronize()
    return {**d, "out": out, "plan": p, "ws": ws}


def same(a, b):
    return bool(torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8)))


def check(args, t, g, what="", finite=None):
    ref = [wl.to_bits(t[n]) for n in ("q", "k", "v")] + [t["alpha"].numpy(), t["state_pool"].numpy(), args["chunk_lens"],
                                                         args["state_in"], args["state_out"], args["scale"]]
    o, pool = oracle.lin.chunked_prefill(*ref)
    size, psize = oracle.lin.sizes(*ref)
    lens = np.asarray(args["chunk_lens"])
    blocks = np.repeat(lens > 10, lens)[:, None, None]
    bound = np.where(blocks, 1.1 * 2.0 ** -7, 1.02 * 2.0 ** -8) * size + 1e-30
    err = np.abs(g["out"].float().cpu().numpy().astype(np.float64) - o)
    assert (err <= bound).all(), (what, (err / bound).max())
    got = g["state_pool"].cpu()
    worst = 0.0
    written = {int(s): int(c) for s, c in zip(args["state_out"], lens) if c}
    for s in range(got.shape[0]):
        if s in written:
            b = (2.0 ** -15 if written[s] > 10 else 2.0 ** -18) * psize[s] + 1e-30
            e = np.abs(got[s].numpy().astype(np.float64) - pool[s])
            assert (e <= b).all(), (what, s, (e / b).max())
            worst = max(worst, (e / b).max())
        else:
            assert same(got[s], t["state_pool"][s]), f"slot {s} changed"
    print(f"[lin] {what}: out {(err / bound).max() if err.size else 0:.2f} of its bound, states {worst:.2f}", flush=True)


@pytest.mark.parametrize("dk,dv", DIMS)
@pytest.mark.parametrize("H,Hqk", [(4, 4), (6, 2), (5, 1), (8, 2)])
@pytest.mark.parametrize("per_token", [True, False])
def test_chunks_of_all_lengths(dk, dv, H, Hqk, per_token):
    lens = [1, 63, 0, 64, 65, 2, 10, 11, 130, 200, 1]
    s_in = [0, -1, 3, 1, 2, 3, -1, 4, 5, -1, 6]
    s_out = [0, 7, 3, 1, 8, 3, 9, 10, 11, 12, 6]
    args, t = make(lens, s_in, s_out, H, Hqk, dk, dv, seed=41, per_token=per_token, slots=14)
    check(args, t, on_gpu(args, t), f"{dk}x{dv} {H}/{Hqk}")


@pytest.mark.parametrize("dk,dv", DIMS)
def test_decays_of_zero_and_near_it(dk, dv):
    args, t = make([300, 5, 64], [0, 1, -1], [0, 1, 2], 7, 7, dk, dv, seed=42, decay="hard")
    check(args, t, on_gpu(args, t), "hard decays")


@pytest.mark.parametrize("decay", [0.0, 1.0, 1e-38])
def test_constant_decays(decay):
    args, t = make([150, 9], [0, 1], [0, 1], 2, 1, 128, 128, seed=43, per_token=False, decay=decay)
    check(args, t, on_gpu(args, t), f"decay {decay}")


@pytest.mark.parametrize("H,lens,s_in,s_out", [(2, [3000], [0], [0]), (3, [2000, 700, 12], [-1, 1, 2], [3, 1, 2]),
                                               (1, [4097], [-1], [0])])
def test_segments(H, lens, s_in, s_out):
    args, t = make(lens, s_in, s_out, H, 1, 128, 64, seed=44)
    g = on_gpu(args, t)
    assert g["plan"].info()["num_partials"] > 0
    check(args, t, g, "segments")


def test_many_heads_and_requests():
    args, t = make([70] * 9 + [1] * 9, list(range(18)), list(range(18)), 32, 8, 128, 64, seed=45)
    check(args, t, on_gpu(args, t), "many")


def test_chunk_by_chunk_and_token_by_token_equal_one_run():
    """A prompt in three waves and then ten single tokens on one plan, each resuming in place from the GPU's own state."""
    H, Hqk, dk, dv, lens = 4, 2, 128, 128, [100, 17, 64]
    n = sum(lens) + 10
    args, t = make([n], [-1], [0], H, Hqk, dk, dv, seed=46)
    ref = [wl.to_bits(t[x]) for x in ("q", "k", "v")] + [t["alpha"].numpy(), np.zeros((1, H, dk, dv)), [n], [-1], [0], args["scale"]]
    o, pool = oracle.lin.chunked_prefill(*ref)
    size, psize = oracle.lin.sizes(*ref)
    d = {x: t[x].cuda() for x in t}
    state = torch.full((1, H, dk, dv), float("nan"), device="cuda")
    got, at = [], 0
    step = None
    for i, c in enumerate(lens + [1] * 10):
        if c > 1 or step is None:
            p = wp.lin_plan(**{**args, "chunk_lens": [c], "state_in": [0 if i else -1]})
            ws = wp.new_workspace(p)
            wp.lin_upload(p, ws)
            step = p if c == 1 else None
        out = torch.empty(c, H, dv, dtype=torch.bfloat16, device="cuda")
        wp.lin_chunked_prefill(p, *(d[x][at:at + c].contiguous() for x in ("q", "k", "v", "alpha")), state, out, ws)
        got.append(out.float().cpu().numpy())
        at += c
    assert (np.abs(np.concatenate(got) - o) <= 1.1 * 2.0 ** -7 * size).all()
    assert (np.abs(state.cpu().numpy() - pool) <= 2.0 ** -15 * psize).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("name", ["q", "k", "v", "alpha"])
def test_tokens_before_a_bad_number_are_as_without_it(name, bad):
    lens = [200, 9, 90]
    args, t = make(lens, [-1, 0, 1], [2, 3, 1], 3, 3, 128, 64, seed=47)
    a = on_gpu(args, t)
    spoiled = {n: x.clone() for n, x in t.items()}
    for at in (75, 203, 290):                       # in the second block, in a token-by-token chunk, in a last block
        spoiled[name][at] = bad
    b = on_gpu(args, spoiled)
    clean = np.ones(sum(lens), dtype=bool)
    for lo, hi in ((75, 76 if name == "q" else 200), (203, 204 if name == "q" else 209), (290, 291 if name == "q" else 299)):
        clean[lo:hi] = False
    x, y = (g["out"].float().cpu().numpy()[clean] for g in (a, b))
    assert np.isfinite(y).all()
    ref = [wl.to_bits(t[n]) for n in ("q", "k", "v")] + [t["alpha"].numpy(), t["state_pool"].numpy(), lens, args["state_in"],
                                                         args["state_out"], args["scale"]]
    size = oracle.lin.sizes(*ref)[0][clean]
    assert (np.abs(x - y) <= 2.2 * 2.0 ** -7 * size).all()
    gone = b["out"].float().cpu().numpy()[[75, 203, 290]]
    assert not np.isfinite(gone).any()


@pytest.mark.parametrize("dv", [64, 128])
def test_a_bad_number_of_one_head_leaves_the_others_alone(dv):
    """Heads that share q and k: a value or a decay of one that is not finite changes no bit of another's."""
    args, t = make([200, 9, 90], [-1, 0, 1], [2, 3, 1], 4, 2, 128, dv, seed=54)
    a = on_gpu(args, t)
    for name, head in (("v", 0), ("v", 3), ("alpha", 1), ("alpha", 2)):
        spoiled = {n: x.clone() for n, x in t.items()}
        for at in (3, 75, 203, 290):
            spoiled[name][at, head] = float("nan") if at != 75 else float("inf")
        b = on_gpu(args, spoiled)
        rest = [h for h in range(4) if h != head]
        assert same(a["out"][:, rest], b["out"][:, rest]) and same(a["state_pool"][:, rest], b["state_pool"][:, rest])
        assert not torch.isfinite(b["out"][75, head].float()).any()


def test_repeated_calls_are_bit_identical_and_stale_workspaces_write_nothing():
    args, t = make([700, 1, 3], [-1, 1, 2], [0, 3, 4], 2, 2, 128, 128, seed=48)
    a, b = on_gpu(args, t), on_gpu(args, t)
    assert a["plan"].info()["num_partials"] > 0
    assert same(a["out"], b["out"]) and same(a["state_pool"], b["state_pool"])
    a["ws"].zero_()
    pool, out = t["state_pool"].cuda(), torch.zeros_like(a["out"])
    wp.lin_chunked_prefill(a["plan"], a["q"], a["k"], a["v"], a["alpha"], pool, out, a["ws"])
    assert not out.view(torch.int16).any() and same(pool.cpu(), t["state_pool"])


def test_graph_replays_match_eager():
    """A wave with segments and single tokens captured once and replayed on new inputs, eager work in between."""
    cases = [make([900, 1, 40], [-1, 1, 2], [0, 1, 3], 2, 1, 128, 64, seed=50 + i) for i in range(3)]
    eager = [on_gpu(a, t) for a, t in cases]
    p, ws = eager[0]["plan"], eager[0]["ws"]
    buf = {n: x.cuda() for n, x in cases[0][1].items()}
    out = torch.empty_like(eager[0]["out"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        wp.lin_chunked_prefill(p, buf["q"], buf["k"], buf["v"], buf["alpha"], buf["state_pool"], out, ws)
    torch.cuda.synchronize()
    assert same(out, eager[0]["out"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        wp.lin_chunked_prefill(p, buf["q"], buf["k"], buf["v"], buf["alpha"], buf["state_pool"], out, ws)
    for i in (0, 1, 2, 1):
        for n, x in cases[i][1].items():
            buf[n].copy_(x)
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert same(out, eager[i]["out"]) and same(buf["state_pool"], eager[i]["state_pool"]), i


def test_idle_wave():
    args, t = make([0, 0], [0, 1], [1, 0], 2, 2, 64, 64, seed=53)
    g = on_gpu(args, t)
    assert g["out"].shape[0] == 0 and same(g["state_pool"].cpu(), t["state_pool"])
