"""Rotary positions on the GPU against their fp64 oracle, through the C ABI.

Tolerance, fixed before the first run.  The angle is off by at most 2^-22 and 2^-52 of itself (the header's words; the positions
here keep the second under 2^-24), cos and sin in fp32 by two steps more, and each of the two products and the sum by half a
step of fp32; the output is rounded to bf16 once, half a step, 2^-8 of itself.  So with r = magnitude (|a| + |b|) a turned value
is off by no more than 2^-8 |y| + (2^-22 + 2^-24 + 8 * 2^-24) r.  Values that are not turned keep every bit.
"""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_35263_amd as wp
import workloads as wl

pytestmark = pytest.mark.gpu


def plan(q, kv, dim, prefix, chunk, cache="bf16", page=64):
    latent = dim == 576
    spec = wl.custom_wave(q, kv, dim, 512 if latent else dim, page, prefix, chunk, kv_shared=latent, seed=3)
    p = {"bf16": wp.plan_for, "q4": wp.q4_plan_for, "q8": wp.q8_plan_for}[cache](spec)
    ws = wp.new_workspace(p)
    wp.plan_upload(p, ws)
    return spec, p, ws


def rows(T, q, kv, dim, seed=1):
    gen = torch.Generator().manual_seed(seed)
    return [torch.randn(T, h, dim, generator=gen).to(torch.bfloat16).cuda() for h in (q, kv)]


def positions_of(spec):
    return np.concatenate([p + np.arange(c) for p, c in zip(spec.prefix_lens, spec.chunk_lens)]).astype(np.int64)


def same(a, b):
    return bool(torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8)))


def check(x, y, pos, rot, freqs, offset=0, interleaved=False, magnitude=1.0, what=""):
    x, got = x.cpu(), y.float().cpu().numpy().astype(np.float64)
    f = x.float().numpy().astype(np.float64)
    want = oracle.rope.turn(f, pos, freqs, offset, interleaved, np.float64(np.float32(magnitude)))
    part = np.abs(f[..., offset:offset + rot])
    n = rot // 2
    if interleaved:
        r = np.repeat(part[..., 0::2] + part[..., 1::2], 2, axis=-1)
    else:
        r = np.tile(part[..., :n] + part[..., n:], 2)
    bound = 2.0 ** -8 * np.abs(want[..., offset:offset + rot]) + 13 * 2.0 ** -24 * magnitude * r
    err = np.abs(got - want)[..., offset:offset + rot]
    print(f"[rope] {what}: {(err / np.maximum(bound, 1e-300)).max():.3f} of its bound", flush=True)
    assert (err <= bound).all()
    keep = np.ones(x.shape[-1], dtype=bool)
    keep[offset:offset + rot] = False
    assert same(x[..., keep], y.cpu()[..., keep])


SHAPES = [
    # q heads, KV heads, dim, turned values, offset
    (64, 8, 128, 128, 0), (32, 8, 128, 64, 64), (16, 1, 128, 32, 0), (24, 4, 64, 64, 0), (8, 2, 64, 16, 48), (128, 1, 576, 64, 512),
    (3, 1, 64, 48, 8), (5, 5, 128, 48, 80),
    (4, 2, 64, 2, 0), (4, 2, 64, 6, 3), (7, 1, 128, 22, 5), (2, 2, 64, 62, 1), (5, 1, 128, 128, 0), (16, 1, 576, 30, 511),
    (128, 1, 576, 256, 320),
]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("q,kv,dim,rot,offset", SHAPES)
def test_shapes_against_the_oracle(q, kv, dim, rot, offset, interleaved):
    """Into other buffers, in place, q alone and k alone: the same bits, with the values around the turned ones as they were."""
    spec, p, ws = plan(q, kv, dim, [0, 700, 100000, 0], [5, 1, 17, 0])
    pos = positions_of(spec)
    x = rows(len(pos), q, kv, dim)
    r = wp.Rope(rot_dim=rot, rot_offset=offset, interleaved=interleaved)
    out = [torch.full_like(a, float("nan")) for a in x]
    before = [a.clone() for a in x]
    wp.rope_apply(r, p, *x, *out, ws)
    torch.cuda.synchronize()
    assert all(same(a, b) for a, b in zip(x, before))
    for a, y, name in zip(x, out, "qk"):
        check(a, y, pos, rot, oracle.rope.frequencies(rot), offset, interleaved, what=f"{name} {q}/{kv} of {dim}, {rot} from {offset}")
    place = [a.clone() for a in x]
    wp.rope_apply(r, p, *place, *place, ws)
    alone = [torch.zeros_like(a) for a in x]
    wp.rope_apply(r, p, x[0], None, alone[0], None, ws)
    wp.rope_apply(r, p, None, x[1], None, alone[1], ws)
    half = [x[0].clone(), torch.zeros_like(x[1])]
    wp.rope_apply(r, p, half[0], x[1], *half, ws)
    torch.cuda.synchronize()
    for i in range(2):
        assert same(place[i], out[i]) and same(alone[i], out[i]) and same(half[i], out[i])


SCALINGS = [{"scaling": "linear", "factor": 4.0},
            {"scaling": "turns", "factor": 8.0, "original_length": 8192, "slow_turns": 1.0, "fast_turns": 4.0},
            {"scaling": "index", "factor": 32.0, "original_length": 4096, "slow_turns": 1.0, "fast_turns": 32.0, "magnitude": 1.35},
            {"magnitude": 0.5}]


@pytest.mark.parametrize("scaling", SCALINGS)
@pytest.mark.parametrize("base", [1e4, 5e5])
def test_scalings(scaling, base):
    spec, p, ws = plan(32, 8, 128, [0, 131071, 1000000], [40, 1, 3])
    pos = positions_of(spec)
    x = rows(len(pos), 32, 8, 128)
    r = wp.Rope(rot_dim=128, base=base, **scaling)
    out = [torch.empty_like(a) for a in x]
    wp.rope_apply(r, p, *x, *out, ws)
    f = oracle.rope.frequencies(128, base, **{n: v for n, v in scaling.items() if n != "magnitude"})
    for a, y in zip(x, out):
        check(a, y, pos, 128, f, magnitude=scaling.get("magnitude", 1.0), what=str(scaling))


@pytest.mark.parametrize("cache", ["bf16", "q4", "q8"])
@pytest.mark.parametrize("page", [16, 64])
def test_plans_of_every_cache_and_many_requests(cache, page):
    """More requests than lanes, idle ones among them: every token finds its own request."""
    rng = np.random.default_rng(5)
    for R in (1, 2, 63, 64, 65, 700, 4097):
        prefix, chunk = rng.integers(0, 90, R), rng.integers(0, 3, R)
        chunk[rng.integers(R)] = 7
        if R > 2:
            chunk[:2] = chunk[-2:] = 0
            chunk[R // 2] = 1
        spec, p, ws = plan(4, 2, 64, prefix, chunk, cache, page)
        pos = positions_of(spec)
        x = rows(len(pos), 4, 2, 64)
        r = wp.Rope(rot_dim=64)
        out = [torch.empty_like(a) for a in x]
        wp.rope_apply(r, p, *x, *out, ws)
        for a, y in zip(x, out):
            check(a, y, pos, 64, oracle.rope.frequencies(64), what=f"{R} requests, {cache}")


def test_given_positions_and_frequencies():
    """Any int32 position, negative and the extremes among them."""
    T = 64
    spec, p, ws = plan(4, 2, 64, [9], [T])
    pos = np.concatenate(([0, -1, 5, 2 ** 31 - 1, -2 ** 31, 10 ** 9], np.random.default_rng(6).integers(-10 ** 6, 10 ** 6, T - 6)))
    f = np.random.default_rng(7).uniform(-1.0, 1.0, 16) * 10.0 ** -np.arange(0, 8, 0.5)
    r = wp.Rope(rot_dim=32, rot_offset=8, frequencies=f)
    assert np.array_equal(r.frequencies(), f)
    x = rows(T, 4, 2, 64)
    out = [torch.empty_like(a) for a in x]
    at = torch.from_numpy(pos.astype(np.int32)).cuda()
    wp.rope_apply(r, p, *x, *out, ws, positions=at)
    # 2^-52 of an angle of 2^31 is 2^-21, so the far ones get that beside the rest
    near = np.abs(pos) < 2 ** 27
    for a, y in zip(x, out):
        check(a[torch.from_numpy(near)], y[torch.from_numpy(near)], pos[near], 32, f, 8, what="positions")
        want = oracle.rope.turn(a.float().cpu().numpy(), pos, f, 8)
        err = np.abs(y.float().cpu().numpy() - want)
        assert (err <= 2.0 ** -8 * np.abs(want) + 2.0 ** -17 * np.abs(a.float().cpu().numpy()).max()).all()
    # turned back by the opposite positions, every value is within two roundings of what it was
    back = [torch.empty_like(a) for a in x]
    keep = np.clip(pos, -2 ** 31 + 1, None)
    wp.rope_apply(r, p, *x, *out, ws, positions=torch.from_numpy(keep.astype(np.int32)).cuda())
    wp.rope_apply(r, p, *out, *back, ws, positions=torch.from_numpy(-keep.astype(np.int32)).cuda())
    for a, y in zip(x, back):
        a, y = a.float().cpu().numpy(), y.float().cpu().numpy()
        size = np.hypot(a[..., 8:24], a[..., 24:40])
        assert (np.abs(y - a)[..., 8:40] <= np.tile(2.1 * 2.0 ** -8 * 1.5 * size, 2)).all()


def test_infinities_and_nan_stay_in_their_pairs():
    spec, p, ws = plan(2, 1, 64, [3], [4])
    x = rows(4, 2, 1, 64)
    clean = [torch.empty_like(a) for a in x]
    r = wp.Rope(rot_dim=64)
    wp.rope_apply(r, p, *x, *clean, ws)
    bad = [a.clone() for a in x]
    bad[0][2, 1, 7], bad[1][1, 0, 40] = float("nan"), float("inf")
    out = [torch.empty_like(a) for a in x]
    wp.rope_apply(r, p, *bad, *out, ws)
    touched = [torch.zeros(a.shape, dtype=torch.bool) for a in x]
    touched[0][2, 1, [7, 39]] = True
    touched[1][1, 0, [8, 40]] = True
    for y, c, m in zip(out, clean, touched):
        assert same(y.cpu()[~m], c.cpu()[~m])
    assert torch.isnan(out[0].cpu()[touched[0]].float()).all() and not torch.isfinite(out[1].cpu()[touched[1]].float()).any()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot,offset", [(128, 0), (30, 9)])
def test_slices_of_a_packed_projection(rot, offset, interleaved):
    """q and k as slices of rows that hold q, k and v: in place, and out of it into other rows that lie apart."""
    q, kv, dim = 8, 2, 128
    spec, p, ws = plan(q, kv, dim, [11, 500], [33, 1])
    T = spec.total_tokens
    packed = torch.randn(T, q + 2 * kv, dim, generator=torch.Generator().manual_seed(8)).to(torch.bfloat16).cuda()
    first = packed.clone()
    r = wp.Rope(rot_dim=rot, rot_offset=offset, interleaved=interleaved)
    want = [torch.empty(T, h, dim, dtype=torch.bfloat16, device="cuda") for h in (q, kv)]
    wp.rope_apply(r, p, packed[:, :q].contiguous(), packed[:, q:q + kv].contiguous(), *want, ws)
    wide = torch.full((T, q + kv + 3, dim), 7.0, dtype=torch.bfloat16, device="cuda")
    wp.rope_apply(r, p, packed[:, :q], packed[:, q:q + kv], wide[:, :q], wide[:, q + 1:q + 1 + kv], ws)
    torch.cuda.synchronize()
    assert same(packed, first)
    assert same(wide[:, :q], want[0]) and same(wide[:, q + 1:q + 1 + kv], want[1])
    assert (wide[:, q] == 7.0).all() and (wide[:, q + 1 + kv:] == 7.0).all()
    wp.rope_apply(r, p, packed[:, :q], packed[:, q:q + kv], packed[:, :q], packed[:, q:q + kv], ws)
    assert same(packed[:, :q], want[0]) and same(packed[:, q:q + kv], want[1]) and same(packed[:, q + kv:], first[:, q + kv:])


def test_a_layers_step_captured_and_replayed():
    """Turn, store and attend, as a layer does them, on a side stream, then captured into one graph and replayed with new rows:
    against the oracle of each step on the step's own inputs, and every replay against the eager call."""
    q, kv, dim, page = 16, 2, 128, 64
    spec = wl.custom_wave(q, kv, dim, dim, page, [300, 77, 0], [1, 1, 6], seed=9)
    p = wp.q8_plan_for(spec, score_cap=30.0)
    ws = wp.new_workspace(p)
    wp.plan_upload(p, ws)
    r = wp.Rope(rot_dim=64, base=5e5)
    T, pos = spec.total_tokens, positions_of(spec)
    gen = torch.Generator().manual_seed(10)
    packed = [torch.randn(T, q + 2 * kv, dim, generator=gen).to(torch.bfloat16).cuda() for _ in range(3)]
    pools = [torch.from_numpy(oracle.q8.quantise_pool(np.random.default_rng(i).standard_normal((spec.num_pages, kv, page, dim)))).cuda()
             for i in range(2)]
    buf = torch.empty_like(packed[0])
    k_pool, v_pool = (torch.empty_like(x) for x in pools)
    turned = [torch.empty(T, h, dim, dtype=torch.bfloat16, device="cuda") for h in (q, kv)]
    v_new = torch.empty_like(turned[1])
    out, lse = torch.empty_like(turned[0]), torch.empty(T, q, device="cuda")

    def step():
        wp.rope_apply(r, p, buf[:, :q], buf[:, q:q + kv], *turned, ws)
        v_new.copy_(buf[:, q + kv:])
        wp.q8_append_kv(p, turned[1], v_new, k_pool, v_pool, ws)
        wp.q8_chunked_prefill(p, turned[0], k_pool, v_pool, out, lse, ws)

    def load(i):
        buf.copy_(packed[i])
        k_pool.copy_(pools[0])
        v_pool.copy_(pools[1])
        for t in (*turned, out):
            t.fill_(float("nan"))

    eager = []
    side = torch.cuda.Stream()
    for i in range(3):
        load(i)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        eager.append([t.clone() for t in (*turned, k_pool, v_pool, out, lse)])
    from tests.test_gpu_q8 import check as check_attention
    for i in range(3):
        tq, tk, kp, vp, o, l = eager[i]
        f = oracle.rope.frequencies(64, 5e5)
        check(packed[i][:, :q], tq, pos, 64, f, what="step q")
        check(packed[i][:, q:q + kv], tk, pos, 64, f, what="step k")
        t = {"q": tq.cpu(), "k_new": tk.cpu(), "v_new": packed[i][:, q + kv:].contiguous().cpu(), "k_pool": pools[0].cpu(), "v_pool": pools[1].cpu()}
        check_attention(spec, t, {"k_pool": kp, "v_pool": vp, "out": o, "lse": l}, "step", cap=30.0)
    load(0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in (0, 1, 2, 1):
        load(i)
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip((*turned, k_pool, v_pool, out, lse), eager[i]):
            assert same(got, want), i


def test_overlapping_and_misplaced_buffers_are_refused():
    """Outputs that share elements with another buffer, strides and addresses that the kernels cannot take: nothing is enqueued."""
    spec, p, ws = plan(4, 2, 64, [10], [6])
    r = wp.Rope(rot_dim=64)
    buf = torch.zeros(6, 40, 64, dtype=torch.bfloat16, device="cuda")
    q, k, q2, k2 = buf[:, 0:4], buf[:, 4:6], buf[:, 6:10], buf[:, 10:12]
    wp.rope_apply(r, p, q, k, q2, k2, ws)
    for a in ((q, k, buf[:, 1:5], k2), (q, k, buf[:, 3:7], k2), (q, k, q2, buf[:, 9:11]), (q, k, q2, buf[:, 3:5]), (q, k, k2.repeat(1, 2, 1), q[:, 1:3])):
        with pytest.raises(wp.WaveppError) as e:
            wp.rope_apply(r, p, *a, ws)
        assert e.value.status == -4, e.value
    flat = torch.zeros(8000, dtype=torch.bfloat16, device="cuda")
    other = torch.zeros(6, 4, 64, dtype=torch.bfloat16, device="cuda")
    for bad in (flat[1:1 + 6 * 256].view(6, 4, 64), flat.as_strided((6, 4, 64), (260, 64, 1)), flat.as_strided((6, 4, 64), (64, 64, 1))):
        with pytest.raises((wp.WaveppError, ValueError)):
            wp.rope_apply(r, p, bad, None, other, None, ws)
    lib = wp.load_library()
    step = buf.stride(0)
    for stride in (4 * 64 - 8, step + 4, 0, -step, 1 << 31, 1 << 62):
        for i in range(2):
            s = [step, step]
            s[i] = stride
            assert lib.wavepp_rope_apply(r.handle, p.handle, q.data_ptr(), s[0], None, 0, q2.data_ptr(), s[1], None, 0, None, ws.data_ptr(), ws.nbytes, None) == -1
            assert b"stride" in lib.wavepp_last_error()
    at = torch.zeros(6, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        wp.rope_apply(r, p, q, k, q2, k2, ws, positions=at[:5])
    with pytest.raises(ValueError):
        wp.rope_apply(r, p, q, k, q2, k2, ws, positions=at.long())
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        wp.rope_apply(r, p, q, k, q2, k2, ws, stream=side)
    torch.cuda.synchronize()
    assert not buf.any()


def test_idle_waves_and_overwritten_workspaces():
    spec, p, ws = plan(4, 2, 64, [10, 20], [0, 0])
    x = rows(0, 4, 2, 64)
    wp.rope_apply(wp.Rope(rot_dim=64), p, *x, *x, ws)
    spec, p, ws = plan(4, 2, 64, [10, 20], [3, 1])
    x = rows(4, 4, 2, 64)
    ws.zero_()
    for rot in (64, 6):
        out = [torch.zeros_like(a) for a in x]
        wp.rope_apply(wp.Rope(rot_dim=rot), p, *x, *out, ws)
        torch.cuda.synchronize()
        assert not any(o.view(torch.int16).any() for o in out)
