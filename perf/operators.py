"""The measured calls of the 4-bit paged cache and of linear attention with a decay for each head.

Three kinds of case:

* "append": the K/V rows of a wave's new tokens go into 4-bit pages (blocks of 32 values along the head
  dim share a power-of-two scale byte, each value is a 4-bit e2m1 code) and are read back as bf16.
* "attn": a wave's queries attend causally over such pages: one token a request (decoding) or a chunk.
* "lin": one wave of a layer S_t = alpha_t S_{t-1} + k_t v_t^T, o_t = scale S_t^T q_t, whose state is resumed
  from and left in snapshot slots: one token a request or a chunk.

A page of one KV head is page * dim / 2 code bytes (element 2i in the low nibble of byte i of its row, 2i + 1 in the
high one), then page * dim / 32 scale bytes.  The plain forms are elementary torch operations in 32 bits.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
# (query heads, KV heads, head dim) of the repository's workloads and tests
GROUPED = ((8, 2, 64), (24, 4, 64), (32, 8, 128), (64, 8, 128), (16, 16, 128), (16, 1, 128))
# (heads, heads of q and k, d_k, d_v)
LINEAR = ((64, 64, 128, 128), (32, 8, 128, 64), (16, 1, 64, 64), (24, 24, 64, 128))
MAX_SCORES = 4.3e9          # query rows x longest length of a drawn case: memory of the plain form
MAX_POOL_VALUES = 2.2e9     # cached K values of a drawn case
MAX_TOKEN_HEADS = 1 << 20   # of a drawn "lin" case


def listed():
    def attn(name, heads, page, requests, prefix, chunk, spans=1):
        q, kv, dim = heads
        return {"name": name, "op": "attn", "q_heads": q, "kv_heads": kv, "dim": dim, "page": page, "requests": requests,
                "prefix_lo": prefix[0], "prefix_hi": prefix[1], "chunk_lo": chunk[0], "chunk_hi": chunk[1], "spans": spans}

    def append(*a, **k):
        return {**attn(*a, **k), "op": "append"}

    def lin(name, heads, requests, chunk, resumed, per_token=True, spans=1):
        h, qk, dk, dv = heads
        return {"name": name, "op": "lin", "heads": h, "qk_heads": qk, "dk": dk, "dv": dv, "requests": requests,
                "chunk_lo": chunk[0], "chunk_hi": chunk[1], "resumed": resumed, "per_token": per_token, "spans": spans}

    return [
        # one conversation being answered on an idle GPU: the latency of a token
        attn("decode_one", (32, 8, 128), 64, 1, (8191, 8191), (1, 1)),
        # a serving batch, one token each behind histories of all lengths: the cache is streamed
        attn("decode_batch", (64, 8, 128), 64, 64, (1000, 32768), (1, 1)),
        # many short conversations, small pages and heads
        attn("decode_small_pages", (24, 4, 64), 16, 128, (16, 4000), (1, 1)),
        # the last tokens of prompts whose prefix is cached
        attn("short_chunks", (64, 8, 128), 64, 8, (16384, 32768), (16, 16)),
        # an ordinary wave of prompts with little reuse
        attn("ordinary", (32, 8, 128), 64, 4, (0, 4096), (2048, 2048)),
        # a chunk of a long document
        attn("long_prefix", (64, 8, 128), 64, 1, (65536, 65536), (1024, 1024)),
        # the new token of each of 64 requests, stored
        append("append_tokens", (64, 8, 128), 64, 64, (1000, 32768), (1, 1)),
        # a wave of 16K prompt tokens, stored
        append("append_wave", (64, 8, 128), 64, 8, (0, 8192), (2048, 2048)),
        # one token each of a serving batch: the states are streamed
        lin("lin_tokens", (64, 64, 128, 128), 128, (1, 1), 1.0),
        # one token each of a few requests, heads that share q and k, one decay a head
        lin("lin_tokens_few", (32, 8, 128, 64), 4, (1, 1), 1.0, False),
        # the ordinary wave of 4K-token chunks
        lin("lin_wave", (64, 64, 128, 128), 4, (4096, 4096), 0.5),
        # a few ragged prompts, fewer chains than compute units
        lin("lin_ragged", (32, 8, 128, 64), 3, (700, 9000), 0.34),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("decode", "decode", "chunk", "chunk", "append", "lin tokens", "lin chunk"))
    spans = rng.randrange(1 << 20)
    while True:
        if kind.startswith("lin"):
            h, qk, dk, dv = rng.choice(LINEAR)
            lo, hi = (1, 1) if kind == "lin tokens" else sorted((_log(rng, 2, 16384), _log(rng, 2, 16384)))
            case = {"op": "lin", "heads": h, "qk_heads": qk, "dk": dk, "dv": dv, "requests": _log(rng, 1, 128),
                    "chunk_lo": lo, "chunk_hi": hi, "resumed": 1.0 if hi == 1 else rng.choice((0.0, 0.5, 1.0)),
                    "per_token": rng.random() < 0.7, "spans": spans}
            if case["requests"] * hi * h <= MAX_TOKEN_HEADS and case["requests"] * h <= 8192:
                return case
            continue
        q, kv, dim = rng.choice(GROUPED)
        case = {"op": "append" if kind == "append" else "attn", "q_heads": q, "kv_heads": kv, "dim": dim,
                "page": rng.choice((16, 64, 64))}
        if kind == "decode":
            lo, hi = sorted((_log(rng, 16, 65536), _log(rng, 16, 65536)))
            case |= {"requests": _log(rng, 1, 128), "prefix_lo": lo, "prefix_hi": hi, "chunk_lo": 1, "chunk_hi": 1}
        else:
            lo, hi = sorted((_log(rng, 2, 4096), _log(rng, 2, 4096)))
            p = sorted((_log(rng, 1, 65536), _log(rng, 1, 65536)))
            case |= {"requests": _log(rng, 1, 16), "prefix_lo": p[0], "prefix_hi": p[1], "chunk_lo": lo, "chunk_hi": hi}
        case["spans"] = spans
        n = case["prefix_hi"] + case["chunk_hi"]
        if (case["requests"] * case["chunk_hi"] * q * n <= MAX_SCORES and case["requests"] * n * kv * dim <= MAX_POOL_VALUES
                and case["requests"] * case["chunk_hi"] <= 16384):
            return case


# ---------------------------------------------------------------------------------------------
# lengths, tables and inputs
# ---------------------------------------------------------------------------------------------

def _spans(case):
    """(cached tokens, new tokens) of every request."""
    r = np.random.default_rng(case["spans"])
    n = case["requests"]
    prefix = r.integers(case.get("prefix_lo", 0), case.get("prefix_hi", 0) + 1, n)
    chunk = r.integers(case["chunk_lo"], case["chunk_hi"] + 1, n)
    return prefix.astype(np.int32), chunk.astype(np.int32)


def _table(case):
    prefix, chunk = _spans(case)
    blocks = -(-(prefix + chunk) // case["page"])
    pages = int(blocks.sum())
    order = np.random.default_rng(case["spans"] + 1).permutation(pages).astype(np.int32)
    table = np.zeros((case["requests"], int(blocks.max())), dtype=np.int32)
    at = 0
    for r, b in enumerate(blocks.tolist()):
        table[r, :b] = order[at:at + b]
        at += b
    return prefix, chunk, table, pages


def _slots(case):
    """(state_in, state_out, slots): single tokens go on in place, chunks leave new snapshots."""
    n = case["requests"]
    if case["chunk_hi"] == 1:
        return np.arange(n, dtype=np.int32), np.arange(n, dtype=np.int32), n
    resumed = np.random.default_rng(case["spans"] + 2).random(n) < case["resumed"]
    return np.where(resumed, np.arange(n), -1).astype(np.int32), (n + np.arange(n)).astype(np.int32), 2 * n


def _randn(gen, *shape):
    x = torch.empty(shape, dtype=torch.bfloat16, device=DEV)
    return x.normal_(generator=gen)


def _inputs(case, seed):
    """What the seed alone makes: the tensors of a call, before any plan."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    if case["op"] == "lin":
        T = int(_spans(case)[1].sum())
        h, qk, dk, dv = case["heads"], case["qk_heads"], case["dk"], case["dv"]
        x = {"q": _randn(gen, T, qk, dk), "k": _randn(gen, T, qk, dk), "v": _randn(gen, T, h, dv)}
        rate = torch.rand(h, generator=gen, device=DEV).mul_(math.log(128.0)).sub_(math.log(256.0)).exp_()
        if case["per_token"]:
            z = torch.randn(T, h, generator=gen, device=DEV)
            x["alpha"] = torch.exp(-rate * torch.log1p(z.exp()))
        else:
            x["alpha"] = torch.exp(-rate)
        x["states"] = torch.randn(_slots(case)[2], h, dk, dv, generator=gen, device=DEV)
        return x
    prefix, chunk, table, pages = _table(case)
    T, kv, dim, page = int(chunk.sum()), case["kv_heads"], case["dim"], case["page"]
    # keys have a few large channels, as they do in earnest; values do not
    gain = torch.ones(kv, 1, dim, device=DEV)
    gain[:, :, ::37] = 4.0
    if case["op"] == "append":
        x = {"k_new": (_randn(gen, T, kv, dim) * gain[:, 0].to(torch.bfloat16)), "v_new": _randn(gen, T, kv, dim)}
        x["k_pool"] = torch.randint(0, 256, (pages, kv, _page_bytes(case)), dtype=torch.uint8, generator=gen, device=DEV)
        x["v_pool"] = torch.randint(0, 256, (pages, kv, _page_bytes(case)), dtype=torch.uint8, generator=gen, device=DEV)
        return x
    x = {"q": _randn(gen, T, case["q_heads"], dim)}
    for name in ("k_pool", "v_pool"):
        pool = torch.empty(pages, kv, _page_bytes(case), dtype=torch.uint8, device=DEV)
        step = max(1, (1 << 27) // (kv * page * dim))
        for p in range(0, pages, step):
            m = min(step, pages - p)
            rows = _randn(gen, m, kv, page, dim)
            codes, scales = _quantise(rows.float() * gain[None, :, :, :] if name == "k_pool" else rows.float())
            pool[p:p + m, :, :page * dim // 2] = codes.reshape(m, kv, -1)
            pool[p:p + m, :, page * dim // 2:] = scales.reshape(m, kv, -1)
        x[name] = pool
    return x


def _page_bytes(case):
    return case["page"] * (case["dim"] // 2 + case["dim"] // 32)


def prepare(case, seed):
    s = {"case": case, "x": _inputs(case, seed)}
    if case["op"] == "lin":
        prefix, chunk = _spans(case)
        s["in"], s["out"], slots = _slots(case)
        s["chunk"] = chunk
        T = int(chunk.sum())
        s["o"] = torch.empty(T, case["heads"], case["dv"], dtype=torch.bfloat16, device=DEV)
        if own:
            import paper_2609_35263_amd as lib
            s["plan"] = lib.lin_plan(num_heads=case["heads"], num_qk_heads=case["qk_heads"], head_dim_k=case["dk"],
                                     head_dim_v=case["dv"], num_state_slots=slots, chunk_lens=chunk, state_in=s["in"],
                                     state_out=s["out"], scale=case["dk"] ** -0.5, alpha_per_token=case["per_token"])
            s["ws"] = lib.new_workspace(s["plan"], DEV)
            lib.lin_upload(s["plan"], s["ws"])
        return s
    prefix, chunk, table, pages = _table(case)
    s |= {"prefix": prefix, "chunk": chunk, "table": table}
    T, kv, dim = int(chunk.sum()), case["kv_heads"], case["dim"]
    if case["op"] == "append":
        s["k"] = torch.empty(T, kv, dim, dtype=torch.bfloat16, device=DEV)
        s["v"] = torch.empty_like(s["k"])
    else:
        s["o"] = torch.empty(T, case["q_heads"], dim, dtype=torch.bfloat16, device=DEV)
        s["lse"] = torch.empty(T, case["q_heads"], dtype=torch.float32, device=DEV)
    if own:
        import paper_2609_35263_amd as lib
        s["plan"] = lib.q4_plan(num_q_heads=case["q_heads"], num_kv_heads=kv, head_dim_qk=dim, head_dim_v=dim,
                                page_size=case["page"], num_pages=pages, softmax_scale=dim ** -0.5, prefix_lens=prefix,
                                chunk_lens=chunk, block_table=table)
        s["ws"] = lib.new_workspace(s["plan"], DEV)
        lib.plan_upload(s["plan"], s["ws"])
    return s


def run(s):
    x, op = s["x"], s["case"]["op"]
    if own:
        import paper_2609_35263_amd as lib
        if op == "append":
            lib.q4_append_kv(s["plan"], x["k_new"], x["v_new"], x["k_pool"], x["v_pool"], s["ws"])
            lib.q4_read_kv(s["plan"], x["k_pool"], x["v_pool"], s["k"], s["v"], s["ws"])
            return {"k": s["k"], "v": s["v"]}
        if op == "attn":
            lib.q4_chunked_prefill(s["plan"], x["q"], x["k_pool"], x["v_pool"], s["o"], s["lse"], s["ws"])
            return {"out": s["o"], "lse": s["lse"]}
        lib.lin_chunked_prefill(s["plan"], x["q"], x["k"], x["v"], x["alpha"], x["states"], s["o"], s["ws"])
        return {"out": s["o"], "states": x["states"]}
    if op == "append":
        return _plain_append(s)
    if op == "attn":
        return _plain_attention(s)
    return _plain_tokens(s) if s["case"]["chunk_hi"] == 1 else _plain_chunks(s)


def work(case):
    prefix, chunk = (v.astype(np.int64) for v in _spans(case))
    T = int(chunk.sum())
    if case["op"] == "lin":
        h, qk, dk, dv = case["heads"], case["qk_heads"], case["dk"], case["dv"]
        state_in, state_out, _ = _slots(case)
        states = (int((state_in >= 0).sum()) + len(state_out)) * h * dk * dv * 4
        tokens = T * (2 * qk * dk + 2 * h * dv) * 2 + (T if case["per_token"] else 1) * h * 4
        return {"bytes": tokens + states, "flops": 4 * T * h * dk * dv}
    kv, dim, q = case["kv_heads"], case["dim"], case["q_heads"]
    row = dim // 2 + dim // 32
    if case["op"] == "append":
        return {"bytes": 2 * T * kv * (2 * 2 * dim + 2 * row), "flops": 0}
    pairs = int((chunk * prefix + chunk * (chunk + 1) // 2).sum())
    cached = int((prefix + chunk).sum())
    return {"bytes": 2 * cached * kv * row + T * q * (2 * 2 * dim + 4), "flops": 4 * dim * q * pairs}


# ---------------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------------

def _quantise(x):
    """Rows of fp32 values [..., dim] as packed codes [..., dim / 2] and scale bytes [..., dim / 32]."""
    b = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    amax = b.abs().amax(-1)
    m, e = torch.frexp(amax)                                    # amax = m 2^e, m in [0.5, 1)
    byte = e.sub_(3).add_((m > 0.875).int()).add_(127)          # the smallest s with amax <= 7 s, + 127
    byte = byte.masked_fill_(amax == 0, 0).clamp_(8, 252)
    a = torch.ldexp(b, (127 - byte).unsqueeze(-1)).abs_()
    code = (a > 0.25).to(torch.uint8)
    for above in (a >= 0.75, a > 1.25, a >= 1.75, a > 2.5, a >= 3.5, a > 5.0):
        code += above
    code += torch.signbit(b).to(torch.uint8) * 8
    code = code.reshape(x.shape)
    return code[..., 0::2] | (code[..., 1::2] << 4), byte.to(torch.uint8)


def _values(pages, case):
    """fp32 values [..., page, dim] of pages of bytes [..., page bytes]."""
    page, dim = case["page"], case["dim"]
    grid = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0.0, -.5, -1, -1.5, -2, -3, -4, -6], device=DEV)
    codes = pages[..., :page * dim // 2]
    scales = pages[..., page * dim // 2:].reshape(*pages.shape[:-1], page, dim // 32, 1)
    low, high = grid[(codes & 15).int()], grid[(codes >> 4).int()]
    v = torch.stack((low, high), dim=-1).reshape(*pages.shape[:-1], page, dim // 32, 32)
    return v.mul_(torch.exp2(scales.float() - 127.0)).reshape(*pages.shape[:-1], page, dim)


def _where(s):
    """(page, slot) of every new token, packed in request order."""
    prefix, chunk, table, page = s["prefix"], s["chunk"], s["table"], s["case"]["page"]
    req = np.repeat(np.arange(len(chunk)), chunk)
    pos = np.arange(len(req)) - np.repeat(np.cumsum(chunk) - chunk, chunk) + prefix[req]
    at = np.stack((table[req, pos // page], pos % page)).astype(np.int64)
    at = torch.from_numpy(at).to(DEV)
    return at[0], at[1]


def _plain_append(s):
    case, x = s["case"], s["x"]
    page, dim, kv = case["page"], case["dim"], case["kv_heads"]
    pg, slot = _where(s)
    out = {}
    for name in ("k", "v"):
        codes, scales = _quantise(x[name + "_new"].float())
        pool = x[name + "_pool"]
        rows = slot[:, None] * (dim // 2) + torch.arange(dim // 2, device=DEV)
        marks = page * dim // 2 + slot[:, None] * (dim // 32) + torch.arange(dim // 32, device=DEV)
        heads = torch.arange(kv, device=DEV)[None, :, None]
        pool[pg[:, None, None], heads, rows[:, None, :]] = codes
        pool[pg[:, None, None], heads, marks[:, None, :]] = scales
        codes = pool[pg[:, None, None], heads, rows[:, None, :]]
        scales = pool[pg[:, None, None], heads, marks[:, None, :]]
        one = {**case, "page": 1}
        out[name] = _values(torch.cat((codes, scales), dim=-1), one)[:, :, 0].to(torch.bfloat16)
    return out


def _plain_attention(s):
    """All requests at once, padded to the longest length and chunk."""
    case, x = s["case"], s["x"]
    kv, dim, page, G = case["kv_heads"], case["dim"], case["page"], case["q_heads"] // case["kv_heads"]
    prefix, chunk = (torch.from_numpy(s[n].astype(np.int64)).to(DEV) for n in ("prefix", "chunk"))
    table = torch.from_numpy(s["table"].astype(np.int64)).to(DEV)
    R, C, N = len(chunk), int(s["chunk"].max()), table.shape[1] * page
    at = torch.arange(C, device=DEV)
    real = at[None, :] < chunk[:, None]                                   # [R, C]
    token = (torch.cumsum(chunk, 0) - chunk)[:, None] + at[None, :]
    q = x["q"][token.masked_fill(~real, 0)].float()                       # [R, C, Hq, dim]
    q = q.view(R, C, kv, G, dim).permute(0, 2, 1, 3, 4).reshape(R * kv, C * G, dim)
    k = _values(x["k_pool"][table], case).permute(0, 2, 1, 3, 4).reshape(R * kv, N, dim)
    w = torch.matmul(q, k.transpose(1, 2)).mul_(dim ** -0.5).view(R, kv, C, G, N)
    del k
    seen = torch.arange(N, device=DEV)[None, None, :] <= (prefix[:, None] + at[None, :])[:, :, None]
    w.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    top = w.amax(-1, keepdim=True)
    w.sub_(top).exp_()
    total = w.sum(-1, keepdim=True)
    v = _values(x["v_pool"][table], case).permute(0, 2, 1, 3, 4).reshape(R * kv, N, dim)
    v = v.masked_fill_((torch.arange(N, device=DEV) >= (prefix + chunk)[:, None]).repeat_interleave(kv, 0)[..., None], 0)
    o = torch.matmul(w.view(R * kv, C * G, N), v).view(R, kv, C, G, dim) / total
    lse = (top + total.log()).squeeze(-1)
    o = o.permute(0, 2, 1, 3, 4).reshape(R, C, kv * G, dim)[real]
    return {"out": o.to(torch.bfloat16), "lse": lse.permute(0, 2, 1, 3).reshape(R, C, kv * G)[real]}


def _plain_tokens(s):
    case, x = s["case"], s["x"]
    h, g = case["heads"], case["heads"] // case["qk_heads"]
    slots_in, slots_out = (torch.from_numpy(s[n].astype(np.int64)).to(DEV) for n in ("in", "out"))
    q, k = (x[n].float().repeat_interleave(g, 1) for n in ("q", "k"))
    alpha = x["alpha"].expand(len(q), h)
    S = x["states"][slots_in] * alpha[:, :, None, None]
    S.addcmul_(k[..., None], x["v"].float()[:, :, None, :])
    x["states"][slots_out] = S
    o = S.mul_(q[..., None]).sum(2) * case["dk"] ** -0.5
    return {"out": o.to(torch.bfloat16), "states": x["states"]}


def _plain_chunks(s):
    """Blocks of 64 tokens of all requests, padded to the longest: the products inside a block, each block's own state, and
    the states before the blocks from those of all earlier ones at once.  Logarithms of decays are summed in 64 bits."""
    case, x = s["case"], s["x"]
    h, g, dk, dv, C = case["heads"], case["heads"] // case["qk_heads"], case["dk"], case["dv"], 64
    chunk = torch.from_numpy(s["chunk"].astype(np.int64)).to(DEV)
    R, n = len(chunk), -(-int(s["chunk"].max()) // C)
    at = torch.arange(n * C, device=DEV)
    real = at[None, :] < chunk[:, None]
    token = ((torch.cumsum(chunk, 0) - chunk)[:, None] + at[None, :]).masked_fill(~real, 0)

    def blocks(t, fill):                                       # [R, h, n, C, ...]
        t = t[token].float()
        t[~real] = fill
        t = t.repeat_interleave(h // t.shape[2], 2)
        return t.view(R, n, C, *t.shape[2:]).movedim(3, 1)

    q, k, v = blocks(x["q"], 0.0), blocks(x["k"], 0.0), blocks(x["v"], 0.0)
    alpha = x["alpha"] if case["per_token"] else x["alpha"].expand(len(x["v"]), h)
    L = blocks(alpha[..., None], 1.0)[..., 0].double().log().cumsum(-1)              # [R, h, n, C]
    causal = torch.ones(C, C, device=DEV, dtype=torch.bool).tril()
    D = (L[..., :, None] - L[..., None, :]).exp().float().masked_fill_(~causal, 0)
    P = torch.matmul(q, k.transpose(-1, -2)).mul_(D)
    o = torch.matmul(P, v)
    del P, D
    ends = L[..., -1]                                                                # a whole block's decay
    own_state = torch.matmul((k * (ends[..., None] - L).exp().float()[..., None]).transpose(-1, -2), v)
    del k, v
    M = ends.cumsum(-1)                                                              # [R, h, n]
    first = torch.zeros(R, h, dk * dv, device=DEV)
    resumed = torch.from_numpy(s["in"].astype(np.int64)).to(DEV)
    first[resumed >= 0] = x["states"][resumed[resumed >= 0]].reshape(-1, h, dk * dv)
    # state after block b: first * exp(M_b) + sum over a <= b of own_state_a * exp(M_b - M_a)
    E = (M[..., :, None] - M[..., None, :]).exp().float()
    E = E.masked_fill_(~torch.ones(n, n, device=DEV, dtype=torch.bool).tril(), 0)
    after = torch.matmul(E, own_state.reshape(R, h, n, dk * dv))
    after += M.exp().float()[..., None] * first[:, :, None]
    before = torch.cat((first[:, :, None], after[:, :, :-1]), 2).view(R, h, n, dk, dv)
    o += torch.matmul(q * L.exp().float()[..., None], before)
    x["states"][torch.from_numpy(s["out"].astype(np.int64)).to(DEV)] = after[:, :, -1].view(R, h, dk, dv)
    o = o.movedim(1, 3).reshape(R, n * C, h, dv)[real] * dk ** -0.5
    return {"out": o.to(torch.bfloat16), "states": x["states"]}


# ---------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------

def exact(case, seed):
    x = _inputs(case, seed)
    if case["op"] == "append":
        return {"k": _exact_rounding(x["k_new"]), "v": _exact_rounding(x["v_new"])}
    return _exact_linear(case, x) if case["op"] == "lin" else _exact_attention(case, x)


def _exact_rounding(x):
    """The nearest value of the grid times the block's scale, by distance to each of the eight magnitudes."""
    b = x.double().unflatten(-1, (-1, 32))
    amax = b.abs().amax(-1, keepdim=True).clamp_min(1e-300)
    scale = torch.exp2((amax / 7).log2().ceil().clamp(-119, 125))
    # even codes are 0, 1, 2, 4: among equally near magnitudes the first of this order is the even one
    even_first = (0.0, 1.0, 2.0, 4.0, 0.5, 1.5, 3.0, 6.0)
    a = b.abs() / scale
    best, far = torch.zeros_like(a), a.clone()
    for m in even_first[1:]:
        d = (a - m).abs()
        near = d < far
        best, far = torch.where(near, m, best), torch.where(near, d, far)
    return (torch.copysign(best, b) * scale).flatten(-2)


def _exact_attention(case, x):
    kv, dim, page, G = case["kv_heads"], case["dim"], case["page"], case["q_heads"] // case["kv_heads"]
    prefix, chunk, table, _ = _table(case)
    magnitudes = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=DEV)

    def rows(pool, pages, head, n):
        held = pool[pages, head]
        byte = held[:, :page * dim // 2].reshape(-1, dim // 2).long()
        code = torch.empty(len(byte), dim, dtype=torch.long, device=DEV)
        code[:, 0::2], code[:, 1::2] = byte % 16, byte // 16
        scale = held[:, page * dim // 2:].reshape(-1, dim // 32).double() - 127
        value = torch.where(code >= 8, -magnitudes[code % 8], magnitudes[code % 8])
        return (value.view(-1, dim // 32, 32) * torch.exp2(scale)[..., None]).view(-1, dim)[:n]

    out = torch.empty(x["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.empty(x["q"].shape[:2], dtype=torch.float64, device=DEV)
    first = 0
    for r in range(len(chunk)):
        p, c = int(prefix[r]), int(chunk[r])
        pages = torch.as_tensor(table[r, :-(-(p + c) // page)].astype(np.int64), device=DEV)
        for head in range(kv):
            K, V = rows(x["k_pool"], pages, head, p + c), rows(x["v_pool"], pages, head, p + c)
            step = max(1, (1 << 27) // ((p + c) * G))
            for t in range(0, c, step):
                m = min(step, c - t)
                here = (slice(first + t, first + t + m), slice(head * G, head * G + G))
                w = x["q"][here].double().reshape(m * G, dim) @ K.t() / math.sqrt(dim)
                last = torch.arange(p + t, p + t + m, device=DEV).repeat_interleave(G)
                w[torch.arange(p + c, device=DEV)[None, :] > last[:, None]] = -math.inf
                lse[here] = torch.logsumexp(w, -1).view(m, G)
                out[here] = (torch.softmax(w, -1) @ V).view(m, G, dim)
        first += c
    return {"out": out, "lse": lse}


def _exact_linear(case, x):
    """Token by token; the longest requests first, so that the running ones lead."""
    chunk = _spans(case)[1].astype(np.int64)
    state_in, state_out, _ = _slots(case)
    order = np.argsort(-chunk, kind="stable")
    start = torch.as_tensor((np.cumsum(chunk) - chunk)[order], device=DEV)
    g, h = case["heads"] // case["qk_heads"], case["heads"]
    states = x["states"].double()
    S = torch.stack([states[int(state_in[r])] if state_in[r] >= 0 else torch.zeros_like(states[0]) for r in order])
    alpha = x["alpha"].double().expand(len(x["v"]), h)
    out = torch.empty(x["v"].shape, dtype=torch.float64, device=DEV)
    for t in range(int(chunk.max())):
        n = int((chunk[order] > t).sum())
        at = start[:n] + t
        q, k = (x[name][at].double().repeat_interleave(g, 1) for name in ("q", "k"))
        A = S[:n]
        A.mul_(alpha[at][:, :, None, None])
        A.add_(k[..., None] * x["v"][at].double()[:, :, None, :])
        out[at] = torch.matmul(q.unsqueeze(-2), A).squeeze(-2) * case["dk"] ** -0.5
    for i, r in enumerate(order):
        states[int(state_out[r])] = S[i]
    return {"out": out, "states": states}
