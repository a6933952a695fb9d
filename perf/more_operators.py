"""Cases of the paged 4-bit cache and of what a serving step does around it: page tables and slot maps, rotary positions,
writing and reading back, attention of packed queries.  ``own`` chooses between the plain torch form and the library's
calls."""
import math

import torch

own = False

D = 128            # head dimension of the cache
B = 64             # tokens of a page
GROUP = 32         # dimensions of K that share a scale; V has one for a token's 128
FLOOR = 2.0 ** -100            # least scale
STEP = 0.06666667014360428     # 1 / 15 in 32 bits
BASE = 500000.0                # of the rotary frequencies


def listed():
    return [
        # the new token of 64 running requests: pages taken where a length passes a page's end (the batch of bench.py --decode)
        {"name": "tables_decode_64", "kind": "tables", "S": 64, "len": 8192, "one": 1.0, "chunk": 1, "pad": 0},
        # a server's step: 250 requests of which most have a token, some nothing, some a prompt chunk; padded rows behind
        {"name": "tables_mixed_250", "kind": "tables", "S": 250, "len": 32768, "one": 0.8, "chunk": 1024, "pad": 57},
        # queries and keys of a decode step, 64 requests, a Llama-3.1-8B layer
        {"name": "rotate_token_batch64", "kind": "rotate", "N": 64, "Hq": 32, "H": 8, "d": 128, "rot": 128, "layout": "half", "dtype": "bf16",
         "far": 8192, "scaled": True, "transpose": False},
        # a prompt of odd length far into a long context, half of each head rotated in pairs, in fp32, and the gradient's form
        {"name": "rotate_prompt_8191", "kind": "rotate", "N": 8191, "Hq": 32, "H": 8, "d": 128, "rot": 64, "layout": "interleaved",
         "dtype": "fp32", "far": 131072, "scaled": False, "transpose": True},
        # one decode step's new token, 64 requests
        {"name": "append_token_batch64", "kind": "append", "N": 64, "H": 8, "src": "bf16", "pages": 4096},
        # the prompt of one layer, an odd length, rows of a fused projection
        {"name": "append_prompt_8191", "kind": "append", "N": 8191, "H": 8, "src": "bf16", "pages": 512},
        # decode of one short chat: latency
        {"name": "attend_short", "kind": "attend", "S": 1, "H": 8, "G": 4, "n": 1, "len": 300, "ones": False, "bias": False, "ragged": False},
        # decode of 64 ragged requests, 8K
        {"name": "attend_batch64_8k", "kind": "attend", "S": 64, "H": 8, "G": 4, "n": 1, "len": 8192, "ones": False, "bias": False, "ragged": True},
        # decode of one 128K context: few rows, a long axis
        {"name": "attend_single_128k", "kind": "attend", "S": 1, "H": 8, "G": 4, "n": 1, "len": 131072, "ones": False, "bias": False, "ragged": False},
        # three draft tokens against compact caches with their attention-mass bias, odd length
        {"name": "attend_compact_bias", "kind": "attend", "S": 64, "H": 8, "G": 4, "n": 3, "len": 1641, "ones": False, "bias": True, "ragged": False},
        # a 512-token prompt chunk against a 32K cache
        {"name": "attend_chunk_32k", "kind": "attend", "S": 1, "H": 8, "G": 4, "n": 512, "len": 32768, "ones": False, "bias": False, "ragged": False},
        # one prompt chunk beside 16 decoding requests, ragged
        {"name": "attend_mixed_17", "kind": "attend", "S": 17, "H": 8, "G": 4, "n": 256, "len": 8192, "ones": True, "bias": False, "ragged": True},
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["tables", "rotate", "append", "attend", "attend", "attend"])
    H = rng.choice([1, 2, 4, 8])
    if kind == "tables":
        S = _spread(rng, 1, 250)
        return {"kind": kind, "S": S, "len": _spread(rng, 1, 32768), "one": rng.choice([0.0, 0.5, 0.8, 1.0]), "chunk": _spread(rng, 1, 1024),
                "pad": rng.choice([0, rng.randint(0, 100)])}
    if kind == "rotate":
        d = rng.choice([64, 128, 128, 256])
        return {"kind": kind, "N": _spread(rng, 1, 8191 * 128 // d // 2), "Hq": H * rng.choice([1, 2, 4]), "H": H, "d": d,
                "rot": d // 16 * rng.choice([4, 8, 12, 16]), "layout": rng.choice(["half", "interleaved"]), "dtype": rng.choice(["bf16", "bf16", "fp32"]),
                "far": _spread(rng, 1, 131072), "scaled": rng.random() < 0.5, "transpose": rng.random() < 0.3}
    if kind == "append":
        N = _spread(rng, 1, 8191)
        return {"kind": kind, "N": N, "H": H, "src": rng.choice(["bf16", "fp32"]), "pages": (N + B - 1) // B * rng.choice([1, 2]) + rng.randint(0, 64)}
    G = rng.choice([1, 2, 4, 8])
    shape = rng.random()
    if shape < 0.6:                                 # decode and draft steps
        T = _spread(rng, 1, 131072)
        return {"kind": kind, "S": _spread(rng, 1, max(1, min(64, 4000000 // (T * H)))), "H": H, "G": G, "n": min(T, rng.choice([1, 1, 2, 5])), "len": T,
                "ones": False, "bias": rng.random() < 0.4, "ragged": rng.random() < 0.5}
    n = _spread(rng, 4, 512)                        # prompt chunks, alone or beside decoding requests
    T = _spread(rng, max(64, n), max(600, min(32768, (1 << 26) // (n * G))))
    S = 1 if shape < 0.8 else max(1, min(16, (1 << 29) // (n * G * H * T)))
    return {"kind": kind, "S": S, "H": H, "G": G, "n": n, "len": T, "ones": S > 1, "bias": rng.random() < 0.3, "ragged": S > 1 and rng.random() < 0.5}


# --------------------------------------------------------------------- inputs

def _lengths(case, g, most):
    """Tokens of each request: `most`, or from half of it up."""
    if not case["ragged"]:
        return torch.full((case["S"],), most, dtype=torch.int64, device="cuda")
    x = torch.randint(max(case["n"], most // 2), most + 1, (case["S"],), generator=g, device="cuda")
    x[0] = most
    return x


def _rows(g, n, H, dtype, key):
    """Keys with a few strong channels, or values, as a projection leaves them, [n, H, D]."""
    x = torch.randn(n, H, D, generator=g, device="cuda")
    if key:
        x *= 1.0 + 3.0 * (torch.rand(H, D, generator=g, device="cuda") < 0.03)
    return x.to(dtype)


def _pool(P, H, bias):
    """The plain form's pages: a code a byte, scales and least values apart."""
    z = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt, device="cuda")   # noqa: E731
    return {"K": z(P * B, H, D, dt=torch.uint8), "V": z(P * B, H, D, dt=torch.uint8), "ks": z(P * B, H, D // GROUP), "km": z(P * B, H, D // GROUP),
            "vs": z(P * B, H, 1), "vm": z(P * B, H, 1), "bias": z(P * B, H) if bias else None}


def _prepare_tables(case, g):
    S, M = case["S"], -(-(case["len"] + case["chunk"] + 64) // B)
    # a case has the same lengths and counts whatever the seed, in another order: the batch keeps its size
    f = torch.Generator()
    f.manual_seed(S)
    lens = torch.randint(0, case["len"] + 1, (S,), generator=f)
    counts = torch.where(torch.rand(S, generator=f) < case["one"], 1, torch.randint(0, case["chunk"] + 1, (S,), generator=f))
    counts = counts * (torch.rand(S, generator=f) < 0.95)
    lens = lens.cuda()[torch.randperm(S, generator=g, device="cuda")]
    counts = counts.cuda()[torch.randperm(S, generator=g, device="cuda")]
    held = (lens + B - 1) // B
    used = int(held.sum())
    P = used + int((counts // B + 2).sum())
    order = torch.randperm(P, generator=g, device="cuda")
    j = torch.arange(M, device="cuda")
    first = torch.cumsum(held, 0) - held
    table = torch.where(j < held[:, None], order[(first[:, None] + j).clamp_max(P - 1)], -1).to(torch.int32)
    st = {"counts": counts.to(torch.int32), "old": lens.to(torch.int32), "N": int(counts.sum()) + case["pad"], "table": table, "len": lens.to(torch.int32),
          "free": torch.cat([order[used:], torch.zeros(used, dtype=torch.int64, device="cuda")]).to(torch.int32),
          "n_free": torch.tensor([P - used], dtype=torch.int32, device="cuda")}
    if own:
        import paper_2609_36835_gb300 as pk
        p = pk.pages_alloc(S, 1, P, M * B)
        for name in ("table", "len", "free", "n_free"):
            getattr(p, name).copy_(st[name])
        st["pages"] = p
    return st


def _frequencies(case):
    """Radians a position of each pair, in 64 bits; scaled: the long wavelengths by 1/8, blended in between."""
    r = case["rot"]
    f = BASE ** (-torch.arange(0, r, 2, dtype=torch.float64) / r)
    if case["scaled"]:
        turns = 8192 * f / (2 * math.pi)            # of the trained context
        keep = ((turns - 1.0) / (4.0 - 1.0)).clamp(0.0, 1.0)
        f = f / 8.0 * (1 - keep) + f * keep
    return f.cuda()


def _prepare_rotate(case, g):
    N, dt = case["N"], torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    qkv = torch.randn(N, case["Hq"] + 2 * case["H"], case["d"], generator=g, device="cuda").to(dt)      # a fused projection's rows
    st = {"Q": qkv[:, :case["Hq"]], "K": qkv[:, case["Hq"]:case["Hq"] + case["H"]], "freq": _frequencies(case),
          "pos": torch.randint(0, case["far"] + 1, (N,), generator=g, device="cuda").to(torch.int32)}
    if own:
        import paper_2609_36835_gb300 as pk
        scaling = {"kind": "bands", "factor": 8.0, "low": 1.0, "high": 4.0, "context": 8192} if case["scaled"] else None
        st["rotary"] = pk.rotary(case["rot"], BASE, layout=case["layout"], scaling=scaling)
    return st


def _prepare_append(case, g):
    N, H, P = case["N"], case["H"], case["pages"]
    dt = torch.bfloat16 if case["src"] == "bf16" else torch.float32
    qkv = torch.cat([_rows(g, N, H, dt, True), _rows(g, N, H, dt, False)], 1)
    if N <= 128:                                    # a token of each request, anywhere in its page
        slots = torch.randperm(P, generator=g, device="cuda")[:N] * B + torch.randint(0, B, (N,), generator=g, device="cuda")
        slots = slots if N <= P else torch.randperm(P * B, generator=g, device="cuda")[:N]
    else:                                           # prompts: whole pages in any order
        slots = (torch.randperm(P, generator=g, device="cuda")[:, None] * B + torch.arange(B, device="cuda")).view(-1)[:N]
    st = {"K": qkv[:, :H], "V": qkv[:, H:], "slots": slots.to(torch.int32)}
    if own:
        import paper_2609_36835_gb300 as pk
        st["pages"] = pk.pages_alloc(1, H, P, P * B)
    else:
        st["pool"] = _pool(P, H, False)
    return st


def _prepare_attend(case, g):
    S, H, G, n = case["S"], case["H"], case["G"], case["n"]
    lens = _lengths(case, g, case["len"])
    M = -(-case["len"] // B)
    P = S * M + 3
    counts = torch.full((S,), n, dtype=torch.int64)
    if case["ones"]:
        counts[1:] = 1
    starts = torch.nn.functional.pad(torch.cumsum(counts, 0), (1, 0))
    N = int(starts[-1])
    order = torch.randperm(P, generator=g, device="cuda")
    held = (lens + B - 1) // B
    table = torch.where(torch.arange(M, device="cuda") < held[:, None], order[:S * M].view(S, M), -1).to(torch.int32)
    st = {"starts": starts.to(torch.int32).cuda(), "N": N, "n": n, "table": table, "len": lens.to(torch.int32)}
    if own:
        import paper_2609_36835_gb300 as pk
        p = st["pages"] = pk.pages_alloc(S, H, P, M * B, bias=case["bias"])
        p.table.copy_(table)
        p.len.copy_(st["len"])
    else:
        st["pool"] = _pool(P, H, case["bias"])
    q = torch.empty(N, H, G, D, device="cuda")
    for s in range(S):
        T, c = int(lens[s]), int(counts[s])
        k, v = _rows(g, T, H, torch.bfloat16, True), _rows(g, T, H, torch.bfloat16, False)
        t = torch.arange(T, device="cuda")
        slots = (table[s, t // B] * B + t % B).to(torch.int32)
        bias = torch.rand(T, H, generator=g, device="cuda") * 3.0 - 2.0 if case["bias"] else None
        if own:
            pk.pages_append(st["pages"], k, v, slots, bias=bias)
        else:
            _plain_append(st["pool"], k, v, slots, bias)
        j = torch.randint(0, T, (c * G,), generator=g, device="cuda")
        q[int(starts[s]):int(starts[s]) + c] = k[j].float().view(c, G, H, D).transpose(1, 2)      # queries near keys
    st["Q"] = (q + 0.5 * torch.randn(q.shape, generator=g, device="cuda")).to(torch.bfloat16)
    if own:
        st["ws"] = pk.pages_workspace(st["pages"], n, G)
    return st


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    st = {"tables": _prepare_tables, "rotate": _prepare_rotate, "append": _prepare_append, "attend": _prepare_attend}[case["kind"]](case, g)
    st["case"] = case
    return st


# ----------------------------------------------------------------- plain form

def _plain_tables(st):
    """Takes pages for the new tokens, then gives them back, as a step that is not kept does."""
    counts, lens, table, free = st["counts"].long(), st["len"].long(), st["table"], st["free"]
    S, M = table.shape
    starts = torch.nn.functional.pad(torch.cumsum(counts, 0), (1, 0))
    held, want = (lens + B - 1) // B, (lens + counts + B - 1) // B
    before = torch.cumsum(want - held, 0) - (want - held)         # pages that earlier requests take
    j = torch.arange(M, device="cuda")
    new = (j >= held[:, None]) & (j < want[:, None])
    at = st["n_free"].long() - 1 - (before[:, None] + j - held[:, None])
    wide = torch.where(new, free[at.clamp(0, free.shape[0] - 1)], table)
    i = torch.arange(st["N"], device="cuda")
    s = torch.searchsorted(starts, i, right=True) - 1
    there = s < S
    s = s.clamp_max(S - 1)
    pos = lens[s] + i - starts[s]
    slots = wide[s, (pos // B).clamp_max(M - 1)] * B + pos % B
    # back: the same pages in the same places
    taken = (want - held).sum()
    n_free = st["n_free"].long() - taken
    back = free.clone()
    flat = torch.where(new, n_free + taken - 1 - (before[:, None] + j - held[:, None]), free.shape[0])
    back = torch.cat([back, back[:1]]).scatter(0, flat.view(-1), wide.view(-1))[:-1]
    table = torch.where(j < held[:, None], wide, -1)
    return {"starts": starts.to(torch.int32), "slots": torch.where(there, slots, -1).to(torch.int32), "positions": torch.where(there, pos, -1).to(torch.int32),
            "table": table.to(torch.int32), "len": st["old"] + 0, "n_free": (n_free + taken).to(torch.int32),
            "free": torch.where(torch.arange(free.shape[0], device="cuda") < n_free + taken, back, 0)}


def _plain_rotation(x, pos, freq, case):
    r = case["rot"]
    a = pos.double()[:, None, None] * freq
    c, s = torch.cos(a).float(), torch.sin(a).float()
    s = -s if case["transpose"] else s
    y = x.float()
    if case["layout"] == "half":
        x1, x2 = y[..., :r // 2], y[..., r // 2:r]
        turned = torch.cat([x1 * c - x2 * s, x2 * c + x1 * s], -1)
    else:
        x1, x2 = y[..., 0:r:2], y[..., 1:r:2]
        turned = torch.stack([x1 * c - x2 * s, x2 * c + x1 * s], -1).flatten(-2)
    return torch.cat([turned, y[..., r:]], -1).to(x.dtype)


def _quantise(x):
    """Codes, scale and least value of x [..., n] in 4 bits; each rounding is part of the definition."""
    least, most = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    m = least.to(torch.bfloat16).float()
    s = ((most - m) * STEP).to(torch.bfloat16).float().clamp_min(FLOOR)
    return torch.round((x - m) * (torch.full_like(s, 1.0) / s)).clamp(0.0, 15.0), s, m


def _plain_append(c, K, V, slots, bias):
    n, H = K.shape[:2]
    i = slots.long()
    codes, s, m = _quantise(K.float().reshape(n, H, D // GROUP, GROUP))
    c["K"][i] = codes.view(n, H, D).to(torch.uint8)
    c["ks"][i], c["km"][i] = s[..., 0], m[..., 0]
    codes, s, m = _quantise(V.float())
    c["V"][i] = codes.to(torch.uint8)
    c["vs"][i], c["vm"][i] = s, m
    if bias is not None:
        c["bias"][i] = bias


def _plain_values(codes, s, m):
    """What codes [..., D] stand for, with scales [..., groups]."""
    shape = codes.shape
    return (m[..., None] + codes.float().view(*shape[:-1], s.shape[-1], -1) * s[..., None]).view(shape)


def _plain_append_run(st):
    c = st["pool"]
    _plain_append(c, st["K"], st["V"], st["slots"], None)
    i = st["slots"].long()
    return {"K": _plain_values(c["K"][i], c["ks"][i], c["km"][i]).to(torch.bfloat16), "V": _plain_values(c["V"][i], c["vs"][i], c["vm"][i]).to(torch.bfloat16)}


def _plain_attend(st):
    c, table, lens, starts, Q = st["pool"], st["table"].long(), st["len"].long(), st["starts"].long(), st["Q"]
    S, M = table.shape
    N, H, G, _ = Q.shape
    n, T = st["n"], M * B
    i = (table.clamp_min(0)[:, :, None] * B + torch.arange(B, device="cuda")).view(S, T)
    K = _plain_values(c["K"][i], c["ks"][i], c["km"][i]).transpose(1, 2)                  # [S, H, T, D]
    V = _plain_values(c["V"][i], c["vs"][i], c["vm"][i]).transpose(1, 2)
    counts = starts[1:] - starts[:-1]
    at = starts[:-1, None] + torch.arange(n, device="cuda")                               # rows of a request, as many for each
    real = torch.arange(n, device="cuda") < counts[:, None]
    q = Q[at.clamp_max(N - 1)].float().permute(0, 2, 1, 3, 4).reshape(S, H, n * G, D)
    logits = torch.matmul(q, K.transpose(2, 3)) / math.sqrt(D)
    if c["bias"] is not None:
        logits = logits + c["bias"][i].transpose(1, 2).unsqueeze(2)
    sees = (lens - counts)[:, None] + torch.arange(n, device="cuda") + 1                  # causal
    seen = (torch.arange(T, device="cuda") < torch.minimum(sees, lens[:, None])[..., None]).repeat_interleave(G, 1)
    logits = logits.masked_fill(~seen[:, None], -math.inf)
    top = logits.amax(-1, keepdim=True)
    p = torch.exp(logits - torch.where(torch.isinf(top), 0.0, top))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p / torch.where(total == 0, 1.0, total), V).view(S, H, n, G, D).transpose(1, 2)
    return {"O": o[real].to(torch.bfloat16)}


# ------------------------------------------------------------------------ run

def run(st):
    case = st["case"]
    kind = case["kind"]
    if not own:
        if kind == "rotate":
            return {"Q": _plain_rotation(st["Q"], st["pos"], st["freq"], case), "K": _plain_rotation(st["K"], st["pos"], st["freq"], case)}
        return {"tables": _plain_tables, "append": _plain_append_run, "attend": _plain_attend}[kind](st)
    import paper_2609_36835_gb300 as pk
    if kind == "tables":
        p = st["pages"]
        starts, slots, positions = pk.pages_extend(p, st["counts"], st["N"], check=False)
        pk.pages_truncate(p, st["old"], check=False)
        return {"starts": starts, "slots": slots, "positions": positions, "table": p.table, "len": p.len, "n_free": p.n_free, "free": p.free}
    if kind == "rotate":
        Q, K = pk.rotate(st["rotary"], st["pos"], st["Q"], st["K"], transpose=case["transpose"])
        return {"Q": Q, "K": K}
    if kind == "append":
        pk.pages_append(st["pages"], st["K"], st["V"], st["slots"], check=False)
        K, V = pk.pages_read(st["pages"], st["slots"], dtype=torch.bfloat16, check=False)
        return {"K": K, "V": V}
    return {"O": pk.pages_attend(st["pages"], st["Q"], st["starts"], max_count=case["n"], ws=st["ws"], check=False)}


# ----------------------------------------------------------------------- work

def work(case):
    """Bytes and operations at the mean length: sources and pages once, outputs once."""
    kind = case["kind"]
    if kind == "tables":
        mean = 0.95 * (case["one"] + (1 - case["one"]) * case["chunk"] / 2)
        N, new = case["S"] * mean + case["pad"], case["S"] * mean / B
        return {"bytes": 4 * (2 * N + 7 * case["S"] + 6 * new), "flops": 4 * N}
    if kind == "rotate":
        heads, width = case["Hq"] + case["H"], 2 if case["dtype"] == "bf16" else 4
        return {"bytes": case["N"] * (2 * heads * case["d"] * width + 4) + case["rot"] * 4, "flops": case["N"] * heads * case["rot"] * 3}
    H = case["H"]
    token = D + 4 * (D // GROUP) + 4                # codes, scales and least values of K and V
    if kind == "append":
        width = 2 if case["src"] == "bf16" else 4
        return {"bytes": case["N"] * (H * (2 * D * width + 2 * token + 2 * D * 2) + 8), "flops": case["N"] * H * D * 8}
    S, G, n = case["S"], case["G"], case["n"]
    T = case["len"] * (0.75 if case["ragged"] else 1.0)
    single = S - 1 if case["ones"] else 0           # requests with one row
    rows = (S - single) * n * G + single * G
    seen = (S - single) * n * G * max(T - n / 2, T / 2) + single * G * T
    return {"bytes": S * H * T * (token + (4 if case["bias"] else 0)) + rows * H * D * 4, "flops": 4 * H * D * seen}


# ---------------------------------------------------------------------- exact

def _exact_group(x):
    """What x [..., n] is held as in 4 bits; scale, least value and codes as the format rounds them, values in 64 bits."""
    low = x.min(-1, keepdim=True).values.to(torch.bfloat16)
    span = x.max(-1, keepdim=True).values - low.float()
    scale = (span.double() * STEP).float().to(torch.bfloat16).float()
    scale = torch.maximum(scale, torch.full_like(scale, FLOOR))
    inverse = (1.0 / scale.double()).float()
    code = torch.floor((x - low.float()) * inverse + 0.0)
    rest = ((x - low.float()) * inverse).double() - code.double()
    code = code.double() + ((rest > 0.5) | ((rest == 0.5) & (code % 2 == 1))).double()
    return low.double() + code.clamp(0, 15) * scale.double()


def _exact_attend(case, seed):
    S, H, G, n = case["S"], case["H"], case["G"], case["n"]
    if S * H > 600 or S * H * n * G * case["len"] > 6e9:
        return None
    st = prepare(case, seed)
    lens, starts, out = st["len"].tolist(), st["starts"].tolist(), []
    for s in range(S):
        T, c = lens[s], starts[s + 1] - starts[s]
        t = torch.arange(T, device="cuda")
        at = st["table"][s, t // B].long() * B + t % B
        p = st["pool"]
        sees = torch.tensor([min(T, T - c + 1 + i) for i in range(c)], device="cuda").repeat_interleave(G)
        o = torch.zeros(c, H, G, D, dtype=torch.float64, device="cuda")
        for h in range(H):
            k = p["K"][at, h].double() * p["ks"][at, h].double().repeat_interleave(GROUP, 1) + p["km"][at, h].double().repeat_interleave(GROUP, 1)
            v = p["V"][at, h].double() * p["vs"][at, h].double() + p["vm"][at, h].double()
            q = st["Q"][starts[s]:starts[s + 1], h].double().reshape(c * G, D)
            for i in range(0, c * G, 512):
                a = q[i:i + 512] @ k.T / math.sqrt(D)
                if p["bias"] is not None:
                    a = a + p["bias"][at, h].double()
                a = a.masked_fill(t >= sees[i:i + 512, None], -math.inf)
                top = a.max(1, keepdim=True).values
                e = torch.exp(a - top.masked_fill(top == -math.inf, 0.0))
                z = e.sum(1, keepdim=True)
                row = torch.arange(i, min(i + 512, c * G), device="cuda")
                o[row // G, h, row % G] = (e @ v) / z.masked_fill(z == 0, 1.0)
        out.append(o)
    return {"O": torch.cat(out)}


def exact(case, seed):
    kind = case["kind"]
    if kind == "tables":
        return None
    if kind == "attend":
        return _exact_attend(case, seed)
    st = prepare(case, seed)
    if kind == "append":
        K = st["K"].float()
        return {"K": _exact_group(K.reshape(*K.shape[:2], -1, GROUP)).view(K.shape), "V": _exact_group(st["V"].float())}
    out, r = {}, case["rot"]
    turn = torch.polar(torch.ones(case["N"], r // 2, dtype=torch.float64, device="cuda"), st["pos"].double()[:, None] * st["freq"])[:, None]
    turn = turn.conj() if case["transpose"] else turn
    for name in ("Q", "K"):
        x = st[name].double()
        pairs = x[..., :r].unflatten(-1, (2, r // 2)).transpose(-1, -2) if case["layout"] == "half" else x[..., :r].unflatten(-1, (r // 2, 2))
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        z = z.transpose(-1, -2).flatten(-2) if case["layout"] == "half" else z.flatten(-2)
        out[name] = torch.cat([z, x[..., r:]], -1)
    return out
