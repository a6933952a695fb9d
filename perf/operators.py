"""Cases of the 8-bit cache operators: writing and reading back, attention over the cache, and attention over the blocks
that a score selects.  ``own`` chooses between the plain torch form and the library's calls."""
import math

import torch

own = False

D = 128            # head dimension
B = 64             # tokens of a block
FLOOR = 2.0 ** -100   # least block magnitude
STEP = 0.007874015718698502   # 1 / 127 in 32 bits: a block's scale is its magnitude times this, rounded once


def listed():
    return [
        # one decode step's new token, 64 sequences of a Llama-3.1-8B layer with ragged lengths (the shape of bench.py --decode)
        {"name": "append_token_batch64", "kind": "append", "S": 64, "H": 8, "old": 8192, "n": 1, "src": "bf16", "ragged": True},
        # one new token of a single short chat: latency
        {"name": "append_token_single", "kind": "append", "S": 1, "H": 8, "old": 300, "n": 1, "src": "bf16", "ragged": False},
        # the prompt of one layer, an odd length
        {"name": "append_prompt_8191", "kind": "append", "S": 1, "H": 8, "old": 0, "n": 8191, "src": "bf16", "ragged": False},
        # the fp32 compact caches of all 32 layers of a 32K context at 5 % (1638 rows a head), as arckv_compact returns them
        {"name": "append_compact_layers", "kind": "append", "S": 32, "H": 8, "old": 0, "n": 1638, "src": "fp32", "ragged": False},
        # decode of one short chat: latency
        {"name": "attend_short", "kind": "attend", "S": 1, "H": 8, "G": 4, "n_pos": 1, "len": 300, "causal": False, "bias": False, "ragged": False},
        # decode of 64 ragged sequences, 8K
        {"name": "attend_batch64_8k", "kind": "attend", "S": 64, "H": 8, "G": 4, "n_pos": 1, "len": 8192, "causal": False, "bias": False, "ragged": True},
        # decode of one 128K context: few rows, a long axis
        {"name": "attend_single_128k", "kind": "attend", "S": 1, "H": 8, "G": 4, "n_pos": 1, "len": 131072, "causal": False, "bias": False, "ragged": False},
        # three draft tokens against compact caches with their attention-mass bias, odd length
        {"name": "attend_compact_bias", "kind": "attend", "S": 64, "H": 8, "G": 4, "n_pos": 3, "len": 1641, "causal": True, "bias": True, "ragged": False},
        # a 512-token prompt chunk against a 32K cache
        {"name": "attend_chunk_32k", "kind": "attend", "S": 1, "H": 8, "G": 4, "n_pos": 512, "len": 32768, "causal": True, "bias": False, "ragged": False},
        # sparse decode of one 128K context, 1/16 of its blocks
        {"name": "sparse_single_128k", "kind": "sparse", "S": 1, "H": 8, "G": 4, "n_pos": 1, "len": 131072, "m": 128, "ragged": False},
        # sparse decode of 16 ragged 32K contexts
        {"name": "sparse_batch16_32k", "kind": "sparse", "S": 16, "H": 8, "G": 4, "n_pos": 1, "len": 32768, "m": 64, "ragged": True},
        # a prompt chunk in which each position has its own blocks
        {"name": "sparse_chunk_16k", "kind": "sparse", "S": 1, "H": 8, "G": 4, "n_pos": 128, "len": 16384, "m": 32, "ragged": False},
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "sparse"])
    ragged = rng.random() < 0.5
    H = rng.choice([1, 2, 4, 8])
    if kind == "append":
        if rng.random() < 0.5:                      # tokens of a decode step, a draft or a short chunk
            return {"kind": kind, "S": _spread(rng, 1, 64), "H": H, "old": _spread(rng, 1, 8192), "n": _spread(rng, 1, 100),
                    "src": rng.choice(["bf16", "fp32"]), "ragged": ragged}
        n = _spread(rng, 64, 32768)                 # prompts and compact caches
        S = _spread(rng, 1, max(1, min(32, 400000 // (n * H))))
        return {"kind": kind, "S": S, "H": H, "old": 0, "n": n, "src": rng.choice(["bf16", "fp32"]), "ragged": False}
    if kind == "attend":
        G = rng.choice([1, 2, 4, 8])
        if rng.random() < 0.65:                     # decode and draft steps
            T = _spread(rng, 1, 131072)
            return {"kind": kind, "S": _spread(rng, 1, max(1, min(64, 4000000 // (T * H)))), "H": H, "G": G, "n_pos": rng.choice([1, 1, 2, 5]),
                    "len": T, "causal": rng.random() < 0.5, "bias": rng.random() < 0.4, "ragged": ragged}
        n_pos = _spread(rng, 8, 512)                # prompt chunks and reference queries
        T = _spread(rng, max(64, n_pos), max(128, min(32768, (1 << 26) // (n_pos * G))))
        return {"kind": kind, "S": 1, "H": H, "G": G, "n_pos": n_pos, "len": T, "causal": rng.random() < 0.7, "bias": rng.random() < 0.3, "ragged": False}
    T = _spread(rng, 64, 131072)
    n_pos = rng.choice([1, 1, 3, _spread(rng, 4, 128)])
    m = _spread(rng, 2, 128 if n_pos < 8 else 32)
    S = 1 if n_pos > 3 else _spread(rng, 1, max(1, min(16, 4000000 // (T * H))))
    return {"kind": kind, "S": S, "H": H, "G": rng.choice([1, 2, 4, 8]), "n_pos": n_pos, "len": T, "m": m, "ragged": ragged and S > 1}


# --------------------------------------------------------------------- inputs

def _lengths(case, g, most):
    """Valid tokens of each sequence: `most`, or from half of it up."""
    S = case["S"]
    if not case["ragged"]:
        return torch.full((S,), most, dtype=torch.int32, device="cuda")
    lo = max(1, most // 2)
    x = torch.randint(lo, most + 1, (S,), generator=g, device="cuda", dtype=torch.int64)
    x[0] = most
    return x.to(torch.int32)


def _rows(g, S, H, n, dtype, key):
    """Keys with a few strong channels, or values, as a projection leaves them."""
    x = torch.empty(S, H, n, D, dtype=dtype, device="cuda")
    ch = torch.ones(H, 1, D, device="cuda")
    if key:
        ch += 3.0 * (torch.rand(H, 1, D, generator=g, device="cuda") < 0.03)
    for s in range(S):
        x[s] = (torch.randn(H, n, D, generator=g, device="cuda") * ch).to(dtype)
    return x


def _empty(S, H, cap, bias):
    e = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt, device="cuda")   # noqa: E731
    nb = cap // B
    return {"K": e(S, H, cap, D, dt=torch.uint8), "V": e(S, H, cap, D, dt=torch.uint8), "k_scale": e(S, H, nb), "v_scale": e(S, H, nb),
            "bounds": e(S, H, nb, 2, D, dt=torch.int8), "tail": e(S, H, 2, B, D), "tail_amax": e(S, H, 2, B),
            "len": e(S, dt=torch.int32), "bias": e(S, H, cap) if bias else None}


def _filled(g, S, H, cap, lens, bias):
    """A cache as earlier writes left it, laid out sequence by sequence."""
    c = _empty(S, H, cap, bias)
    for s in range(S):
        length = int(lens[s])
        if length > 0:
            k, v = _rows(g, 1, H, length, torch.bfloat16, True), _rows(g, 1, H, length, torch.bfloat16, False)
            part = {n: (t[s:s + 1] if t is not None else None) for n, t in c.items()}
            _plain_append(part, k, v, torch.zeros(1, dtype=torch.int32, device="cuda"))
    c["len"].copy_(lens)
    if bias:
        c["bias"].copy_(torch.rand(S, H, cap, generator=g, device="cuda") * 3.0 - 2.0)
    return c


def _queries(g, c, lens, S, H, n_pos, G):
    """Queries near keys of the cache: reference queries' law, noise 0.5."""
    q = torch.empty(S, H, n_pos, G, D, device="cuda")
    for s in range(S):
        j = torch.randint(0, max(1, int(lens[s])), (n_pos * G,), generator=g, device="cuda")
        k = c["K"][s][:, j].float() - 128.0
        q[s] = (k * c["k_scale"][s][:, j // B].unsqueeze(-1)).view(H, n_pos, G, D)
    q += 0.5 * torch.randn(q.shape, generator=g, device="cuda")
    return q.to(torch.bfloat16)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    S, H = case["S"], case["H"]
    if case["kind"] == "append":
        at = _lengths(case, g, case["old"]) if case["old"] else torch.zeros(S, dtype=torch.int32, device="cuda")
        # every pass writes the same tokens again, as a rejected draft is written over: the rows before them in their
        # block have to be staged still, so the write ends in the block that it begins in, or begins with a block
        at = at // B * B + torch.clamp(at % B, max=max(0, B - case["n"]))
        cap = -(-(case["old"] + case["n"]) // B) * B
        c = _filled(g, S, H, cap, at, False)
        dt = torch.bfloat16 if case["src"] == "bf16" else torch.float32
        st = {"K": _rows(g, S, H, case["n"], dt, True), "V": _rows(g, S, H, case["n"], dt, False), "at": at}
    else:
        lens = _lengths(case, g, case["len"])
        c = _filled(g, S, H, -(-case["len"] // B) * B, lens, case.get("bias", False))
        st = {"Q": _queries(g, c, lens, S, H, case["n_pos"], case["G"])}
    st["case"], st["cache"] = case, c
    if own:
        import paper_2609_36835_gb300 as pk
        st["cache"] = pk.Cache8(**c)
        if case["kind"] != "append":
            st["ws"] = pk.cache_workspace(st["cache"], case["n_pos"], case["G"])
    return st


# ----------------------------------------------------------------- plain form

def _quantise(x, valid):
    """Codes and scale of blocks x [..., B, D]; rows that are not valid count for nothing."""
    x = x * valid.unsqueeze(-1)
    a = x.abs().amax(dim=(-2, -1)).clamp_min(FLOOR)
    return torch.round(x * (torch.full_like(a, 127.0) / a)[..., None, None]), a * STEP


def _plain_append(c, K, V, at):
    """New rows at tokens at .. at + n of every sequence; returns the first block written and the values of the blocks."""
    S, H, n, _ = K.shape
    nb = (n + 2 * B - 2) // B
    b0 = (at // B).long()
    tok = b0[:, None] * B + torch.arange(nb * B, device="cuda")           # [S, nb * B]
    at_, end = at.long()[:, None], at.long()[:, None] + n
    seq = torch.arange(S, device="cuda")[:, None]
    blk = b0[:, None] + torch.arange(nb, device="cuda")                   # [S, nb]
    there = (blk * B < end)                                               # blocks that hold a token
    valid = (tok < end).view(S, 1, nb, B)
    old = (tok < at_).view(S, 1, nb * B, 1)
    last = (end[:, 0] - 1) // B - b0                                      # the block whose rows stay staged
    values = []
    for which, x in ((0, K), (1, V)):
        src = (tok - at_).clamp(0, n - 1)
        new = x.transpose(1, 2)[seq, src].transpose(1, 2).float()         # [S, H, nb * B, D]
        staged = c["tail"][:, :, which].repeat(1, 1, nb, 1)
        rows = torch.where(old, staged, new).view(S, H, nb, B, D)
        codes, scale = _quantise(rows, valid.expand(S, H, nb, B).float())
        values.append((codes * scale[..., None, None]).view(S, H, nb * B, D))
        s_at, b_at = there.nonzero(as_tuple=True)
        c["KV"[which]].view(S, H, -1, B, D)[s_at, :, blk[s_at, b_at]] = (codes + 128.0).to(torch.uint8)[s_at, :, b_at]
        c[("k_scale", "v_scale")[which]][s_at, :, blk[s_at, b_at]] = scale[s_at, :, b_at]
        if which == 0:
            inf = torch.where(valid, 0.0, 1000.0).unsqueeze(-1)
            lo, hi = (codes + inf).amin(3), (codes - inf).amax(3)
            c["bounds"][s_at, :, blk[s_at, b_at]] = torch.stack([lo, hi], 3).to(torch.int8)[s_at, :, b_at]
        keep = (rows * valid.unsqueeze(-1))[torch.arange(S, device="cuda"), :, last]
        c["tail"][:, :, which] = keep
        c["tail_amax"][:, :, which] = keep.abs().amax(-1)
    c["len"].copy_(end[:, 0])
    return tok, valid, values


def _plain_append_run(st):
    c, K, V, at = st["cache"], st["K"], st["V"], st["at"]
    n = K.shape[2]
    tok, _, values = _plain_append(c, K, V, at)
    count = n if n >= B else B                                            # what is read back: the last `count` tokens
    want = (at.long() + n - count)[:, None] + torch.arange(count, device="cuda")
    out = {}
    seq = torch.arange(K.shape[0], device="cuda")[:, None]
    for name, x, scale in (("K", c["K"], c["k_scale"]), ("V", c["V"], c["v_scale"])):
        w = want.clamp_min(0)
        codes = x.transpose(1, 2)[seq, w].transpose(1, 2).float() - 128.0
        s = scale.transpose(1, 2)[seq, w // B].transpose(1, 2)
        out[name] = torch.where((want >= 0)[:, None, :, None], codes * s.unsqueeze(-1), 0.0).to(torch.bfloat16)
    out["len"] = c["len"]
    return out


def _plain_values(x, scale):
    S, H, cap, _ = x.shape
    return ((x.float() - 128.0).view(S, H, cap // B, B, D) * scale[..., None, None]).view(S, H, cap, D)


def _plain_softmax_rows(logits, seen):
    """exp(l - max) / sum over the seen entries; rows that see nothing are zero."""
    logits = logits.masked_fill(~seen, -math.inf)
    top = logits.amax(-1, keepdim=True)
    p = torch.exp(logits - torch.where(torch.isinf(top), 0.0, top))
    total = p.sum(-1, keepdim=True)
    return p / torch.where(total == 0, 1.0, total)


def _visible(c, n_pos, causal):
    """Tokens that each position sees, [S, n_pos]."""
    n = c["len"].long()[:, None].expand(-1, n_pos)
    return (n - n_pos + 1 + torch.arange(n_pos, device="cuda")).clamp_min(0) if causal else n


def _plain_attend(st):
    c, Q, case = st["cache"], st["Q"], st["case"]
    S, H, n_pos, G, _ = Q.shape
    K, V = _plain_values(c["K"], c["k_scale"]), _plain_values(c["V"], c["v_scale"])
    logits = torch.matmul(Q.float().view(S, H, n_pos * G, D), K.transpose(2, 3)) / math.sqrt(D)
    if c["bias"] is not None:
        logits = logits + c["bias"].unsqueeze(2)
    seen = torch.arange(K.shape[2], device="cuda") < _visible(c, n_pos, case["causal"])[..., None]     # [S, n_pos, cap]
    seen = seen[:, None, :, None].expand(S, 1, n_pos, G, -1).reshape(S, 1, n_pos * G, -1)
    return {"O": torch.matmul(_plain_softmax_rows(logits, seen), V).view(S, H, n_pos, G, D)}


def _plain_select(c, Q, m):
    """The m blocks of the highest scores of each position (the first and the newest always), ascending, -1 after the last."""
    S, H, n_pos, G, _ = Q.shape
    nb = c["k_scale"].shape[2]
    q = Q.float()
    a = q.abs().amax(-1, keepdim=True).clamp_min(FLOOR)
    qc = torch.round(q * (torch.full_like(a, 127.0) / a))
    lo, hi = c["bounds"][:, :, :, 0].float(), c["bounds"][:, :, :, 1].float()
    qc = qc.view(S, H, n_pos * G, D)
    whole = torch.matmul(qc.clamp_min(0), hi.transpose(2, 3)) + torch.matmul(qc.clamp_max(0), lo.transpose(2, 3))
    s_q = (a * STEP).view(S, H, n_pos * G, 1)
    score = ((s_q * whole) * c["k_scale"].unsqueeze(2)).view(S, H, n_pos, G, nb).amax(3)
    cand = (_visible(c, n_pos, n_pos > 1) + B - 1) // B                   # [S, n_pos]
    j = torch.arange(nb, device="cuda")
    cand_ = cand[:, None, :, None]
    score = torch.where((j < 1) | (j == cand_ - 1), math.inf, score)
    score = torch.where(j < cand_, score, -math.inf).expand(S, H, n_pos, nb)
    k = min(m, nb)
    best = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :k]
    best = torch.where(best < cand_, best, nb)
    best = torch.sort(best, dim=-1).values
    best = torch.where(best < nb, best, -1).to(torch.int32)
    return torch.nn.functional.pad(best, (0, m - k), value=-1)


def _plain_sparse(st):
    c, Q, case = st["cache"], st["Q"], st["case"]
    S, H, n_pos, G, _ = Q.shape
    idx = _plain_select(c, Q, case["m"])
    m = idx.shape[-1]
    nb = c["k_scale"].shape[2]
    at = idx.clamp_min(0).long()
    flat = (torch.arange(S * H, device="cuda").view(S, H, 1, 1) * nb + at)
    pick = lambda x, s: ((x.view(S * H * nb, B, D)[flat].float() - 128.0) * s.reshape(-1)[flat][..., None, None]).view(S, H, n_pos, m * B, D)   # noqa: E731
    logits = torch.matmul(Q.float(), pick(c["K"], c["k_scale"]).transpose(3, 4)) / math.sqrt(D)
    tok = (at[..., None] * B + torch.arange(B, device="cuda")).view(S, H, n_pos, 1, m * B)
    seen = (tok < _visible(c, n_pos, n_pos > 1)[:, None, :, None, None]) & (idx >= 0).repeat_interleave(B, -1).unsqueeze(3)
    return {"blocks": idx, "O": torch.matmul(_plain_softmax_rows(logits, seen), pick(c["V"], c["v_scale"]))}


# ------------------------------------------------------------------------ run

def run(st):
    case = st["case"]
    if not own:
        return {"append": _plain_append_run, "attend": _plain_attend, "sparse": _plain_sparse}[case["kind"]](st)
    import paper_2609_36835_gb300 as pk
    c = st["cache"]
    if case["kind"] == "append":
        pk.cache_append(c, st["K"], st["V"], at=st["at"], check=False)
        count = max(case["n"], B)
        K, V = pk.cache_read(c, -count, count, dtype=torch.bfloat16, check=False)
        return {"K": K, "V": V, "len": c.len}
    if case["kind"] == "attend":
        return {"O": pk.cache_attend(c, st["Q"], causal=case["causal"], ws=st["ws"], check=False)}
    causal = case["n_pos"] > 1
    blocks = pk.cache_select(c, st["Q"], case["m"], causal=causal, ws=st["ws"], check=False)
    return {"blocks": blocks, "O": pk.cache_attend(c, st["Q"], blocks=blocks, causal=causal, ws=st["ws"], check=False)}


# ----------------------------------------------------------------------- work

def work(case):
    """Bytes and operations at the mean length: sources and cache once, outputs once."""
    S, H = case["S"], case["H"]
    mean = lambda most: most * (0.75 if case["ragged"] else 1.0)   # noqa: E731
    if case["kind"] == "append":
        n, width = case["n"], 2 if case["src"] == "bf16" else 4
        count = max(n, B)
        scales = (n // B + 1) * (2 * D + 8)
        return {"bytes": S * H * (2 * n * D * width + 2 * n * D + scales + 2 * count * D + 2 * count * D * 2), "flops": 2 * S * H * n * D * 3}
    G, n_pos = case["G"], case["n_pos"]
    n = n_pos * G
    io = S * H * n * D * (2 + 4)
    if case["kind"] == "attend":
        T = mean(case["len"])
        seen = T - n_pos / 2 if case["causal"] and T > n_pos else T
        per = 2 * D + 8 / B + (4 if case["bias"] else 0)
        return {"bytes": S * H * T * per + io, "flops": 4 * S * H * n * seen * D}
    nb = mean(case["len"]) / B
    m = min(case["m"], nb)
    distinct = min(nb, m * n_pos)
    return {"bytes": S * H * (nb * (2 * D + 4) + distinct * (2 * B * D + 8) + n_pos * case["m"] * 4) + io,
            "flops": S * H * n * (4 * m * B * D + 4 * nb * D)}


# ---------------------------------------------------------------------- exact

def _exact_append(case, seed):
    st = prepare(case, seed)
    c = st["cache"] if isinstance(st["cache"], dict) else vars(st["cache"])
    S, H, n, _ = st["K"].shape
    count = max(n, B)
    out = {"len": None}
    for which, name in ((0, "K"), (1, "V")):
        val = torch.zeros(S, H, count, D, dtype=torch.float64, device="cuda")
        for s in range(S):
            at = int(st["at"][s])
            first = at // B * B
            rows = torch.cat([c["tail"][s, :, which, :at - first].double(), st[name][s].double()], 1)    # [H, rows, D] from token `first`
            r = rows.shape[1]
            full = torch.nn.functional.pad(rows, (0, 0, 0, -r % B)).view(H, -1, B, D)
            a = full.abs().amax(dim=(2, 3), keepdim=True).clamp_min(FLOOR)
            got = (torch.round(full * (127.0 / a)) * (a / 127.0)).view(H, -1, D)[:, :r]
            lo = at + n - count                                              # first token that is read back
            if lo < first:                                                   # earlier blocks as they stand
                p, q = max(lo, 0), first
                x = c[name][s, :, p:q].double() - 128.0
                x = x * c[("k_scale", "v_scale")[which]][s].double()[:, torch.arange(p, q, device="cuda") // B].unsqueeze(-1)
                got, lo_ = torch.cat([x, got], 1), p
            else:
                got, lo_ = got[:, lo - first:], lo
            val[s, :, lo_ - lo:] = got
        out[name] = val
    return out


def _exact_rows(q, k, v, bias, visible):
    """softmax(q k^T / sqrt(D) + bias) v in 64 bits; row i sees the first visible[i] keys."""
    a = q @ k.T / math.sqrt(D) + bias
    a = a.masked_fill(torch.arange(k.shape[0], device="cuda") >= visible[:, None], -math.inf)
    top = a.max(dim=1, keepdim=True).values
    e = torch.exp(a - top.masked_fill(top == -math.inf, 0.0))
    z = e.sum(1, keepdim=True)
    return (e @ v) / z.masked_fill(z == 0, 1.0)


def exact(case, seed):
    if case["kind"] == "append":
        return _exact_append(case, seed)
    G, n_pos = case["G"], case["n_pos"]
    if case["S"] * case["H"] * n_pos * G * case["len"] > 6e9 or case["S"] * case["H"] * (n_pos if case["kind"] == "sparse" else 1) > 3000:
        return None
    st = prepare(case, seed)
    c = st["cache"] if isinstance(st["cache"], dict) else vars(st["cache"])
    S, H = case["S"], case["H"]
    causal = case["causal"] if case["kind"] == "attend" else n_pos > 1
    O = torch.zeros(S, H, n_pos, G, D, dtype=torch.float64, device="cuda")
    lens = c["len"].tolist()
    for s in range(S):
        T = lens[s]
        nb = -(-T // B)
        step = torch.arange(T, device="cuda") // B
        for h in range(H):
            k = (c["K"][s, h, :T].double() - 128) * c["k_scale"][s, h, step].double()[:, None]
            v = (c["V"][s, h, :T].double() - 128) * c["v_scale"][s, h, step].double()[:, None]
            bias = c["bias"][s, h, :T].double() if c["bias"] is not None else torch.zeros(T, dtype=torch.float64, device="cuda")
            q = st["Q"][s, h].double()
            if case["kind"] == "attend":
                seen = torch.tensor([max(0, T - n_pos + 1 + p) if causal else T for p in range(n_pos)], device="cuda").repeat_interleave(G)
                rows = q.view(-1, D)
                for i in range(0, rows.shape[0], 512):
                    O[s, h].view(-1, D)[i:i + 512] = _exact_rows(rows[i:i + 512], k, v, bias, seen[i:i + 512])
                continue
            low, high = c["bounds"][s, h, :nb, 0].double(), c["bounds"][s, h, :nb, 1].double()
            for p in range(n_pos):
                sees = max(0, T - n_pos + 1 + p) if causal else T
                cand = -(-sees // B)
                if cand == 0:
                    continue
                # the score is defined with its roundings to 32 bits: quantised query, scale of the query, scale of the block
                best = torch.full((cand,), -math.inf, dtype=torch.float64, device="cuda")
                for g in range(G):
                    a = q[p, g].abs().max().clamp_min(FLOOR)
                    qc = torch.round((q[p, g] * (127.0 / a).float().double()).float()).double()
                    bound = torch.maximum(qc * low[:cand], qc * high[:cand]).sum(1)
                    sq = (a * STEP).float().double()
                    best = torch.maximum(best, ((sq * bound).float().double() * c["k_scale"][s, h, :cand].double()).float().double())
                best[0] = math.inf
                best[cand - 1] = math.inf
                order = sorted(range(cand), key=lambda b, w=best.tolist(): (-w[b], b))[:case["m"]] if cand > case["m"] else range(cand)
                tok = torch.tensor(sorted(order), device="cuda")[:, None] * B + torch.arange(B, device="cuda")
                tok = tok.view(-1)
                tok = tok[tok < sees]
                O[s, h, p] = _exact_rows(q[p], k[tok], v[tok], bias[tok], torch.full((G,), tok.numel(), device="cuda"))
    return {"O": O} if case["kind"] == "attend" else {"O": O, "blocks": None}
