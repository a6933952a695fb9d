"""A serving loop over paged caches held in 4 bits.

Requests of different lengths share one pool of pages.  Prompts come in chunks beside requests that are decoding already: a
step makes room for the new tokens, rotates queries and keys, writes the keys and values into the pages and attends, all
requests packed row after row.  When every prompt is in, the steps have one token a request; such a step is captured in a CUDA
graph once and replayed while the requests grow.  Then the requests end and their pages go back to the pool.

The model is one attention layer of Llama-3.1-8B's shape with random queries, keys and values.

    python examples/serve_4bit.py [--requests 16] [--longest 4096] [--chunk 512] [--steps 64]
"""
from __future__ import annotations

import argparse
import sys
from pathlib import Path

ROOT = Path(__file__).resolve().parent.parent
if str(ROOT) not in sys.path:
    sys.path.insert(0, str(ROOT))


def main(argv=None) -> dict:
    import torch

    import paper_2609_36835_gb300 as pk

    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--requests", type=int, default=16)
    ap.add_argument("--longest", type=int, default=4096, help="tokens of the longest prompt")
    ap.add_argument("--chunk", type=int, default=512, help="tokens of a prompt that a step takes")
    ap.add_argument("--steps", type=int, default=64, help="tokens that each request decodes")
    args = ap.parse_args(argv)
    dev = torch.device("cuda:0")
    torch.cuda.set_device(dev)
    S, H, G = args.requests, 8, 4
    g = torch.Generator(device=dev)
    g.manual_seed(11)
    prompts = torch.randint(max(1, args.longest // 4), args.longest + 1, (S,), generator=g, device=dev).tolist()
    room = max(prompts) + args.steps + 1
    pages = pk.pages_alloc(S, H, sum(-(-(n + args.steps + 1) // pk.PAGE_TOKENS) for n in prompts), room, device=dev)
    rotary = pk.rotary(128, 500000.0, scaling={"kind": "bands", "factor": 8.0, "low": 1.0, "high": 4.0, "context": 8192}, device=dev)

    def step(qkv, counts, most, out, ws):
        """One layer's attention for the packed rows qkv [N, (G + 2) H, 128] of this step's tokens."""
        starts, slots, positions = pk.pages_extend(pages, counts, qkv.shape[0], check=False)
        q, k, v = qkv[:, :H * G], qkv[:, H * G:H * G + H], qkv[:, H * G + H:]
        pk.rotate(rotary, positions, q, k, out=(q, k))
        pk.pages_append(pages, k, v, slots, check=False)
        return pk.pages_attend(pages, q.unflatten(1, (H, G)), starts, max_count=most, out=out, ws=ws, check=False)

    def rows(n):
        return torch.randn(n, (G + 2) * H, 128, generator=g, device=dev).to(torch.bfloat16)

    # prompts, a chunk of one request at a time beside a token of each that is done; what one request has, for the check
    ws = pk.pages_workspace(pages, args.chunk, G)
    kept_k, kept_v, left, checked = [], [], list(prompts), S // 2
    prompt_steps = 0
    while any(left):
        s = next(i for i in range(S) if left[i])
        decodes = prompt_steps < args.steps // 2        # (a request decodes no more than its pages suffice for)
        counts = [int(decodes and left[i] == 0) for i in range(S)]
        counts[s] = min(args.chunk, left[s])
        N = sum(counts)
        qkv = rows(N)
        step(qkv, torch.tensor(counts, dtype=torch.int32, device=dev), args.chunk, None, ws)
        at = sum(counts[:checked])
        kept_k.append(qkv[at:at + counts[checked], H * G:H * G + H])
        kept_v.append(qkv[at:at + counts[checked], H * G + H:])
        left[s] -= counts[s]
        prompt_steps += 1

    # decode, replayed
    held = pages.len.tolist()
    steps = min(args.steps // 2, room - max(held) - 1)
    one = torch.ones(S, dtype=torch.int32, device=dev)
    qkv, out, ws = rows(S), torch.empty(S, H, G, 128, dtype=torch.bfloat16, device=dev), pk.pages_workspace(pages, 1, G)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(qkv.clone(), one, 1, out, ws)              # what a first call sets up
        pk.pages_truncate(pages, torch.tensor(held, dtype=torch.int32, device=dev))
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(qkv, one, 1, out, ws)
    new = rows(steps * S).view(steps, S, -1, 128)
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    e0.record()
    for x in new:
        qkv.copy_(x)
        graph.replay()
    e1.record()
    torch.cuda.synchronize()
    for word in (pages.state, ws):
        status = pk.arckv_query_status(word)
        if status != 0:
            raise pk.ArckvError(status, "serve_4bit")

    # the last token of one request against attention over its rows as they were, before they were held in 4 bits
    mine = new[:, checked]
    kept_k.append(pk.rotate(rotary, torch.arange(held[checked], held[checked] + steps, dtype=torch.int32, device=dev),
                            mine[:, H * G:H * G + H]))
    kept_v.append(mine[:, H * G + H:])
    Q = qkv[checked, :H * G].view(H, G, 128).contiguous()
    K, V = torch.cat(kept_k).transpose(0, 1).contiguous(), torch.cat(kept_v).transpose(0, 1).contiguous()
    ref = pk.attend_joint(Q, K_fixed=K, V_fixed=V)
    tokens, free = int(pages.len.sum()), int(pages.n_free[0])
    pk.pages_truncate(pages, torch.zeros(S, dtype=torch.int32, device=dev))      # the requests end
    figures = {
        "requests": S, "tokens": tokens, "pages_used": pages.free.shape[0] - free, "pages": pages.free.shape[0],
        "pages_free_after": int(pages.n_free[0]),
        "length": K.shape[1], "us_per_step": e0.elapsed_time(e1) * 1e3 / max(1, steps), "prompt_steps": prompt_steps,
        "error": float((out[checked].float() - ref).norm() / ref.norm()),
    }
    print("%(requests)d requests, %(tokens)d tokens in %(pages_used)d pages after %(prompt_steps)d prompt steps; %(us_per_step).1f us a "
          "decode step (one layer)\nerror of a request of %(length)d tokens against bf16 caches: %(error).1e" % figures)
    return figures


if __name__ == "__main__":
    main()
