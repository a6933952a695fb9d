"""Decode steps over a compacted context that is held in 8 bits.

A Llama-3.1-8B-shaped layer (synthetic, seeded) is compacted with ``arckv_compact``; its compact keys, values and biases
are written into an 8-bit cache, and a decode loop then writes each new token behind them and attends over everything.
Beside it the full context is held in 8 bits too, and read whole and, for each query, only in the blocks that a bound of
their logits selects.  A step (write, select, attend) is captured in a CUDA graph once and replayed while the caches grow.

    python examples/decode_8bit.py [--context 8192] [--steps 64] [--blocks 16]
"""
from __future__ import annotations

import argparse
import sys
from pathlib import Path

ROOT = Path(__file__).resolve().parent.parent
if str(ROOT) not in sys.path:
    sys.path.insert(0, str(ROOT))


def rel(a, b) -> float:
    return float((a - b).norm() / b.norm())


def main(argv=None) -> dict:
    import torch

    import paper_2609_36835_gb300 as pk
    import synth
    from paper_2609_36835_gb300 import workload

    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--context", type=int, default=8192)
    ap.add_argument("--steps", type=int, default=64)
    ap.add_argument("--blocks", type=int, default=16, help="blocks of 64 tokens that the sparse read takes")
    args = ap.parse_args(argv)
    dev = torch.device("cuda:0")
    torch.cuda.set_device(dev)

    # one layer of a context, compacted to a tenth
    w = synth.WORKLOADS["llama8b_layer_T8192"]
    H, G, T = w.H_kv, w.G, args.context
    arr = workload.layer_inputs_np(w, 0, list(range(H)), T=T, n_pos=64)
    ten = workload.to_device(arr, dev)
    cfg = workload.layer_config(w, H, T=T, n_pos=64, t=max(1, T // 10))
    out = pk.compact_layer(cfg, ten["K"], ten["V"], ten["Q"], ten["X"], workload.indexer_dict(ten))

    # both caches in 8 bits, with room for the new tokens
    t = out["C_k"].shape[1]
    compact = pk.cache_alloc(1, H, t + args.steps, bias=True, device=dev)
    pk.cache_append(compact, out["C_k"][None], out["C_v"][None], bias=out["beta"][None])
    full = pk.cache_alloc(1, H, T + args.steps, device=dev)
    pk.cache_append(full, ten["K"][None], ten["V"][None])
    ws_c, ws_f = pk.cache_workspace(compact, 1, G), pk.cache_workspace(full, 1, G)

    # new tokens and queries near keys of the context, one step each
    g = torch.Generator(device=dev)
    g.manual_seed(7)
    noise = lambda *s: torch.randn(*s, generator=g, device=dev)   # noqa: E731
    n = args.steps
    new_k, new_v = noise(1, H, n, 128).to(torch.bfloat16), noise(1, H, n, 128).to(torch.bfloat16)
    at = torch.randint(0, T, (n, G), generator=g, device=dev)
    queries = (ten["K"][:, at].float() + 0.5 * noise(H, n, G, 128)).to(torch.bfloat16)[None]   # [1, H, n, G, 128]

    k, v, q = new_k[:, :, :1].clone(), new_v[:, :, :1].clone(), queries[:, :, :1].clone()
    o = {name: torch.empty(1, H, 1, G, 128, device=dev) for name in ("compact", "full", "sparse")}

    def step():
        for c in (compact, full):
            pk.cache_append(c, k, v, check=False)
        pk.cache_attend(compact, q, out=o["compact"], ws=ws_c, check=False)
        pk.cache_attend(full, q, out=o["full"], ws=ws_f, check=False)
        blocks = pk.cache_select(full, q, args.blocks, ws=ws_f, check=False)
        pk.cache_attend(full, q, blocks=blocks, out=o["sparse"], ws=ws_f, check=False)
        return blocks

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()                                     # the first token, and what a first call sets up
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        blocks = step()
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    e0.record()
    for i in range(1, n):
        k.copy_(new_k[:, :, i:i + 1])
        v.copy_(new_v[:, :, i:i + 1])
        q.copy_(queries[:, :, i:i + 1])
        graph.replay()
    e1.record()
    torch.cuda.synchronize()
    for word in (compact.state, full.state, ws_c, ws_f):
        status = pk.arckv_query_status(word)
        if status != 0:
            raise pk.ArckvError(status, "decode_8bit")

    # the last step against the same attention over bf16 / fp32 caches
    Q = q[0, :, 0]
    K, V = torch.cat([ten["K"], new_k[0]], 1), torch.cat([ten["V"], new_v[0]], 1)
    ref_full = pk.attend_joint(Q, K_fixed=K, V_fixed=V)
    ref_compact = pk.attend_joint(Q, out["C_k"], out["beta"], out["C_v"], new_k[0].contiguous(), new_v[0].contiguous())
    # the tokens of the selected blocks (every head lists the newest one, so all have the same number of them)
    tok = (blocks[0, :, 0].long()[:, :, None] * pk.CACHE_BLOCK + torch.arange(pk.CACHE_BLOCK, device=dev)).flatten(1)
    tok = torch.stack([x[(x >= 0) & (x < K.shape[1])] for x in tok])[:, :, None].expand(-1, -1, 128)
    ref_sparse = pk.attend_joint(Q, K_fixed=K.gather(1, tok), V_fixed=V.gather(1, tok))
    got = {name: x[0, :, 0] for name, x in o.items()}
    figures = {
        "tokens": int(full.len[0]), "compact_tokens": int(compact.len[0]),
        "us_per_step": e0.elapsed_time(e1) * 1e3 / max(1, n - 1),
        "full_error": rel(got["full"], ref_full), "compact_error": rel(got["compact"], ref_compact),
        "sparse_error": rel(got["sparse"], ref_sparse),
    }
    print("context %(tokens)d tokens, compact %(compact_tokens)d; %(us_per_step).1f us a step (two writes, three reads, one "
          "layer)\nerror against bf16 / fp32 caches: full %(full_error).1e, compact %(compact_error).1e, the "
          "selected blocks %(sparse_error).1e" % figures)
    return figures


if __name__ == "__main__":
    main()
