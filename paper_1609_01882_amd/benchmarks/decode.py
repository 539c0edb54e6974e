"""Attention over a memory held in 4 bits and to a budget, as a generating model's layer would use it: a prompt is written
and attended to in chunks, cut to the budget by the weights that its tokens received, then tokens follow one at a time --
appended, attended, and the memory cut again whenever it is `--slack` tokens over.  Random vectors stand in for the
layer's queries, keys and values.  Prints one JSON line: milliseconds for the prompt, for a token eagerly and as a replayed
HIP graph, and how far the first chunk's outputs are from attention over the vectors as they were.

    python -m paper_1609_01882_amd.benchmarks.decode --batch 16 --prompt 16384 --budget 4096 --tokens 256
"""
from __future__ import annotations

import argparse
import json
import math


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--batch", type=int, default=16)
    ap.add_argument("--kv-heads", type=int, default=8)
    ap.add_argument("--group", type=int, default=4, help="query heads of a kv head")
    ap.add_argument("--dim", type=int, default=128, choices=(64, 128, 256))
    ap.add_argument("--page", type=int, default=64)
    ap.add_argument("--prompt", type=int, default=16384)
    ap.add_argument("--chunk", type=int, default=2048)
    ap.add_argument("--budget", type=int, default=4096)
    ap.add_argument("--sinks", type=int, default=4, help="first tokens that are never cut")
    ap.add_argument("--recent", type=int, default=512, help="latest tokens that are never cut")
    ap.add_argument("--slack", type=int, default=64)
    ap.add_argument("--tokens", type=int, default=256)
    args = ap.parse_args()
    import torch

    import paper_1609_01882_amd as psc
    from ._common import graph_replay_ms, time_ms

    batch, heads, dim, group = args.batch, args.kv_heads, args.dim, args.group
    width = -(-max(args.prompt, args.budget + max(args.slack, 1)) // args.page)    # a token is written before the cut
    slots = width * args.page
    cache = psc.KvCache.empty(batch * width, heads, dim, args.page)
    table = torch.randperm(batch * width, device="cuda").int().view(batch, width)
    lengths = torch.zeros(batch, dtype=torch.int32, device="cuda")
    seen = torch.zeros(batch, dtype=torch.int32, device="cuda")
    positions = torch.zeros((batch, heads, slots), dtype=torch.int32, device="cuda")
    weights = torch.zeros((batch, heads, slots), device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(1)

    def qkv(rows):
        """What the layer's product gives: query heads, then key heads, then value heads."""
        x = torch.randn((batch * rows, heads * (group + 2), dim), generator=g, device="cuda").bfloat16()
        return x[:, :heads * group], x[:, heads * group:heads * (group + 1)], x[:, heads * (group + 1):]

    def write(k, v, rows):
        cache.append(k, v, table, lengths, first=seen, positions=positions, weights=weights)
        lengths.add_(rows)
        seen.add_(rows)

    def attend(q, rows, **more):
        # nothing has been cut while the prompt is read: slots are positions
        return cache.attend(q, table, lengths, first=seen - rows, weights=weights, weights_out=weights, **more)

    def cut():
        kept = torch.empty((batch, heads, args.budget), dtype=torch.int32, device="cuda")
        cache.evict(table, lengths, weights, args.budget, sinks=args.sinks, recent=args.recent, positions=positions, seen=seen,
                    out=(kept, lengths, positions, weights))

    def prompt():
        first = None
        for at in range(0, args.prompt, args.chunk):
            rows = min(args.chunk, args.prompt - at)
            q, k, v = qkv(rows)
            write(k, v, rows)
            out = attend(q, rows)[0]
            first = first or (q, k, v, out, rows)
        cut()
        return first

    def as_they_were(q, k, v, rows):
        """Attention of sequence 0's first rows over the vectors before rounding."""
        q, k, v = (x[:rows].float().transpose(0, 1) for x in (q, k, v))
        s = (q.reshape(heads, group * rows, dim) @ k.transpose(1, 2).contiguous()).view(heads, group, rows, rows) / math.sqrt(dim)
        s = s.masked_fill(torch.ones((rows, rows), dtype=torch.bool, device="cuda").triu(1), -math.inf)
        return (s.softmax(-1).reshape(heads, group * rows, rows) @ v).reshape(heads * group, rows, dim).transpose(0, 1)

    q, k, v, out, rows = prompt()
    want = as_they_were(q, k, v, rows)
    off = ((out[:rows].float() - want).norm() / want.norm()).item()
    del q, k, v, out, want
    lengths.zero_()
    seen.zero_()
    prompt_ms = time_ms(lambda: (lengths.zero_(), seen.zero_(), prompt()), 1, 1)

    held = int(lengths.max())
    for step in range(args.tokens):
        q, k, v = qkv(1)
        write(k, v, 1)
        cache.attend(q, table, lengths, first=seen - 1, positions=positions, weights=weights, weights_out=weights)
        held += 1
        if held >= args.budget + args.slack:
            cut()
            held = args.budget
    assert bool((lengths == held).all()) and bool((seen == args.prompt + args.tokens).all())

    # one token into the memory as it is now, over and over
    q, k, v = qkv(1)
    before, after = lengths - 1, lengths.clone()
    at = seen - 1
    res = (torch.empty_like(q.contiguous()), torch.empty(q.shape[:2], device="cuda"))
    ws = torch.empty(cache.attend_workspace_bytes(batch, width, batch, 1, heads * group, q.dtype, positions=True, weights=True),
                     dtype=torch.uint8, device="cuda")

    def token():
        cache.append(k, v, table, before, first=at, positions=positions, weights=weights)
        cache.attend(q, table, after, first=at, positions=positions, weights=weights, weights_out=weights, out=res, workspace=ws)

    print(json.dumps({
        "metric": "attention memory in 4 bits, one layer", "unit": "ms", "batch": batch, "kv_heads": heads, "query_heads": heads * group,
        "head_dim": dim, "prompt": args.prompt, "budget": args.budget, "dtype": "bf16 over 4-bit floats", "data": "synthetic",
        "prompt_ms": prompt_ms, "token_ms": time_ms(token, 200, 20), "token_replayed_ms": graph_replay_ms(token, 200),
        "cut_ms": time_ms(lambda: (lengths.fill_(args.budget + args.slack), cut()), 20, 3), "bytes_of_a_token": heads * (dim + dim // 16), "bytes_of_a_token_bf16": heads * dim * 4,
        "first_chunk_off_by": off}))


if __name__ == "__main__":
    main()
