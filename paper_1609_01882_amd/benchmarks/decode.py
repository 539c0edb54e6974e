"""Attention over a memory held in 4 bits and to a budget, as a generating model's layer would use it: a prompt is written
and attended to in chunks, cut to the budget by the weights that its tokens received, then tokens follow one at a time --
appended, attended, and the memory cut again whenever it is `--slack` tokens over.  Random vectors stand in for the
layer's queries, keys and values.  Prints one JSON line: milliseconds for the prompt, for a token eagerly and as a replayed
HIP graph, and how far the first chunk's outputs are from attention over the vectors as they were.  `--rotary` turns that many
coordinates of queries and keys by their positions, on their way into the memory; `--differential` takes the difference of two maps over
pairs of kv heads, normed; `--stream` puts a residual stream of that width around it, normed before and after, gated.

    python -m paper_1609_01882_amd.benchmarks.decode --batch 16 --prompt 16384 --budget 4096 --tokens 256
    python -m paper_1609_01882_amd.benchmarks.decode --rotary 128 --differential --stream 4096
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
    ap.add_argument("--rotary", type=int, default=0, help="coordinates of a head that are turned by their position (a multiple of 16)")
    ap.add_argument("--differential", action="store_true", help="two maps over pairs of kv heads")
    ap.add_argument("--stream", type=int, default=0, help="width of a residual stream around the attention")
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

    rope = psc.Rotary(args.rotary) if args.rotary else None
    q_heads = heads * group
    lam = torch.full((q_heads // 2,), 0.3, device="cuda")
    norm = torch.ones(2 * dim, device="cuda")
    ones = torch.ones(max(args.stream, 1), device="cuda")

    def put(q, k, v, lengths, first, **out):
        """Keys and values into the memory; the queries as attention takes them."""
        if rope is None:
            cache.append(k, v, table, lengths, first=first, positions=positions, weights=weights)
            return q
        return cache.append(k, v, table, lengths, first=first, positions=positions, weights=weights, rotary=rope, q=q, **out)

    def write(q, k, v, rows):
        q = put(q, k, v, lengths, seen)
        lengths.add_(rows)
        seen.add_(rows)
        return q

    def attend_any(q, lengths, **more):
        more = dict(weights=weights, weights_out=weights, **more)
        if args.differential:
            return cache.attend_difference(q, lam, table, lengths, norm=norm, factor=0.7, **more)
        return cache.attend(q, table, lengths, **more)

    def attend(q, rows, **more):
        # nothing has been cut while the prompt is read: slots are positions
        return attend_any(q, lengths, first=seen - rows, **more)

    def around(out):
        """The norms, gate and residual before and behind the attention; the products between them are not part of this."""
        if args.stream:
            rows = out.shape[0]
            x, y = (torch.randn((rows, args.stream), generator=g, device="cuda").bfloat16() for _ in range(2))
            x, _ = psc.residual_norm(x, before=ones)
            psc.residual_norm(x, y, gate=y, activation="sigmoid", after=ones, before=ones)
        return out

    def cut():
        kept = torch.empty((batch, heads, args.budget), dtype=torch.int32, device="cuda")
        cache.evict(table, lengths, weights, args.budget, sinks=args.sinks, recent=args.recent, positions=positions, seen=seen,
                    out=(kept, lengths, positions, weights))

    def prompt():
        first = None
        for at in range(0, args.prompt, args.chunk):
            rows = min(args.chunk, args.prompt - at)
            q, k, v = qkv(rows)
            turned = write(q, k, v, rows)
            out = around(attend(turned, rows)[0])
            first = first or (q, k, v, out, rows)
        cut()
        return first

    def as_they_were(q, k, v, rows):
        """Attention of sequence 0's first rows over the vectors before rounding."""
        q, k, v = (x[:rows].float() for x in (q, k, v))
        if rope is not None:
            q, k = rope(q), rope(k)
        q, k, v = (x.transpose(0, 1) for x in (q, k, v))
        s = (q.reshape(heads, group * rows, dim) @ k.transpose(1, 2).contiguous()).view(heads, group, rows, rows) / math.sqrt(dim)
        p = s.masked_fill(torch.ones((rows, rows), dtype=torch.bool, device="cuda").triu(1), -math.inf).softmax(-1)
        if not args.differential:
            return (p.reshape(heads, group * rows, rows) @ v).reshape(heads * group, rows, dim).transpose(0, 1)
        pairs, both = heads // 2, torch.cat((v[0::2], v[1::2]), -1)
        p = p.view(pairs, 2, group, rows, rows)
        o = ((p[:, 0] - 0.3 * p[:, 1]).reshape(pairs, group * rows, rows) @ both).reshape(pairs * group, rows, 2 * dim)
        return (0.7 * o * torch.rsqrt(o.square().mean(-1, keepdim=True) + 1e-6)).transpose(0, 1)

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
        q = write(q, k, v, 1)
        around(attend_any(q, lengths, first=seen - 1, positions=positions)[0])
        held += 1
        if held >= args.budget + args.slack:
            cut()
            held = args.budget
    assert bool((lengths == held).all()) and bool((seen == args.prompt + args.tokens).all())

    # one token into the memory as it is now, over and over
    q, k, v = qkv(1)
    before, after = lengths - 1, lengths.clone()
    at = seen - 1
    shape = (batch, q_heads // 2, 2 * dim) if args.differential else (batch, q_heads, dim)
    res = (torch.empty(shape, dtype=q.dtype, device="cuda"), torch.empty((batch, q_heads), device="cuda"))
    space = cache.attend_difference_workspace_bytes if args.differential else cache.attend_workspace_bytes
    ws = torch.empty(space(batch, width, batch, 1, q_heads, q.dtype, positions=True, weights=True), dtype=torch.uint8, device="cuda")
    turned = torch.empty((batch, q_heads, dim), dtype=q.dtype, device="cuda")
    x, y = (torch.randn((batch, max(args.stream, 1)), generator=g, device="cuda").bfloat16() for _ in range(2))

    def token():
        if args.stream:
            psc.residual_norm(x, before=ones)
        attend_any(put(q, k, v, before, at, q_out=turned), after, first=at, positions=positions, out=res, workspace=ws)
        if args.stream:
            psc.residual_norm(x, y, gate=y, activation="sigmoid", after=ones, before=ones)

    print(json.dumps({
        "metric": "attention memory in 4 bits, one layer", "unit": "ms", "batch": batch, "kv_heads": heads, "query_heads": heads * group,
        "head_dim": dim, "rotary": args.rotary, "differential": args.differential, "stream": args.stream, "prompt": args.prompt, "budget": args.budget, "dtype": "bf16 over 4-bit floats", "data": "synthetic",
        "prompt_ms": prompt_ms, "token_ms": time_ms(token, 200, 20), "token_replayed_ms": graph_replay_ms(token, 200),
        "cut_ms": time_ms(lambda: (lengths.fill_(args.budget + args.slack), cut()), 20, 3), "bytes_of_a_token": heads * (dim + dim // 16), "bytes_of_a_token_bf16": heads * dim * 4,
        "first_chunk_off_by": off}))


if __name__ == "__main__":
    main()
