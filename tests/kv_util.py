"""The attention memory in 4 bits from its definition, in 64 bits on the host, and how far float32 arithmetic with the
kernels' documented roundings may be from it."""
import numpy as np
import torch

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
UNIT = {name: torch.finfo(t).eps / 2 for name, t in TYPES.items()}      # half a step of the type's mantissa


def round_to_4_bits(k, v):
    """k, v [..., d] float64 -> codes [..., d] (0..15), scale bytes [..., d / 32] of both."""
    finite = np.isfinite(k).all(-1) & np.isfinite(v).all(-1)
    res = []
    for x in (k, v):
        x = np.where(finite[..., None], x, 0.0).reshape(*x.shape[:-1], -1, 32)
        top = np.abs(x).max(-1)
        e = np.floor(np.log2(np.where(top > 0, top, 1e-300))) - 2
        e = np.where(top > 7.0 * 2.0 ** e, e + 1, e).clip(-23, 13)
        size = np.minimum(np.abs(x) / 2.0 ** e[..., None], 6.0)
        off = np.abs(size[..., None] - GRID)
        code = off.argmin(-1)                                  # the lower code on a tie ...
        tie = (code < 7) & (np.take_along_axis(off, np.minimum(code + 1, 7)[..., None], -1)[..., 0] == off.min(-1))
        code = np.where(tie & (code % 2 == 1), code + 1, code)  # ... but the even one
        code = (code + 8 * np.signbit(x)).reshape(*x.shape[:-2], -1)
        res += [code.astype(np.uint8), (e + 127).astype(np.uint8)]
    res[1][~finite] = 255
    res[3][~finite] = 127 - 23
    return res


def pack(codes):
    return codes[..., 0::2] | (codes[..., 1::2] << 4)


def values(codes, scales):
    """Packed codes [..., d / 2], scale bytes [..., d / 32] (numpy) -> float64 [..., d]."""
    code = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], 2 * codes.shape[-1])
    x = np.where(code >= 8, -1.0, 1.0) * GRID[code & 7]
    scale = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return x * np.repeat(scale, 32, -1)


def random_cache(rng, pages, heads, page, dim):
    """Host buffers with values of about one."""
    make = lambda: rng.integers(0, 256, (pages, heads, page, dim // 2), dtype=np.uint8)  # noqa: E731
    scale = lambda: rng.integers(124, 127, (pages, heads, page, dim // 32), dtype=np.uint8)  # noqa: E731
    return [make(), scale(), make(), scale()]


def held(buffers, table, b, head, n):
    """K and V [n, dim] (float64) of a sequence's first n slots, and which slots have a page."""
    page, pages = buffers[0].shape[2], buffers[0].shape[0]
    slot = np.arange(n)
    pg = table[b][slot // page]
    there = (pg >= 0) & (pg < pages)
    pg = np.where(there, pg, 0)
    at = slot % page
    k = values(buffers[0][pg, head, at], buffers[1][pg, head, at])
    v = values(buffers[2][pg, head, at], buffers[3][pg, head, at])
    k[~there], v[~there] = 0.0, 0.0
    return k, v, there


def attend(q, buffers, table, lengths, offsets, first, positions, scale, causal, window, sinks, dtype):
    """(out, lse, received) in float64 and the tolerances of each, elementwise.  q [rows, q_heads, dim] float64."""
    heads, page, dim = buffers[0].shape[1], buffers[0].shape[2], q.shape[2]
    group, slots = q.shape[1] // heads, table.shape[1] * page
    out, lse = np.zeros(q.shape), np.full(q.shape[:2], -np.inf)
    got = np.zeros((len(lengths), heads, slots))
    tol_out, tol_lse, tol_got = np.zeros_like(out), np.zeros_like(lse), np.zeros_like(got)
    eps = 2.0 ** -24
    # probabilities are held in float16 (float32 rows: in two), whose steps end at 2^-24 of the largest
    unit_p = torch.finfo(torch.float16).eps / 2
    unit_p = unit_p ** 2 if dtype == "f32" else unit_p
    for b in range(len(lengths)):
        n = min(int(lengths[b]), slots)
        rows = np.arange(offsets[b], offsets[b + 1])
        pos_q = (n - len(rows) if first is None else first[b]) + np.arange(len(rows))
        for h in range(heads):
            k, v, there = held(buffers, table, b, h, n)
            pos_k = np.arange(n) if positions is None else positions[b, h, :n].astype(np.int64)
            for j, r in enumerate(rows):
                sees = there.copy()
                if causal:
                    sees &= pos_k <= pos_q[j]
                if window:
                    sees &= (pos_q[j] - pos_k < window) | (pos_k < sinks)
                if not sees.any():
                    continue
                for hq in range(h * group, (h + 1) * group):
                    s = scale * (k[sees] @ q[r, hq])
                    top = s.max()
                    e = np.exp(s - top)
                    p = e / e.sum()
                    out[r, hq], lse[r, hq] = p @ v[sees], top + np.log(e.sum())
                    if np.isnan(s).any():
                        out[r, hq], lse[r, hq] = np.nan, np.nan
                        continue
                    got[b, h, :n][sees] += p
                    # a score: dim products and sums, then the scaling; a probability: two scores, two roundings of the
                    # scaled ones, exp2, the sum over n
                    span = scale * (np.abs(k[sees]) @ np.abs(q[r, hq])).max()
                    off = 2 * (dim + 4) * eps * span + 4 * eps * np.abs(s).max() + (8 + np.sqrt(n) + n / 64) * eps
                    size = p @ np.abs(v[sees])
                    tol_out[r, hq] = UNIT[dtype] * np.abs(out[r, hq]) + (unit_p + off) * size + 2.0 ** -25 * np.abs(v[sees]).sum(0) / e.sum()
                    tol_lse[r, hq] = off + 4 * eps * abs(lse[r, hq])
                    tol_got[b, h, :n][sees] += p * off + 2.0 ** -125
    return (out, lse, got), (1.01 * tol_out + 1e-30, tol_lse, tol_got + 4 * eps * got)


def evict(lengths, weights, positions, seen, budget, sinks, recent):
    """kept [batch][heads][budget] by sorting on the host."""
    batch, heads = weights.shape[:2]
    kept = np.full((batch, heads, budget), -1, np.int32)
    for b in range(batch):
        n = min(max(int(lengths[b]), 0), weights.shape[2])
        for h in range(heads):
            w = weights[b, h, :n].astype(np.float64)
            pos = np.arange(n) if positions is None else positions[b, h, :n].astype(np.int64)
            stays = (pos < sinks) | (pos >= (n if seen is None else int(seen[b])) - recent)
            rank = sorted(range(n), key=lambda s: (not stays[s], np.isnan(w[s]) and not stays[s],
                                                   0.0 if stays[s] or np.isnan(w[s]) else -w[s], s))
            keep = np.zeros(n, bool)
            keep[rank[:budget]] = True
            source = np.arange(min(n, budget), dtype=np.int32)
            source[~keep[:budget]] = np.flatnonzero(keep[budget:]) + budget
            kept[b, h, :len(source)] = source
    return kept
