"""Rotary positions, differential attention and norms around a block from their definitions, in 64 bits on the host, and how far float32
arithmetic with the kernels' documented roundings may be from them."""
import math

import numpy as np
import torch

import kv_util as U

UNIT, TYPES = U.UNIT, U.TYPES
EPS32 = 2.0 ** -24


def turned(x, positions, frequencies, dims, interleaved, factor=1.0, back=False):
    """x [rows, heads, dim] float64, positions [rows] (integers), frequencies [dims / 2] -> the same shape in 64 bits."""
    y = np.array(x, np.float64)
    i = np.arange(dims // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + dims // 2)
    # angles modulo a turn in more bits than a double has
    t = np.asarray(positions, np.longdouble)[:, None] * np.asarray(frequencies, np.longdouble)
    cos, sin = (np.asarray(f(t), np.float64)[:, None] * factor for f in (np.cos, np.sin))
    sin = -sin if back else sin
    y[..., a], y[..., b] = x[..., a] * cos - x[..., b] * sin, x[..., b] * cos + x[..., a] * sin
    return y


def turned_tolerance(x, dims, interleaved, factor, dtype):
    """Sine and cosine rounded to float32 and scaled, two products and a sum, the output's rounding."""
    i = np.arange(dims // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + dims // 2)
    size = np.abs(np.array(x, np.float64))
    pair = size[..., a] + size[..., b]
    size[..., a] = size[..., b] = pair * abs(factor)
    tol = (UNIT[dtype] + 4 * EPS32) * size
    return 1.01 * tol + (2.0 ** -25 if dtype == "f16" else 2.0 ** -134)      # denormal float16 / bfloat16 steps


def difference(q, lam, buffers, table, lengths, offsets, first, positions, scale, causal, window, sinks, norm, eps, factor, dtype):
    """(out, lse, received) in float64 and the tolerances of each.  q [rows, q_heads, dim] float64, lam [rows, q_heads / 2].  The maps' own
    tolerances are those of `kv_util.attend`."""
    heads, page, dim = buffers[0].shape[1], buffers[0].shape[2], q.shape[2]
    group, slots, rows = q.shape[1] // heads, table.shape[1] * page, q.shape[0]
    unit_p = torch.finfo(torch.float16).eps / 2
    unit_p = unit_p ** 2 if dtype == "f32" else unit_p
    o, t = (np.zeros((rows, heads // 2, 2, group, 2 * dim)) for _ in range(2))
    lse, tol_lse = np.full((rows, heads, group), -np.inf), np.zeros((rows, heads, group))
    got, tol_got = (np.zeros((len(lengths), heads // 2, slots)) for _ in range(2))
    for b in range(len(lengths)):
        n, mine = min(int(lengths[b]), slots), slice(int(offsets[b]), int(offsets[b + 1]))
        count = mine.stop - mine.start
        if n <= 0 or count == 0:
            continue
        pos_q = (n - count if first is None else int(first[b])) + np.arange(count)
        for j in range(heads // 2):
            held = [U.held(buffers, table, b, 2 * j + w, n) for w in (0, 1)]
            v, there = np.concatenate([x[1] for x in held], -1), held[0][2]
            pos_k = np.arange(n) if positions is None else positions[b, 2 * j, :n].astype(np.int64)
            sees = np.broadcast_to(there, (count, n)).copy()
            if causal:
                sees &= pos_k <= pos_q[:, None]
            if window:
                sees &= (pos_q[:, None] - pos_k < window) | (pos_k < sinks)
            sees, some = sees[:, None], sees.any(-1)[:, None]                       # of every query head alike
            v = np.where(there[:, None], v, 0.0)
            for w in (0, 1):
                k, qs = held[w][0], q[mine, (2 * j + w) * group:(2 * j + w + 1) * group]
                with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
                    s = np.where(sees, scale * (qs.reshape(-1, dim) @ k.T).reshape(count, group, n), -np.inf)
                    top = s.max(-1, keepdims=True)
                    e = np.exp(s - np.where(top == -np.inf, 0.0, top))
                    total = e.sum(-1, keepdims=True)
                    p = np.where(some[..., None], e / total, 0.0)
                    span = np.where(sees, scale * (np.abs(qs).reshape(-1, dim) @ np.abs(k).T).reshape(count, group, n), 0.0).max(-1, keepdims=True)
                    # a score: dim products and sums, then the scaling; a probability: two scores, two roundings of the scaled ones, exp2, the sum
                    off = 2 * (dim + 4) * EPS32 * span + 4 * EPS32 * np.abs(np.where(sees, s, 0.0)).max(-1, keepdims=True) + (8 + np.sqrt(n) + n / 64) * EPS32
                    flat = lambda x, m: (x.reshape(-1, n) @ m).reshape(count, group, -1)  # noqa: E731
                    size, seen_v = flat(p, np.abs(v)), flat(np.broadcast_to(sees, s.shape).astype(float), np.abs(v))
                    o[mine, j, w] = flat(p, v)
                    t[mine, j, w] = np.where(some[..., None], (unit_p + off) * size + 2.0 ** -25 * seen_v / total, 0.0) + 4 * EPS32 * np.abs(o[mine, j, w])
                    lse[mine, 2 * j + w] = np.where(some, (top + np.log(total))[..., 0], -np.inf)
                    tol_lse[mine, 2 * j + w] = off[..., 0] + 4 * EPS32 * np.abs(lse[mine, 2 * j + w])
                    lost = np.isnan(np.where(sees, s, 0.0)).any(-1, keepdims=True)             # (adds nothing)
                    got[b, j, :n] += np.where(lost, 0.0, p).sum((0, 1))
                    tol_got[b, j, :n] += np.where(lost, 0.0, p * off + 2.0 ** -125 * sees).sum((0, 1))
    l = np.asarray(lam, np.float64).reshape(rows, heads // 2, group)[..., None]
    out = (o[:, :, 0] - l * o[:, :, 1]).reshape(rows, -1, 2 * dim)
    tol = (t[:, :, 0] + np.abs(l) * t[:, :, 1] + 3 * EPS32 * (np.abs(o[:, :, 0]) + np.abs(l * o[:, :, 1]))).reshape(rows, -1, 2 * dim)
    if norm is not None:
        root = np.sqrt((out ** 2).mean(-1, keepdims=True) + eps)
        # d(o / root): the coordinate's own error, and the root's, at most that of the error's root mean square
        tol = (tol + np.abs(out) / root * np.sqrt((tol ** 2).mean(-1, keepdims=True))) / root * np.abs(norm) + 16 * EPS32 * np.abs(out / root * norm)
        out = out / root * norm
    out, tol = out * factor, tol * abs(factor)
    tol = 1.02 * tol + (UNIT[dtype] + 2 * EPS32) * np.abs(out) + (2.0 ** -25 if dtype == "f16" else 1e-30)
    pair, tol_pair = got.repeat(2, 1), tol_got.repeat(2, 1)
    return (out, lse.reshape(rows, -1), pair), (tol, tol_lse.reshape(rows, -1), tol_pair + 8 * EPS32 * pair)


def act(name, g):
    return g if name == "none" else 1 / (1 + torch.exp(-g)) if name == "sigmoid" else g / (1 + torch.exp(-g))


def residual_norm(given, activation, residual_scale, block_scale, eps, dh=None, dz=None):
    """(h, z) and the gradients {name: tensor}, in 64 bits on the host.  given: {x, y, gate, after, before}, float64 or None."""
    leaf = {n: None if t is None else t.detach().double().cpu().requires_grad_() for n, t in given.items()}
    rms = lambda t: t / torch.sqrt((t * t).mean(-1, keepdim=True) + eps)  # noqa: E731
    u = 0.0
    if leaf["y"] is not None:
        u = leaf["y"] if leaf["after"] is None else rms(leaf["y"]) * leaf["after"]
        if leaf["gate"] is not None:
            u = u * act(activation, leaf["gate"]).repeat_interleave(u.shape[0] // leaf["gate"].shape[0], 0)
    h = block_scale * u + (0.0 if leaf["x"] is None else residual_scale * leaf["x"])
    z = None if leaf["before"] is None else rms(h) * leaf["before"]
    grads = {}
    if dh is not None or dz is not None:
        loss = 0.0
        if dh is not None:
            loss = loss + (h * dh.double().cpu()).sum()
        if dz is not None:
            loss = loss + (z * dz.double().cpu()).sum()
        names = [n for n, t in leaf.items() if t is not None]
        for n, gr in zip(names, torch.autograd.grad(loss, [leaf[n] for n in names], allow_unused=True)):
            grads[n] = torch.zeros_like(leaf[n]) if gr is None else gr
    return h.detach(), None if z is None else z.detach(), grads


def random_memory(rng, batch, heads, dim, page, tokens, missing=()):
    """Buffers, table and lengths (numpy) with pages in random order; slots of `missing` (sequence, page) have none."""
    used = [max(1, -(-t // page)) for t in tokens]
    width, pages = max(used), sum(used) + 2
    order = rng.permutation(pages).astype(np.int32)
    table = np.full((batch, width), -1, np.int32)
    at = 0
    for b, u in enumerate(used):
        table[b, :u] = order[at:at + u]
        at += u
    for b, p in missing:
        table[b, p] = -1
    return U.random_cache(rng, pages, heads, page, dim), table, np.asarray(tokens, np.int32)


def finite_or_same(got, want, tol):
    """Largest |got - want| / tol; NaN and infinities have to stand in the same places."""
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    assert np.array_equal(np.isnan(got), np.isnan(want)), "NaN in other places"
    inf = np.isinf(want)
    assert np.array_equal(np.isinf(got), inf) and np.array_equal(got[inf], want[inf]), "infinities in other places"
    fine = np.isfinite(want)
    return float(np.max(np.abs(got[fine] - want[fine]) / tol[fine])) if fine.any() else 0.0


assert math.isclose(UNIT["bf16"], 2.0 ** -8)
