"""Calls around the attention memory that their documentation allows and where they can go wrong (needs an MI355X)."""
import numpy as np
import pytest
import torch

import kv_util as U
import layer_util as L
import test_gpu_difference as D

pytestmark = pytest.mark.gpu


def _cuda(x):
    return None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda()


# ------------------------------------------------------------------------------------------- differential attention
# (pairs, group, lengths, rows, first): one workgroup to a unit; units cut into parts and joined; waves with rows of their own; those cut into parts.
# Sequences that have no tokens, or whose tokens' pages are all missing (lengths below 0 stand for so many).
WAYS = {
    "whole": (2, 3, [0, 40, -64], [2, 3, 2], None),
    "parts": (1, 2, [5000, -5000, 0, 33], [1, 2, 3, 1], None),
    "rows": (8, 8, [600, 0, -300, 256], [128, 128, 128, 128], [500, 0, 10, 128]),
    "rows_64": (8, 8, [600, 0, -300, 256], [256, 256, 256, 256], [500, 0, 10, 0]),
    "rows_in_parts": (16, 8, [4100, -4100, 128, 0], [9, 20, 16, 11], None),
}


@pytest.mark.parametrize("dtype,dim,way", [("bf16", 64, "whole"), ("f32", 128, "whole"), ("f16", 64, "parts"), ("bf16", 128, "parts"), ("f32", 64, "parts"), ("f16", 128, "rows"),
                                           ("bf16", 64, "rows_64"), ("f16", 64, "rows_in_parts")])
def test_rows_that_see_nothing_are_0_whatever_norms_them(dtype, dim, way):
    import paper_1609_01882_amd as psc
    pairs, group, lengths, rows, first = WAYS[way]
    rng = np.random.default_rng(dim)
    tokens = [abs(n) for n in lengths]
    buffers, table, held = L.random_memory(rng, len(lengths), 2 * pairs, dim, 16, [max(n, 1) for n in tokens])
    held[:] = tokens
    for b, n in enumerate(lengths):
        if n < 0:
            table[b] = -1
    offsets = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    blind = np.concatenate([np.full(r, n <= 0) for n, r in zip(lengths, rows)])
    n, heads = len(blind), 2 * pairs * group
    lam = rng.uniform(0.1, 0.9, (n, heads // 2)).astype(np.float32)
    wild = lam.copy()
    wild[blind, 0], wild[blind, -1] = np.inf, np.nan
    cache = psc.KvCache(*(_cuda(x) for x in buffers))
    q = torch.from_numpy(rng.normal(size=(n, heads, dim))).to(U.TYPES[dtype]).cuda()
    norm = torch.ones(2 * dim, device="cuda")
    print(f"nothing seen: {way} {dtype} {dim}", flush=True)
    call = lambda lam, eps: cache.attend_difference(q, _cuda(lam), _cuda(table), _cuda(held), offsets=_cuda(offsets), max_rows=max(rows),  # noqa: E731
                                                    first=_cuda(None if first is None else np.array(first, np.int32)), norm=norm, eps=eps)
    got, lse = call(wild, 0.0)
    at = _cuda(blind)
    assert bool((got[at] == 0).all()) and bool((lse[at] == -np.inf).all())
    # (2^-126 is lost beside any mean square of the others')
    want, _ = call(lam, 2.0 ** -126)
    assert bool(torch.isfinite(got).all()) and torch.equal(got, want)


@pytest.mark.parametrize("dtype,dim", [("bf16", 64), ("f16", 128), ("f32", 128)])
@pytest.mark.parametrize("batch,rows", [(70, 1), (130, 2)])
def test_parts_of_more_sequences_than_a_wave_has_lanes(dtype, dim, batch, rows):
    # 64 sequences at a time are looked through for a part's own: the long ones stand at both sides of every 64th, some have no tokens or no rows
    rng = np.random.default_rng(batch)
    tokens, counts = rng.integers(1, 60, batch), np.full(batch, rows)
    for b, n in ((3, 1500), (63, 2000), (64, 1200), (69, 3000), (batch - 1, 1700)):
        tokens[b] = n
    tokens[5], tokens[66], counts[7], counts[65], counts[batch - 2] = 0, 0, 0, 0, 0
    D._case(batch, dtype, dim, 1, 2, 16, tokens, counts, nobody=(1, 3))
    D._case(batch + 1, dtype, dim, 2, 3, 32, tokens, counts, evicted=True, lam_rows=True)
    D._case(batch + 2, dtype, dim, 1, 2, 16, tokens, np.full(batch, rows), window=300, sinks=5, weights=False)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("batch,pairs", [(70, 2), (130, 1)])
def test_rows_in_parts_of_more_sequences_than_a_wave_has_lanes(dtype, batch, pairs):
    # the same where waves have rows of their own: 64 rows times query heads to a sequence and more, 16 blocks to a workgroup and more
    rng = np.random.default_rng(batch)
    tokens, counts = rng.integers(20, 60, batch), rng.integers(8, 17, batch)
    for b, n in ((0, 900), (63, 2000), (64, 1200), (69, 4100), (batch - 1, 1700)):
        tokens[b], counts[b] = n, 16
    tokens[5], tokens[66], counts[7], counts[65], counts[batch - 2] = 0, 0, 0, 1, 0
    slots, most = 4112, int(counts.max())
    assert 64 < most * 8 <= 128 and counts.sum() * 8 >= 64 * batch and batch * pairs <= 512 and batch * pairs * (slots // 32) >= 512 * 16
    D._case(batch, dtype, 64, pairs, 8, 16, tokens, counts, nobody=(1, 3))
    D._case(batch + 1, dtype, 64, pairs, 8, 16, tokens, counts, evicted=True, weights=False, lam_rows=True)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("dim,tokens,rows", [(64, 500, 3), (128, 4000, 1), (64, 300, 60)])
def test_maps_that_nearly_cancel(dtype, dim, tokens, rows):
    """Equal keys, queries and lam that differ by little: what is left of the maps is small beside what the rounding of their probabilities
    leaves, and the norm makes it large; the definition's tolerance follows it."""
    import paper_1609_01882_amd as psc
    rng = np.random.default_rng(tokens)
    buffers, table, lengths = L.random_memory(rng, 1, 2, dim, 16, [tokens])
    for buf in buffers[:2]:
        buf[:, 1] = buf[:, 0]
    q = rng.normal(size=(rows, 1, dim)).repeat(2, 1)
    q[:, 1] += rng.normal(size=(rows, dim)) * 0.02
    q = torch.from_numpy(q).to(U.TYPES[dtype]).cuda()
    lam, norm, offsets = np.full((rows, 1), 1.0 - 2.0 ** -6, np.float32), np.ones(2 * dim, np.float32), np.array([0, rows])
    cache, args = psc.KvCache(*(_cuda(x) for x in buffers)), dict(scale=dim ** -0.5, eps=1e-12)
    for weight in (None, norm):
        out, lse = cache.attend_difference(q, _cuda(lam), _cuda(table), _cuda(lengths), norm=_cuda(weight), **args)
        ref, tol = L.difference(q.double().cpu().numpy(), lam, buffers, table, lengths, offsets, None, None, float(np.float32(dim ** -0.5)), True, 0, 0, weight,
                                float(np.float32(1e-12)), 1.0, dtype)
        got = out.double().cpu().numpy()
        worst = L.finite_or_same(got, ref[0], tol[0])
        assert worst <= 1.0, (weight is None, worst)
        if weight is None and dtype != "f32":
            # That is the worst case, and here more than a value.  A probability p is off by at most 2^-11 p and, taken as spread evenly, by 2^-11 p / sqrt(3)
            # in the root mean square; tokens are off independently.  Twice that, and the output's rounding.
            k, v = (np.stack([U.held(buffers, table, 0, w, tokens)[i] for w in (0, 1)]) for i in (0, 1))
            at = np.arange(tokens) <= tokens - rows + np.arange(rows)[:, None]
            p = np.exp(np.einsum("rwd,wtd->wrt", q.double().cpu().numpy(), k) * dim ** -0.5 - ref[1].T[..., None]) * at
            size = (p[0] ** 2 + (lam.astype(np.float64) * p[1]) ** 2) @ np.concatenate((v[0], v[1]), -1) ** 2
            bound = 2 * np.sqrt(size.sum() * 2.0 ** -22 / 3) + U.UNIT[dtype] * np.linalg.norm(ref[0])
            off = np.linalg.norm(got - ref[0])
            print(f"cancel {dtype} {dim} {tokens} {rows}: off by {off / np.linalg.norm(ref[0]):.2g} of the output, {off / bound:.2f} of what is allowed", flush=True)
            assert off <= bound


# ------------------------------------------------------------------------------------------- rotary positions
def _odd_bits(seed, shape, dtype):
    """Numbers among which a third are infinities, NaN (quiet and signalling), zeros of both signs and denormal numbers; as bits, and the type to view them as."""
    kind, odd = {"bf16": (torch.int16, [0x7f80, -0x80, 0x7fc0, 0x7f81, -1, -0x8000, 0, 1, -0x7fff]), "f16": (torch.int16, [0x7c00, -0x400, 0x7e00, 0x7c01, -1, -0x8000, 0, 1, -0x7fff]),
                 "f32": (torch.int32, [0x7f800000, -0x800000, 0x7fc00000, 0x7f800001, -1, -0x80000000, 0, 1, -0x7fffffff])}[dtype]
    g = torch.Generator().manual_seed(seed)
    bits = torch.randn(shape, generator=g).to(U.TYPES[dtype]).view(kind)
    which = torch.tensor(odd, dtype=kind)[torch.randint(len(odd), shape, generator=g)]
    return torch.where(torch.rand(shape, generator=g) < 0.33, which, bits).cuda(), kind


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,dims", [(64, 64), (128, 96), (88, 32), (50, 26)])
def test_what_is_copied_keeps_its_bits(dtype, interleaved, dim, dims):
    import paper_1609_01882_amd as psc
    bits, kind = _odd_bits(dim, (40, 5, dim), dtype)
    x = bits.view(U.TYPES[dtype])
    rope = psc.Rotary(dims, interleaved=interleaved, factor=0.5)
    offsets = torch.tensor([7, 7, 20, 33], dtype=torch.int32, device="cuda")          # rows 0 .. 6 and 33 .. 39 are nobody's
    nobodys = torch.tensor([r < 7 or r >= 33 for r in range(40)], device="cuda")
    into = torch.zeros_like(x)
    for got in (rope(x, offsets=offsets), rope.inverse(x, offsets=offsets), rope(x[:, ::2], offsets=offsets), rope(x, offsets=offsets, out=into), rope(x[..., :dim], offsets=offsets)):
        want = bits[:, ::2] if got.shape[1] == 3 else bits
        assert torch.equal(got.view(kind)[nobodys], want[nobodys])
        assert torch.equal(got.view(kind)[..., dims:], want[..., dims:])
    rope(x, offsets=offsets, out=x)
    assert torch.equal(x.view(kind)[nobodys], into.view(kind)[nobodys]) and torch.equal(x.nan_to_num(7.0), into.nan_to_num(7.0))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,dims", [(64, 64), (128, 96), (256, 16)])
def test_queries_that_an_append_copies_keep_their_bits(dtype, interleaved, dim, dims):
    import paper_1609_01882_amd as psc
    bits, kind = _odd_bits(dims, (40, 6, dim), dtype)
    k = torch.randn((40, 2, dim), device="cuda").to(U.TYPES[dtype])
    cache = psc.KvCache.empty(6, 2, dim, 16)
    table = torch.arange(6, dtype=torch.int32, device="cuda").view(2, 3)
    lengths, offsets = (torch.tensor(t, dtype=torch.int32, device="cuda") for t in ([1, 0], [7, 20, 33]))
    q = bits.view(U.TYPES[dtype])
    got = cache.append(k, k, table, lengths, offsets=offsets, rotary=psc.Rotary(dims, interleaved=interleaved), q=q).view(kind)
    assert torch.equal(got[:7], bits[:7]) and torch.equal(got[33:], bits[33:]) and torch.equal(got[..., dims:], bits[..., dims:])


# ------------------------------------------------------------------------------------------- norms around a block
@pytest.mark.parametrize("block", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("activation", ["sigmoid", "silu"])
@pytest.mark.parametrize("rows,gates", [(6, 6), (1100, 1100), (700, 1), (3000, 1500), (2, 1)])
def test_slopes_of_open_and_shut_gates(rows, gates, activation, block):
    """The gate's gradient where y and the gradient of h are 1: the slope itself, times the rows that share it."""
    import paper_1609_01882_amd as psc
    g = torch.cat([torch.linspace(-80.0, 80.0, 101), torch.tensor([0.0, 1e-3, -1e-3, 8.0, 10.0, 14.0, 17.0, 20.0, 30.0, -8.0, -17.0, -30.0, 1.278, -1.278])]).to(U.TYPES[block])
    gate = g.repeat(gates, 1).cuda().requires_grad_()
    ones = torch.ones((rows, len(g)), dtype=g.dtype, device="cuda")
    h, _ = psc.residual_norm(None, ones, gate=gate, activation=activation)
    dgate, = torch.autograd.grad(h, gate, ones)
    g = g.double()
    s, rest = 1 / (1 + torch.exp(-g)), 1 / (1 + torch.exp(g))
    slope = s * rest
    want, size = (slope, slope) if activation == "sigmoid" else (s + g * slope, s + g.abs() * slope)
    # In units of 2^-24: the power (a step of exp2's result, 2, and what is put back, 1), 1 + it 1, the quotient 2 -- 6, of m and no more of
    # m (1 - m), where 1 - m and the product take 1 each; with a sum and the product with what flows in 10, and 16 are allowed.  Then the output's rounding.
    want, size = want * (rows // gates), size * (rows // gates)
    tol = 16 * L.EPS32 * size + U.UNIT[block] * want.abs() + (2.0 ** -25 if block == "f16" else 2.0 ** -126)
    off = (dgate.double().cpu() - want).abs()
    assert bool((off <= tol).all()), (g[(off > tol).any(0)], (off / tol).max())


@pytest.mark.parametrize("rows,gates,width", [(3, 1, 40), (9, 3, 40), (5, 1, 700), (3000, 3, 64), (2, 1, 2000)])
def test_an_infinity_in_the_last_row_that_shares_a_gate(rows, gates, width):
    # rows that a workgroup has past a gate's last one are that row again, and do not count
    import paper_1609_01882_amd as psc
    y, dh = torch.ones((rows, width), device="cuda"), torch.ones((rows, width), device="cuda")
    each = rows // gates
    y[each - 1::each, 5] = float("inf")
    y[each - 1::each, 7] = -float("inf")
    gate = torch.ones((gates, width), device="cuda", requires_grad=True)
    h, _ = psc.residual_norm(None, y, gate=gate)
    dgate, = torch.autograd.grad(h, gate, dh)
    want = y.view(gates, each, width).sum(1)
    assert torch.equal(dgate, want)


# ------------------------------------------------------------------------------------------- forward-mode derivatives
def test_tangents_are_refused():
    import paper_1609_01882_amd as psc
    from torch.autograd import forward_ad
    rope, w = psc.Rotary(64), torch.ones(64, device="cuda")
    x = torch.randn((4, 2, 64), device="cuda")
    cache = psc.KvCache.empty(4, 2, 64, 16)
    table, lengths = torch.arange(4, dtype=torch.int32, device="cuda").view(4, 1), torch.ones(4, dtype=torch.int32, device="cuda")
    lam, norm = torch.ones(1, device="cuda"), torch.ones(128, device="cuda")
    want = rope(x), psc.residual_norm(x, x, before=w)[1], cache.attend_difference(x, lam, table, lengths)[0]
    with forward_ad.dual_level():
        dual = lambda t: forward_ad.make_dual(t, torch.ones_like(t))  # noqa: E731
        for call in (lambda: rope(dual(x)), lambda: rope.inverse(dual(x)), lambda: psc.residual_norm(dual(x), x, before=w), lambda: psc.residual_norm(x, x, before=dual(w)),
                     lambda: cache.append(dual(x), x, table, lengths, rotary=rope), lambda: cache.append(x, x, table, lengths, rotary=rope, q=dual(x)),
                     lambda: cache.attend(dual(x), table, lengths), lambda: cache.attend_difference(dual(x), lam, table, lengths),
                     lambda: cache.attend_difference(x, dual(lam), table, lengths), lambda: cache.attend_difference(x, lam, table, lengths, norm=dual(norm))):
            with pytest.raises(psc.PscError, match="tangent"):
                call()
        # the others go on as ever
        got = rope(x), psc.residual_norm(x, x, before=w)[1], cache.attend_difference(x, lam, table, lengths)[0]
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert torch.equal(rope(x), want[0])


# ------------------------------------------------------------------------------------------- what is refused
def test_tensors_without_dimensions_are_refused():
    import paper_1609_01882_amd as psc
    rope, w, none = psc.Rotary(64), torch.ones(64, device="cuda"), torch.zeros((), device="cuda")
    x = torch.zeros((4, 2, 64), device="cuda")
    cache = psc.KvCache.empty(4, 2, 64, 16)
    table, lengths = torch.arange(4, dtype=torch.int32, device="cuda").view(4, 1), torch.ones(4, dtype=torch.int32, device="cuda")
    lam = torch.ones(1, device="cuda")
    for call in (lambda: rope(none), lambda: rope(x, first=none.int()), lambda: rope(x, offsets=none.int()), lambda: psc.residual_norm(none, before=w), lambda: psc.residual_norm(x, before=none),
                 lambda: cache.append(none, none, table, lengths), lambda: cache.append(none, none, table, lengths, rotary=rope), lambda: cache.append(x, x, table, lengths, rotary=rope, q=none),
                 lambda: cache.attend(none, table, lengths), lambda: cache.attend(x, none.int(), lengths), lambda: cache.attend_difference(none, lam, table, lengths),
                 lambda: cache.attend_difference(x, none, table, lengths), lambda: cache.attend_difference(x, lam, table, lengths, norm=none)):
        with pytest.raises(psc.PscError):
            call()


def test_numbers_beyond_32_bits_are_refused():
    import paper_1609_01882_amd as psc
    rope, w = psc.Rotary(64), torch.ones(64, device="cuda")
    x, many = torch.zeros((4, 2, 64), device="cuda"), (1 << 32) + 4
    long = torch.zeros((1, 2, 64), device="cuda").expand(many, 2, 64)                    # (as 32 bits: 4)
    cache = psc.KvCache.empty(4, 2, 64, 16)
    table, lengths = torch.arange(4, dtype=torch.int32, device="cuda").view(4, 1), torch.ones(4, dtype=torch.int32, device="cuda")
    lam, offsets = torch.ones(1, device="cuda"), torch.arange(5, dtype=torch.int32, device="cuda")
    out, lse = torch.zeros((1, 2, 64), device="cuda").expand(many, 2, 64), torch.zeros((1, 2), device="cuda").expand(many, 2)
    space = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    for call in (lambda: rope(long, out=out), lambda: rope(long, offsets=offsets, out=out), lambda: rope.inverse(long, out=out),
                 lambda: rope(x[:, :1].expand(4, many, 64), out=x[:, :1].expand(4, many, 64)),
                 lambda: cache.append(long, long, table, lengths, offsets=offsets), lambda: cache.append(long, long, table, lengths, offsets=offsets, rotary=rope),
                 lambda: cache.attend(long, table, lengths, offsets=offsets, max_rows=1, out=(out, lse), workspace=space),
                 lambda: psc.residual_norm(long[:, 0], long[:, 1], before=w), lambda: psc.residual_norm(x, x, before=w, residual_scale=1e39), lambda: psc.residual_norm(x, x, before=w, eps=1e39)):
        with pytest.raises(psc.PscError):
            call()
