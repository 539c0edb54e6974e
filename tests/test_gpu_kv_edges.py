"""Attention memory in 4 bits (`psc_kv_*`, needs an MI355X) where it is easy to get wrong: tails of a softmax, very large
scores, calls without rows, rows and slots that nothing stands behind."""
import numpy as np
import pytest
import torch

import kv_util as U

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24


def _cuda(x):
    return None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda()


def _softmax_case(dtype, scores, v, q, buffers, n, scale, score_error, rows, group, page, weights):
    """attend against the softmax of `scores` [rows * group, n] (float64, what the held keys and q give), values v [n, dim].
    Tolerances: a probability is off by score_error [rows * group, 1] (relative), by its two float16 or one and by half a
    step of 2^-39 of the largest; a sum of n float32 terms by sqrt(n) + n / 64 roundings, exp2 and the rest by 8."""
    import paper_1609_01882_amd as psc
    cache = psc.KvCache(*(_cuda(x) for x in buffers))
    table = torch.arange(buffers[0].shape[0], dtype=torch.int32, device="cuda")[None]
    received = torch.full((1, 1, buffers[0].shape[0] * page), np.nan, device="cuda") if weights else None
    out, lse = cache.attend(q.cuda().view(rows, group, -1), table, torch.tensor([n], dtype=torch.int32, device="cuda"), causal=False,
                            scale=scale, weights_out=received)
    top = scores.max(-1, keepdims=True)
    e = np.exp(scores - top)
    p = e / e.sum(-1, keepdims=True)
    want, size, least = p @ v, p @ np.abs(v), 2.0 ** -40 * np.abs(v).sum(0) / e.sum(-1, keepdims=True)
    unit_p = U.UNIT["f16"] ** 2 if dtype == "f32" else U.UNIT["f16"]
    off = score_error + (8 + np.sqrt(n) + n / 64) * EPS
    tol = U.UNIT[dtype] * np.abs(want) + (unit_p + off) * size + least
    worst = np.max(np.abs(out.double().cpu().numpy().reshape(want.shape) - want) / (1.01 * tol))
    assert worst <= 1.0, f"out: {worst} times the tolerance"
    want = (top + np.log(e.sum(-1, keepdims=True)))[:, 0]
    worst = np.max(np.abs(lse.double().cpu().numpy().reshape(-1) - want) / (off[:, 0] + 16 * EPS * np.abs(want)))
    assert worst <= 1.0, f"lse: {worst} times the tolerance"
    if weights:
        got, want = received.double().cpu().numpy()[0, 0, :n], p.sum(0)
        worst = np.max(np.abs(got - want) / ((p * off).sum(0) + 4 * EPS * want + 2.0 ** -125))
        assert worst <= 1.0, f"weights: {worst} times the tolerance"


# ------------------------------------------------------------------------------------------- very large scores
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("n,rows,group", [(100, 1, 1), (100, 5, 3), (4096, 1, 8), (700, 90, 1)])
def test_scores_beyond_the_integers_of_a_float(dtype, sign, n, rows, group):
    """Scores up to 2^40 (float16: 2^29), whose products with the scale are rounded by more than exp2 can take: the largest
    ones share the row.  Rows with ordinary scores beside them stay as exact as ever."""
    rng = np.random.default_rng(n + rows)
    dim, page, scale = 64, 64, 0.125
    pages = -(-n // page)
    buffers = [np.zeros((pages, 1, page, dim // d), np.uint8) for d in (2, 32, 2, 32)]
    k, ks, v, vs = (b[:, 0].reshape(pages * page, -1) for b in buffers)
    ks[:], vs[:] = 127 + 10, 126
    k[:, 0] = rng.integers(1, 8, pages * page)
    v[:] = rng.integers(0, 256, v.shape)
    sizes = 2.0 ** np.array([-13, 18, 5, 20, 14, 3, 30, 24, 27] if dtype != "f16" else [-13, 13, 5, 15, 14, 3, 12, 11, 10])
    q = torch.zeros((rows * group, dim), dtype=U.TYPES[dtype])
    q[:, 0] = torch.from_numpy(sign * 1.3671875 * np.resize(sizes if rows * group > 1 else sizes[3:], rows * group)).to(q.dtype)
    scores = scale * q[:, :1].double().numpy() * U.values(k, ks)[None, :n, 0]
    size = np.abs(scores).max(-1, keepdims=True)
    # (from 2^10 on two different scores are so far apart that only the largest remains)
    print(f"large {dtype} n={n} rows={rows}x{group} sign={sign}", flush=True)
    _softmax_case(dtype, scores, U.values(v, vs)[:n], q, buffers, n, scale, np.where(size < 1024, 8 * EPS * size, 0.0), rows, group, page, True)


# ------------------------------------------------------------------------------------------- tails
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("gap", [14, 16, 18])
@pytest.mark.parametrize("n,rows,group", [(2000, 1, 1), (4096, 1, 4), (131_072, 1, 2), (2000, 20, 2), (5000, 3, 8)])
@pytest.mark.parametrize("sink_at", [0, -1])
def test_a_long_tail_far_below_one_token(dtype, gap, n, rows, group, sink_at):
    """One token without a value scores `gap` above thousands of others, which are all that comes out: their probabilities,
    some 2^-20 to 2^-26 of the largest, have to be held as well as the largest is."""
    rng = np.random.default_rng(n + gap)
    dim, page = 64, 64
    pages = -(-n // page)
    buffers = [np.zeros((pages, 1, page, dim // d), np.uint8) for d in (2, 32, 2, 32)]
    k, ks, v, vs = (b[:, 0].reshape(pages * page, -1) for b in buffers)
    ks[:, 0], ks[:, 1], vs[:] = 129, 124, 126
    k[:, dim // 4:] = rng.integers(0, 256, (pages * page, dim // 4))
    v[:] = rng.integers(1, 8, v.shape) | rng.integers(1, 8, v.shape) << 4          # all above zero: nothing cancels
    sink = sink_at % n
    k[sink], v[sink] = 0, 0
    k[sink, 0] = 6                                                                 # 4 * 2^2
    q = torch.from_numpy(0.5 * rng.normal(size=(rows * group, dim))).to(U.TYPES[dtype])
    q[:, :dim // 2] = 0.0
    q[:, 0] = gap / 16
    kv, qv = U.values(k, ks)[:n], q.double().numpy()
    scores = qv @ kv.T
    span = (np.abs(qv) @ np.abs(kv).T).max(-1, keepdims=True)
    print(f"tail {dtype} gap={gap} n={n} rows={rows}x{group}", flush=True)
    _softmax_case(dtype, scores, U.values(v, vs)[:n], q, buffers, n, 1.0, 2 * (dim + 4) * EPS * span + 4 * EPS * gap, rows, group, page, True)


# ------------------------------------------------------------------------------------------- no rows
def test_no_rows_of_sequences_that_could_have_some():
    """A step in which no sequence has a row, over a table of many pages: weights go through as they are."""
    import paper_1609_01882_amd as psc
    cache = psc.KvCache.empty(8, 2, 128, 32)
    table = torch.full((3, 4096), -1, dtype=torch.int32, device="cuda")
    lengths = torch.zeros(3, dtype=torch.int32, device="cuda")
    w, out = torch.rand((3, 2, 4096 * 32), device="cuda"), torch.full((3, 2, 4096 * 32), np.nan, device="cuda")
    q, offsets = torch.empty((0, 4, 128), device="cuda").half(), torch.zeros(4, dtype=torch.int32, device="cuda")
    o, lse = cache.attend(q, table, lengths, offsets=offsets, max_rows=4, weights=w, weights_out=out)
    assert o.shape == (0, 4, 128) and lse.shape == (0, 4) and torch.equal(w, out)
    cache.attend(q, table, lengths, offsets=offsets, max_rows=4)


def test_a_workspace_sized_with_another_most_than_the_call_uses():
    """Without offsets `max_rows` is not used by the call, so whatever it was sized with has to be enough."""
    import paper_1609_01882_amd as psc
    rng = np.random.default_rng(3)
    cache = psc.KvCache(*(_cuda(x) for x in U.random_cache(rng, 8, 2, 32, 128)))
    table = torch.full((3, 4096), -1, dtype=torch.int32, device="cuda")
    table[:, :2] = torch.arange(6, dtype=torch.int32, device="cuda").view(3, 2)
    lengths = torch.tensor([64, 50, 30], dtype=torch.int32, device="cuda")
    for rows in (60, 3, 600):
        q = torch.randn((rows, 4, 128), device="cuda").bfloat16()
        want = cache.attend(q, table, lengths)
        for most in (0, 1, rows, 5000):
            size = cache.attend_workspace_bytes(3, 4096, rows, most, 4, q.dtype)
            got = cache.attend(q, table, lengths, workspace=torch.empty(size, dtype=torch.uint8, device="cuda"))
            assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


# ------------------------------------------------------------------------------------------- sizes, rows of no sequence
def test_a_most_that_does_not_fit_is_refused():
    import paper_1609_01882_amd as psc
    cache = psc.KvCache.empty(4, 2, 64, 16)
    table, lengths = torch.zeros((2, 2), dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    q, offsets = torch.zeros((6, 4, 64), device="cuda"), torch.tensor([0, 1, 6], dtype=torch.int32, device="cuda")
    for bad in ((1 << 32) + 5, 1 << 31, -1 << 40):
        with pytest.raises(psc.PscError):
            cache.attend(q, table, lengths, offsets=offsets, max_rows=bad)
    with pytest.raises(psc.PscError):
        cache.attend_workspace_bytes(2, 2, 6, (1 << 32) + 5, 4, q.dtype)
    with pytest.raises(psc.PscError):
        cache.attend_workspace_bytes(2, 2, 6, 5, 4, q.dtype, window=1 << 32)
    with pytest.raises(psc.PscError):
        cache.evict_workspace_bytes(2, 2, (1 << 32) + 5)


@pytest.mark.parametrize("width", [4, 200])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_no_sequence_has_come_out_nan(width, dtype):
    """Rows outside `offsets` and those past `max_rows` are nobody's: NaN, not what the memory held before.  The others are
    what they would be alone, at the places that they have among all rows of their sequence."""
    import paper_1609_01882_amd as psc
    rng = np.random.default_rng(width)
    cache = psc.KvCache(*(_cuda(x) for x in U.random_cache(rng, 2 * width, 2, 32, 128)))
    table = _cuda(rng.permutation(2 * width).reshape(2, width).astype(np.int32))
    lengths = torch.tensor([32 * width - 1, 100], dtype=torch.int32, device="cuda")
    q = torch.randn((50, 6, 128), device="cuda").to(U.TYPES[dtype])
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    for offsets, most, first, there in (((1, 4, 48), 44, None, range(1, 48)), ((0, 20, 50), 25, None, range(45)), ((0, 3, 50), 25, (7, 20), range(28)),
                                        ((0, 0, 50), 49, None, range(49)), ((50, 50, 50), 25, None, range(0)), ((0, 0, 0), 30, (0, 0), range(0))):
        out = torch.full((50, 6, 128), 7.0, device="cuda", dtype=q.dtype), torch.full((50, 6), 7.0, device="cuda")
        cache.attend(q, table, lengths, offsets=ints(*offsets), max_rows=most, first=None if first is None else ints(*first), out=out)
        mine = torch.zeros(50, dtype=torch.bool, device="cuda")
        mine[list(there)] = True
        assert bool(out[0][~mine].isnan().all()) and bool(out[1][~mine].isnan().all()), (offsets, most)
        for b in range(2):
            lo, hi = offsets[b], offsets[b + 1]
            if lo < hi:
                at = ints(int(lengths[b]) - (hi - lo) if first is None else first[b])
                want = cache.attend(q[lo:hi], table[b:b + 1], lengths[b:b + 1], first=at)
                n = min(hi - lo, most)
                # (parts of another number are joined in another order: a rounding or two)
                for x, y in zip((o[lo:lo + n] for o in out), want):
                    assert torch.allclose(x.float(), y[:n].float(), rtol=2.0 ** -7 if dtype == "bf16" else 2.0 ** -15, atol=2.0 ** -8 if dtype == "bf16" else 2.0 ** -16)


def test_rows_that_no_sequence_has_are_not_written():
    import paper_1609_01882_amd as psc
    cache = psc.KvCache.empty(4, 2, 64, 16)
    table, lengths = torch.tensor([[0, 1], [2, 3]], dtype=torch.int32, device="cuda"), torch.tensor([3, 15], dtype=torch.int32, device="cuda")
    offsets = torch.tensor([1, 3, 5], dtype=torch.int32, device="cuda")
    w = torch.full((2, 2, 32), 3.0, device="cuda")
    x = torch.ones((9, 2, 64), device="cuda")
    cache.append(x, x, table, lengths, offsets=offsets, weights=w)
    want = torch.full((2, 32), 3.0, device="cuda")
    want[0, 3:5] = want[1, 15:17] = 0.0
    assert torch.equal(w, want[:, None].expand(2, 2, 32))
    k, _ = cache.read(table, torch.zeros_like(lengths), 64)
    assert torch.equal(k[:, 0, 0], (want == 0).float().flatten())
    k, v = cache.read(table, lengths, 9, offsets=offsets)
    there = torch.tensor([0, 1, 1, 1, 1, 0, 0, 0, 0], dtype=torch.float32, device="cuda")
    assert torch.equal(k, there.view(9, 1, 1).expand_as(k)) and torch.equal(v, k)
    cache.append(x, x, table, torch.tensor([20, 20], dtype=torch.int32, device="cuda"), offsets=offsets)
    k, v = cache.read(table, torch.full_like(lengths, 20), 9, offsets=offsets)      # 20, 21 of both; the rest were never written
    assert torch.equal(k, there.view(9, 1, 1).expand_as(k))
    k, _ = cache.read(table, torch.zeros_like(lengths), 64)
    assert int(k[:, 0, 0].sum()) == 8


# ------------------------------------------------------------------------------------------- gradients
def test_queries_that_want_a_gradient_are_refused():
    """Attention over codes has no backward pass: silence would train on a gradient of nothing."""
    import paper_1609_01882_amd as psc
    cache = psc.KvCache.empty(4, 2, 64, 16)
    table, lengths = torch.zeros((2, 2), dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    q = torch.zeros((2, 4, 64), device="cuda", requires_grad=True)
    with pytest.raises(psc.PscError, match="gradient"):
        cache.attend(q, table, lengths)
    with torch.no_grad():
        cache.attend(q, table, lengths)
    cache.attend(q.detach(), table, lengths)


# ------------------------------------------------------------------------------------------- eviction
def _evict_reference(lengths, weights, positions, seen, budget, sinks, recent, paged):
    """kept as in kv_util.evict, where paged [batch][slots] says which slots have a page."""
    batch, heads = weights.shape[:2]
    kept = np.full((batch, heads, budget), -1, np.int32)
    for b in range(batch):
        n = min(max(int(lengths[b]), 0), weights.shape[2])
        for h in range(heads):
            w, there = weights[b, h, :n].astype(np.float64), paged[b, :n]
            pos = np.arange(n) if positions is None else positions[b, h, :n].astype(np.int64)
            stays = (pos < sinks) | (pos >= (n if seen is None else int(seen[b])) - recent) | (~there & (np.arange(n) < budget))
            stays &= there | (np.arange(n) < budget)

            def order(s):
                if stays[s]:
                    return (0, 0.0, s)
                if not there[s]:
                    return (3, 0.0, s)
                return (2, 0.0, s) if np.isnan(w[s]) else (1, -w[s], s)
            keep = np.zeros(n, bool)
            keep[sorted(range(n), key=order)[:budget]] = True
            source = np.arange(min(n, budget), dtype=np.int32)
            source[~keep[:budget]] = np.flatnonzero(keep[budget:]) + budget
            kept[b, h, :len(source)] = source
    return kept


@pytest.mark.parametrize("page,width,budget", [(16, 20, 100), (16, 200, 700), (64, 8, 200), (256, 3, 300), (16, 1300, 5000), (32, 700, 17_000), (128, 200, 9000)])
@pytest.mark.parametrize("kind", ["spread", "ties", "nan"])
@pytest.mark.parametrize("reordered", [False, True])
def test_slots_without_a_page_neither_keep_a_token_nor_take_one(page, width, budget, kind, reordered):
    import paper_1609_01882_amd as psc
    rng = np.random.default_rng(page + width)
    batch, heads, dim, slots = 3, 2, 64, width * page
    lengths = np.array([slots, slots - page // 2 - 1, min(slots, budget + 5)], np.int32)
    pages = batch * width + 1
    table = rng.permutation(pages)[:batch * width].reshape(batch, width).astype(np.int32)
    lost = rng.random((batch, width)) < 0.2
    lost[0, 0] = lost[1, (budget - 1) // page] = True
    lost[2, : (budget - 1) // page] = False
    table[lost] = rng.choice([-1, pages, 1 << 30, -9], int(lost.sum()))
    paged = np.repeat(~lost, page, 1)
    w = np.exp(rng.normal(size=(batch, heads, slots))).astype(np.float32)
    if kind == "ties":
        w = rng.integers(0, 2, w.shape).astype(np.float32)
    elif kind == "nan":
        w[rng.random(w.shape) < 0.9] = np.nan
    positions = seen = None
    if reordered:
        positions = np.stack([np.stack([rng.permutation(2 * slots)[:slots] for _ in range(heads)]) for _ in range(batch)]).astype(np.int32)
        seen = np.full(batch, 2 * slots, np.int32)
    want = _evict_reference(lengths, w, positions, seen, budget, 4, budget // 3, paged)
    buffers = U.random_cache(rng, pages, heads, page, dim)
    cache = psc.KvCache(*(_cuda(x) for x in buffers))
    print(f"evict without pages: page={page} slots={slots} budget={budget} {kind}", flush=True)
    kept, out_len, pos, out_w = (t.cpu().numpy() for t in cache.evict(_cuda(table), _cuda(lengths), _cuda(w), budget, sinks=4, recent=budget // 3,
                                                                     positions=_cuda(positions), seen=_cuda(seen)))
    assert np.array_equal(kept, want) and np.array_equal(out_len, np.minimum(lengths, budget))
    b, h = np.arange(batch)[:, None, None], np.arange(heads)[None, :, None]
    assert np.array_equal(out_w, np.where(want < 0, np.float32(0), w[b, h, want]), equal_nan=True)
    assert np.array_equal(pos, np.where(want < 0, -1, want if positions is None else positions[b, h, want]))
    ref = [x.copy() for x in buffers]
    for bi, hi, to in np.argwhere((want >= 0) & (want != np.arange(budget))):
        src = want[bi, hi, to]
        assert paged[bi, src] and paged[bi, to]
        for x, y in zip(ref, buffers):
            x[table[bi, to // page], hi, to % page] = y[table[bi, src // page], hi, src % page]
    for x, t in zip(ref, (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)):
        assert np.array_equal(x, t.cpu().numpy())


# ------------------------------------------------------------------------------------------- strides
def test_strides_of_one_row_and_of_one_head_are_never_used():
    """A single row out of a buffer of odd pitch begins where it has to; what leads to a next one does not matter."""
    import paper_1609_01882_amd as psc
    rng = np.random.default_rng(5)
    for dtype in (torch.bfloat16, torch.float32):
        cache = psc.KvCache.empty(2, 1, 64, 16)
        table, lengths = torch.tensor([[0, 1]], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        x = torch.from_numpy(rng.normal(size=(5, 64))).cuda().to(dtype)
        k = x[:1].clone().as_strided((1, 1, 64), (3, 5, 1))
        v = x[1:2].clone().as_strided((1, 1, 64), (67, 1, 1))
        cache.append(k, v, table, lengths)
        rows = torch.zeros((3, 2 * 64), device="cuda", dtype=dtype)
        rows[:, :64] = x[2:]
        lengths += 1
        cache.append(rows.as_strided((3, 1, 64), (128, 7, 1)), rows.as_strided((3, 1, 64), (128, 1, 1)), table, lengths)
        lengths += 3
        other = psc.KvCache.empty(2, 1, 64, 16)
        other.append(torch.cat([x[:1], x[2:]])[:, None], torch.cat([x[1:2], x[2:]])[:, None], table, torch.zeros_like(lengths))
        for a, b in zip((cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales), (other.k_codes, other.k_scales, other.v_codes, other.v_scales)):
            assert torch.equal(a, b)
        want = cache.attend(x[:1, None], table, lengths)
        got = cache.attend(x[:1].clone().as_strided((1, 1, 64), (9, 11, 1)), table, lengths)
        assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


# ------------------------------------------------------------------------------------------- what a call keeps
@pytest.mark.parametrize("rows,group", [(1, 8), (2, 4)])
def test_weights_of_memories_whose_tables_are_very_wide(rows, group):
    """Too many slots to keep every score of: the weights come from the keys once more, and are the same."""
    import paper_1609_01882_amd as psc
    rng = np.random.default_rng(rows)
    batch, heads, page, dim, width = 4, 32, 256, 64, 4352
    cache = psc.KvCache(*(_cuda(x) for x in U.random_cache(rng, 3 * batch, heads, page, dim)))
    table = torch.full((batch, width), -1, dtype=torch.int32, device="cuda")
    table[:, :3] = _cuda(rng.permutation(3 * batch).reshape(batch, 3).astype(np.int32))
    lengths = torch.tensor([700, 3, 512, 768], dtype=torch.int32, device="cuda")
    q = torch.randn((batch * rows, heads * group, dim), device="cuda").bfloat16()
    narrow, wide = torch.empty((batch, heads, 3 * page), device="cuda"), torch.full((batch, heads, width * page), np.nan, device="cuda")
    a = cache.attend(q, table[:, :3].contiguous(), lengths, weights_out=narrow)
    b = cache.attend(q, table, lengths, weights_out=wide)
    assert torch.allclose(a[0].float(), b[0].float(), rtol=2.0 ** -7, atol=2.0 ** -8) and torch.allclose(a[1], b[1], rtol=2.0 ** -18, atol=2.0 ** -18)
    assert torch.allclose(narrow, wide[..., :3 * page], rtol=2.0 ** -17, atol=2.0 ** -60) and bool((wide[..., 3 * page:] == 0).all())


# ------------------------------------------------------------------------------------------- streams
def test_the_current_stream_is_found_without_torchs_private_names(monkeypatch):
    import importlib.util

    from paper_1609_01882_amd import kv
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream")
    spec = importlib.util.spec_from_file_location("paper_1609_01882_amd.kv_of_another_torch", kv.__file__)
    other = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(other)
    rng = np.random.default_rng(8)
    buffers = [_cuda(x) for x in U.random_cache(rng, 4, 2, 64, 128)]
    table, lengths = _cuda(np.arange(4, dtype=np.int32)[None]), torch.tensor([200], dtype=torch.int32, device="cuda")
    q = torch.randn((1, 8, 128), device="cuda").bfloat16()
    want = kv.KvCache(*buffers).attend(q, table, lengths)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        cache = other.KvCache(*buffers)
        assert cache._stream() == side.cuda_stream
        got = cache.attend(q, table, lengths)
    side.synchronize()
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


# ------------------------------------------------------------------------------------------- the example
def test_the_example_has_room_for_the_token_that_is_cut_at_once(monkeypatch, capsys):
    import json
    import sys

    import paper_1609_01882_amd as psc
    from paper_1609_01882_amd.benchmarks import decode
    append = psc.KvCache.append

    def fits(self, k, v, table, lengths, **kw):
        assert int(lengths.max()) + k.shape[0] // table.shape[0] <= table.shape[1] * self.page
        return append(self, k, v, table, lengths, **kw)
    monkeypatch.setattr(psc.KvCache, "append", fits)
    monkeypatch.setattr("paper_1609_01882_amd.benchmarks._common.graph_replay_ms", lambda fn, steps: 0.0)    # (the check above is no work for a graph)
    monkeypatch.setattr(sys, "argv", "decode --batch 1 --kv-heads 1 --group 2 --page 32 --prompt 60 --chunk 50 --budget 64 --recent 30 --slack 0 --tokens 9".split())
    decode.main()
    assert json.loads(capsys.readouterr().out)["token_ms"] > 0
