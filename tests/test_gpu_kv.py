"""Attention memory in 4 bits (`psc_kv_*`, needs an MI355X) against its definition in 64 bits on the host."""
import numpy as np
import pytest
import torch

import kv_util as U

pytestmark = pytest.mark.gpu


def _table(rng, batch, width, pages):
    return rng.permutation(pages)[:batch * width].reshape(batch, width).astype(np.int32)


def _cuda(x):
    return None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda()


def _cache(psc, buffers):
    return psc.KvCache(*(_cuda(x) for x in buffers))


# ------------------------------------------------------------------------------------------- append, read
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("dim,heads,page", [(64, 3, 16), (128, 2, 64), (256, 1, 256)])
def test_appended_codes_are_the_definitions(dtype, dim, heads, page):
    import paper_1609_01882_amd as psc
    rng = np.random.default_rng(dim + heads)
    lengths, rows = np.array([0, 15, 31, page - 1], np.int32), np.array([1, 0, 33, 70])
    batch, width = len(lengths), -(-(page + 70) // page) + 1
    pages = batch * width + 3
    table = _table(rng, batch, width, pages)
    offsets = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    n = int(offsets[-1])
    x = rng.normal(size=(n, 2, heads, dim)) * 2.0 ** rng.integers(-6, 6, size=(n, 2, heads, dim // 32)).repeat(32, -1)
    x[0, 0, 0, :32] = 0.0                                             # a block of zeros
    edges = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, -0.25])
    x[1, :, 0, :32] = np.concatenate([edges, -edges])                 # ties; the largest is 7/4 of a power of two
    x[2, 0, 0, :32] = np.linspace(-7.03125, 7.03125, 32)              # just over it
    x[3, 0, 0, :32] = np.linspace(-6e4, 6e4, 32)                      # over 6 * 2^13: cut
    x[4, 1, 0, :32] = np.linspace(-1, 1, 32) * 2.0 ** -24             # under the smallest scale's grid
    x[5, 0, 0, 7], x[6, 1, 0, dim - 1], x[7, 1, heads - 1, 3] = np.nan, np.inf, -np.inf
    xt = torch.from_numpy(x).to(U.TYPES[dtype])
    kc, ks, vc, vs = U.round_to_4_bits(*(xt.double().numpy()[:, i] for i in range(2)))
    cache = psc.KvCache.empty(pages, heads, dim, page)
    want = [np.zeros(t.shape, np.uint8) for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)]
    positions = torch.full((batch, heads, width * page), -5, dtype=torch.int32, device="cuda")
    weights = torch.full((batch, heads, width * page), 3.0, device="cuda")
    first = np.array([7, 8, 9, 1000], np.int32)
    xd = xt.cuda()
    cache.append(xd[:, 0], xd[:, 1], _cuda(table), _cuda(lengths), offsets=_cuda(offsets), first=_cuda(first), positions=positions, weights=weights)
    pos_want, w_want = positions.cpu().numpy() * 0 - 5, np.full(weights.shape, 3.0, np.float32)
    for b in range(batch):
        for j in range(rows[b]):
            slot, r = lengths[b] + j, offsets[b] + j
            at = (table[b, slot // page], slice(None), slot % page)
            for buf, y in zip(want, (U.pack(kc), ks, U.pack(vc), vs)):
                buf[at] = y[r]
            pos_want[b, :, slot], w_want[b, :, slot] = first[b] + j, 0.0
    for got, ref, name in zip((cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales), want, ("k", "k scales", "v", "v scales")):
        assert np.array_equal(got.cpu().numpy(), ref), name
    assert np.array_equal(positions.cpu().numpy(), pos_want) and np.array_equal(weights.cpu().numpy(), w_want)
    for out in ("f32", "bf16", "f16"):
        k, v = cache.read(_cuda(table), _cuda(lengths), n, offsets=_cuda(offsets), dtype=U.TYPES[out])
        assert np.array_equal(k.double().cpu().numpy(), U.values(U.pack(kc), ks), equal_nan=True)
        assert np.array_equal(v.double().cpu().numpy(), U.values(U.pack(vc), vs))


def test_append_and_read_leave_out_slots_without_a_page():
    import paper_1609_01882_amd as psc
    cache = psc.KvCache.empty(4, 2, 64, 16)
    table = torch.tensor([[1, -1, 9, 2], [3, -7, 1 << 30, 0]], dtype=torch.int32, device="cuda")
    x = torch.ones((2 * 70, 2, 64), device="cuda")
    starts = torch.zeros(2, dtype=torch.int32, device="cuda")
    cache.append(x, x, table, starts)                      # 70 rows over tables of 64 slots
    assert bool((cache.k_codes != 0).all())                # the four pages are full
    k, v = cache.read(table, starts, 140)
    want = torch.zeros((2, 70), device="cuda")
    want[:, :16] = want[:, 48:64] = 1.0
    assert torch.equal(k, want.view(140, 1, 1).expand_as(k)) and torch.equal(v, k)


# ------------------------------------------------------------------------------------------- attention
def _attend_case(seed, dtype, dim, heads, group, page, lengths, rows, window=0, sinks=0, causal=True, evicted=False, weights=True,
                 first=None, missing=(), scale=None, poison=(), q_scale=2.0, garbage=True):
    """One call against the definition.  Slots behind the lengths hold NaN scales."""
    import paper_1609_01882_amd as psc
    rng = np.random.default_rng(seed)
    lengths, rows = np.array(lengths, np.int32), np.array(rows)
    batch = len(lengths)
    width = max(1, -(-int(lengths.max()) // page))
    pages = batch * width + 2
    table = _table(rng, batch, width, pages)
    buffers = U.random_cache(rng, pages, heads, page, dim)
    if garbage:
        for b in range(batch):
            for s in range(max(0, int(lengths[b])), width * page):
                buffers[1][table[b, s // page], :, s % page] = 255
                buffers[3][table[b, s // page], :, s % page] = 255
    for b, s in poison:  # what append makes of a token that is not finite
        buffers[1][table[b, s // page], :, s % page] = 255
        buffers[2][table[b, s // page], :, s % page] = 0
    for b, p, value in missing:
        table[b, p] = value
    positions = seen = None
    if evicted:
        seen = 3 * np.maximum(lengths, 1)
        positions = np.zeros((batch, heads, width * page), np.int32)
        for b in range(batch):
            for h in range(heads):
                positions[b, h] = rng.permutation(3 * width * page)[:width * page]
        if first is None:
            first = (seen - rows).astype(np.int32)
    offsets = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    n = int(offsets[-1])
    # queries as they lie beside keys and values in one product's output
    qkv = torch.from_numpy(rng.normal(size=(n, heads * group + 2 * heads, dim)) * q_scale).to(U.TYPES[dtype]).cuda()
    q = qkv[:, :heads * group]
    scale = scale or 1.0 / np.sqrt(dim)
    given = rng.random((batch, heads, width * page)).astype(np.float32)
    uniform = len(set(rows)) == 1
    out = torch.full((batch, heads, width * page), np.nan, device="cuda") if weights else None
    cache = _cache(psc, buffers)
    print(f"attend {dtype} d={dim} h={heads}x{group} page={page} n={lengths.tolist()} rows={rows.tolist()}", flush=True)
    got, lse = cache.attend(q, _cuda(table), _cuda(lengths), offsets=None if uniform else _cuda(offsets), max_rows=int(rows.max()),
                            first=_cuda(None if first is None else np.asarray(first, np.int32)), positions=_cuda(positions), scale=scale,
                            causal=causal, window=window, sinks=sinks, weights=_cuda(given) if weights else None, weights_out=out)
    ref, tol = U.attend(q.double().cpu().numpy(), buffers, table, lengths, offsets, first, positions, float(np.float32(scale)), causal,
                        window, sinks, dtype)
    results = [got.double().cpu().numpy(), lse.double().cpu().numpy()]
    refs, tols = list(ref[:2]), list(tol[:2])
    if weights:
        results.append(out.double().cpu().numpy())
        refs.append(ref[2] + given)
        tols.append(tol[2] + 2.0 ** -23 * refs[2])
    for x, y, t, name in zip(results, refs, tols, ("out", "lse", "weights")):
        assert np.array_equal(np.isnan(x), np.isnan(y)), f"{name}: NaN in other places"
        assert np.array_equal(np.isinf(x), np.isinf(y)), name
        ok = np.isfinite(y)
        worst = np.max(np.abs(x[ok] - y[ok]) / t[ok], initial=0.0)
        assert worst <= 1.0, f"{name}: {worst} times the tolerance"
    return results


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("group", [1, 4, 7])
def test_one_token(dtype, dim, group):
    _attend_case(1, dtype, dim, 2, group, 32, [1, 2, 31, 32, 33, 127, 128, 129, 500, 1000, 0], [1] * 11)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("rows", [2, 5, 9, 40, 130])
def test_several_rows(dtype, dim, rows):
    _attend_case(2, dtype, dim, 2, 3, 64, [rows, rows + 1, 200, 333], [rows, rows, rows, rows])


@pytest.mark.parametrize("batch", [64, 65, 150])
@pytest.mark.parametrize("rows", [1, 3])
def test_many_sequences_of_very_different_lengths(batch, rows):
    lengths = np.random.default_rng(batch).integers(0, 60, batch)
    lengths[[3, batch - 1]] = 900, 1300
    lengths[[0, 40]] = 0
    _attend_case(14, "bf16", 64, 1, 2, 16, lengths, [rows] * batch, first=None if rows == 1 else lengths)
    lengths[:] = 0
    lengths[batch // 2] = 700
    _attend_case(15, "f32", 64, 1, 2, 16, lengths, [rows] * batch, weights=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [16, 128, 256])
def test_ragged_rows(dtype, page):
    _attend_case(3, dtype, 128, 2, 2, page, [300, 17, 0, 64, 257], [37, 17, 0, 1, 150])


@pytest.mark.parametrize("dtype,dim,rows", [("bf16", 64, 1), ("f16", 128, 6), ("f32", 128, 70), ("bf16", 128, 300)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (16, 4), (33, 40), (100, 1), (1000, 64)])
def test_window_and_first_tokens(dtype, dim, rows, window, sinks):
    _attend_case(4, dtype, dim, 1, 2, 32, [rows, 310, 420], [rows] * 3)
    _attend_case(4, dtype, dim, 1, 2, 32, [max(rows, 99), 310, 420], [rows] * 3, window=window, sinks=sinks)


@pytest.mark.parametrize("dtype,dim,rows", [("bf16", 128, 1), ("f16", 64, 5), ("f32", 256, 3), ("bf16", 256, 100)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (200, 7)])
def test_slots_in_any_order(dtype, dim, rows, window, sinks):
    _attend_case(5, dtype, dim, 2, 3, 16, [rows, 90, 255], [rows] * 3, window=window, sinks=sinks, evicted=True)


@pytest.mark.parametrize("rows", [1, 20, 200])
def test_rows_that_see_nothing_or_everything(rows):
    # positions before the first token, between, and behind the last
    out, lse, _ = _attend_case(6, "bf16", 128, 2, 2, 32, [100, 100, 100, 0], [rows] * 4, first=[-rows, -rows // 2, 1000, 5])
    assert np.all(out[:rows] == 0) and np.all(lse[:rows] == -np.inf) and np.all(out[3 * rows:] == 0)
    _attend_case(6, "f16", 64, 2, 2, 32, [100, 77], [rows] * 2, causal=False)
    _attend_case(6, "bf16", 64, 2, 2, 32, [100, 77], [rows] * 2, first=[100 + 50, 2000], window=60)      # nothing in the second window
    _attend_case(6, "bf16", 64, 2, 2, 32, [100, 77], [rows] * 2, first=[2 ** 31 - 300, 2 ** 31 - 300], window=2 ** 31 - 1, sinks=3)


@pytest.mark.parametrize("rows", [1, 6, 120])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_tokens_that_are_not_finite_reach_only_the_rows_that_see_them(dtype, rows):
    out, _, w = _attend_case(7, dtype, 128, 2, 2, 32, [130, 130, 140], [rows] * 3, poison=[(0, 128), (1, 3)], window=60, sinks=2)
    assert np.isfinite(out[2 * rows:]).all() and np.isfinite(w).all()
    if rows == 6:
        assert np.isfinite(out[:4]).all() and np.isnan(out[4:6]).all()


@pytest.mark.parametrize("rows", [1, 100])
def test_tables_with_missing_pages(rows):
    _attend_case(8, "bf16", 128, 2, 2, 16, [200, 210, 220], [rows] * 3, missing=[(0, 0, -1), (0, 5, 1 << 20), (1, 13, -9), (2, 2, 44), (2, 3, -1)])


@pytest.mark.parametrize("rows,window", [(1, 0), (9, 0), (9, 700), (100, 300), (60, 0)])
def test_memories_of_a_thousand_tokens_and_more(rows, window):
    """Few sequences: their blocks are shared out over the workgroups."""
    _attend_case(16, "f16", 128, 1, 3, 64, [2300, 1, 1500, 0], [rows] * 4, window=window, sinks=5)
    _attend_case(17, "bf16", 256, 1, 2, 16, [1900, 700], [rows] * 2, window=window, evicted=True)
    _attend_case(18, "f32", 64, 1, 1, 32, [3000, 40], [rows] * 2, window=window, missing=[(0, 7, -1), (0, 50, 1 << 20)])


@pytest.mark.parametrize("blocks", [65, 129, 257, 272, 288, 305, 513, 529, 785, 800, 1025, 1040])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_numbers_of_parts(blocks, dtype):
    """One memory of many blocks of 32 tokens: its parts are joined, four at a time, 64 at a time."""
    _attend_case(19, dtype, 64, 1, 1, 32, [32 * blocks - 5], [1], weights=False, garbage=False)


@pytest.mark.parametrize("q_scale", [1e-3, 60.0])
def test_flat_and_sharp_scores(q_scale):
    for dtype in ("bf16", "f16", "f32"):
        _attend_case(9, dtype, 64, 2, 4, 32, [700, 300], [3, 3], q_scale=q_scale)


def test_lengths_beyond_the_table_and_below_zero():
    import paper_1609_01882_amd as psc
    rng = np.random.default_rng(10)
    buffers = U.random_cache(rng, 6, 2, 32, 64)
    table = np.array([[0, 3], [2, 5]], np.int32)
    q = torch.randn((2, 4, 64), device="cuda")
    cache = _cache(psc, buffers)
    a, la = cache.attend(q, _cuda(table), torch.tensor([64, 0], dtype=torch.int32, device="cuda"))
    b, lb = cache.attend(q, _cuda(table), torch.tensor([1 << 30, -5], dtype=torch.int32, device="cuda"))
    assert torch.equal(a, b) and torch.equal(la, lb) and bool((b[1] == 0).all())


def test_long_memory_behind_32_bit_offsets():
    """Codes of over 4 GiB, the sequence on its last pages; split over many workgroups."""
    import paper_1609_01882_amd as psc
    heads, page, dim, width = 8, 256, 128, 40
    pages = (1 << 32) // (heads * page * dim // 2) + 2 * width
    rng = np.random.default_rng(11)
    small = U.random_cache(rng, width, heads, page, dim)
    cache = psc.KvCache(*(torch.empty((pages, *x.shape[1:]), dtype=torch.uint8, device="cuda") for x in small))
    assert cache.k_codes.numel() > 1 << 32
    table = np.arange(pages - width, pages, dtype=np.int32)[::-1].copy()[None]
    for t, x in zip((cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales), small):
        t[pages - width:] = _cuda(x)
    n = width * page - 3
    q = torch.randn((1, 16, dim), device="cuda").bfloat16()
    lengths = torch.tensor([n], dtype=torch.int32, device="cuda")
    out, lse = cache.attend(q, _cuda(table), lengths)
    ref, tol = U.attend(q.double().cpu().numpy(), small, table - (pages - width), [n], [0, 1], None, None, float(np.float32(dim ** -0.5)),
                        True, 0, 0, "bf16")
    assert np.all(np.abs(out.double().cpu().numpy() - ref[0]) <= tol[0]) and np.all(np.abs(lse.double().cpu().numpy() - ref[1]) <= tol[1])
    x = torch.randn((1, heads, dim), device="cuda")
    cache.append(x, x, _cuda(table), lengths)
    kc, ks, _, _ = U.round_to_4_bits(*(x.double().cpu().numpy(),) * 2)
    at = (pages - width, slice(None), n % page)                       # the table runs backwards: its last page is the first of them
    assert np.array_equal(cache.k_codes[at].cpu().numpy(), U.pack(kc)[0]) and np.array_equal(cache.v_scales[at].cpu().numpy(), ks[0])
    k, v = cache.read(_cuda(table), lengths, 1)
    assert torch.equal(k, v) and np.array_equal(k.double().cpu().numpy(), U.values(U.pack(kc), ks))


def test_weights_in_place_and_without_a_start():
    import paper_1609_01882_amd as psc
    rng = np.random.default_rng(12)
    cache = _cache(psc, U.random_cache(rng, 8, 2, 32, 128))
    table, lengths = _cuda(np.arange(8, dtype=np.int32).reshape(2, 4)), torch.tensor([100, 61], dtype=torch.int32, device="cuda")
    q = torch.randn((6, 8, 128), device="cuda").half()
    alone, inplace = torch.full((2, 2, 128), np.nan, device="cuda"), torch.rand((2, 2, 128), device="cuda")
    start = inplace.clone()
    cache.attend(q, table, lengths, weights_out=alone)
    cache.attend(q, table, lengths, weights=inplace, weights_out=inplace)
    assert torch.equal(inplace, start + alone)
    assert bool((alone[0, :, 100:] == 0).all()) and abs(alone.sum().item() - 6 * 8) < 1e-4
    out, lse = cache.attend(q[:0], table, lengths, weights_out=alone)    # no rows: nothing is received
    assert out.shape == (0, 8, 128) and bool((alone == 0).all())


def test_results_repeat_on_another_stream_and_workspace():
    import paper_1609_01882_amd as psc
    rng = np.random.default_rng(13)
    cache = _cache(psc, U.random_cache(rng, 64, 2, 64, 128))
    table, lengths = _cuda(np.arange(64, dtype=np.int32).reshape(2, 32)), torch.tensor([2000, 1500], dtype=torch.int32, device="cuda")
    q = torch.randn((2, 8, 128), device="cuda").bfloat16()
    want = cache.attend(q, table, lengths)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ws = torch.randint(0, 256, (32 << 20,), dtype=torch.uint8, device="cuda")
        got = cache.attend(q, table, lengths, workspace=ws)
    side.synchronize()
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


def test_arguments_that_do_not_fit_are_refused():
    import paper_1609_01882_amd as psc
    cache = psc.KvCache.empty(4, 2, 64, 16)
    table, lengths = torch.zeros((2, 2), dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    q, w = torch.zeros((2, 4, 64), device="cuda"), torch.zeros((2, 2, 32), device="cuda")
    attend = lambda **kw: cache.attend(**{**dict(q=q, table=table, lengths=lengths), **kw})  # noqa: E731
    attend()
    for bad in (dict(window=1 << 40), dict(window=-1), dict(scale=0.0), dict(q=q.double()), dict(q=q[:, :3]), dict(q=q.cpu()),
                dict(q=torch.zeros((2, 4, 128), device="cuda")[..., ::2]), dict(q=torch.zeros(2 * 4 * 64 + 1, device="cuda")[1:].view(2, 4, 64)),
                dict(table=table.long()), dict(table=table.cpu()), dict(lengths=lengths[:1]), dict(lengths=None), dict(positions=w), dict(weights=w),
                dict(weights_out=w[..., ::2]), dict(offsets=lengths), dict(out=(q, q)), dict(workspace=w), dict(causal=False, window=3)):
        with pytest.raises(psc.PscError):
            attend(**bad)
    with pytest.raises(psc.PscError):
        cache.append(q[:, :2], q[:, :2].half(), table, lengths)
    with pytest.raises(psc.PscError):
        cache.evict(table, lengths, w, 1 << 40)
    with pytest.raises(psc.PscError):
        cache.evict(table, lengths, w, 8, sinks=5, recent=4)
    with pytest.raises(psc.PscError):
        psc.KvCache(cache.k_codes, cache.k_scales, cache.v_codes[:2], cache.v_scales)


# ------------------------------------------------------------------------------------------- eviction
def _evict_case(seed, dim, heads, page, lengths, budget, sinks=0, recent=0, evicted=False, kind="spread", inplace=False, seen=None):
    import paper_1609_01882_amd as psc
    rng = np.random.default_rng(seed)
    lengths = np.array(lengths, np.int32)
    batch, width = len(lengths), max(1, -(-int(lengths.max()) // page))
    if inplace:
        width = max(width, -(-budget // page))
    slots, pages = width * page, batch * width + 1
    table = _table(rng, batch, width, pages)
    buffers = U.random_cache(rng, pages, heads, page, dim)
    w = np.exp(2 * rng.normal(size=(batch, heads, slots))).astype(np.float32)
    if kind == "ties":
        w = rng.integers(0, 3, w.shape).astype(np.float32)
    elif kind == "equal":
        w[:] = 0.25
    elif kind == "odd":
        w = rng.choice(np.array([np.nan, np.inf, -np.inf, -1.0, 0.0, -0.0, 1e-45, 3e38, 1.0], np.float32), w.shape)
    positions = None
    if evicted:
        positions = np.stack([np.stack([rng.permutation(2 * slots)[:slots] for _ in range(heads)]) for _ in range(batch)]).astype(np.int32)
        seen = np.full(batch, 2 * slots, np.int32) if seen is None else np.array(seen, np.int32)
    kept = U.evict(lengths, w, positions, seen, budget, sinks, recent)
    cache = _cache(psc, buffers)
    d_w, d_pos, d_len, d_table = _cuda(w), _cuda(positions), _cuda(lengths), _cuda(table)
    print(f"evict n={lengths.tolist()} budget={budget} {kind}", flush=True)
    out = None
    if inplace:
        out = (torch.empty((batch, heads, budget), dtype=torch.int32, device="cuda"), d_len,
               d_pos if evicted else torch.empty((batch, heads, slots), dtype=torch.int32, device="cuda"), d_w)
    got = cache.evict(d_table, d_len, d_w, budget, sinks=sinks, recent=recent, positions=d_pos, seen=_cuda(seen), out=out)
    g_kept, g_len, g_pos, g_w = (t.cpu().numpy() for t in got)
    assert np.array_equal(g_kept, kept)
    assert np.array_equal(g_len, np.clip(lengths, 0, budget))
    b, h = np.arange(batch)[:, None, None], np.arange(heads)[None, :, None]
    pos = np.broadcast_to(np.arange(slots), (batch, heads, slots)) if positions is None else positions
    assert np.array_equal(g_pos[..., :budget], np.where(kept < 0, -1, pos[b, h, kept]))
    assert np.array_equal(g_w[..., :budget], np.where(kept < 0, np.float32(0), w[b, h, kept]), equal_nan=True)
    want = [x.copy() for x in buffers]
    for bi, hi, to in np.argwhere((kept >= 0) & (kept != np.arange(budget))):
        src = kept[bi, hi, to]
        for x, y in zip(want, buffers):
            x[table[bi, to // page], hi, to % page] = y[table[bi, src // page], hi, src % page]
    for x, t, name in zip(want, (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales), ("k", "k scales", "v", "v scales")):
        assert np.array_equal(x, t.cpu().numpy()), name


@pytest.mark.parametrize("dim,page", [(64, 16), (128, 64), (256, 128)])
@pytest.mark.parametrize("kind", ["spread", "ties", "equal", "odd"])
@pytest.mark.parametrize("budget", [1, 63, 64, 200])
def test_evict(dim, page, kind, budget):
    _evict_case(21, dim, 2, page, [0, 1, 63, 64, 65, 200, 201, 500], budget, kind=kind)
    _evict_case(22, dim, 2, page, [300, 170, 222], budget, sinks=min(4, budget // 2), recent=budget // 2, kind=kind, evicted=True)


@pytest.mark.parametrize("lengths,budget", [([5000, 4096, 1025], 1024), ([33_000, 20_000], 7000), ([40_000], 39_999), ([70_001], 100)])
@pytest.mark.parametrize("kind", ["spread", "ties"])
def test_evict_long(lengths, budget, kind):
    _evict_case(23, 64, 1, 256, lengths, budget, sinks=4, recent=budget // 3, kind=kind)
    _evict_case(24, 64, 1, 256, lengths, budget, sinks=4, recent=budget // 3, kind=kind, evicted=True)


@pytest.mark.parametrize("evicted", [False, True])
def test_evict_in_place(evicted):
    _evict_case(25, 128, 3, 32, [400, 100, 300, 1], 150, sinks=4, recent=20, inplace=True, evicted=evicted)
    _evict_case(26, 128, 3, 32, [100, 50], 150, sinks=150, recent=0, inplace=True, evicted=evicted)      # a budget over all lengths


def test_evict_keeps_the_first_and_the_last_whatever_their_weight():
    _evict_case(27, 64, 2, 16, [300, 64], 50, sinks=20, recent=30, kind="odd")
    _evict_case(28, 64, 2, 16, [300, 64], 50, sinks=0, recent=50, kind="odd")


# ------------------------------------------------------------------------------------------- together
def test_a_recorded_step_replays():
    """append, attend and evict of one step under capture: every replay, with new inputs in the recorded buffers and eager
    calls between, equals the eager step."""
    import paper_1609_01882_amd as psc
    rng = np.random.default_rng(31)
    batch, heads, group, dim, page, width = 3, 2, 4, 128, 32, 4
    start = [_cuda(x) for x in U.random_cache(rng, batch * width, heads, page, dim)]
    table = _cuda(_table(rng, batch, width, batch * width))
    cache = psc.KvCache(*(t.clone() for t in start))
    bufs = (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)
    qkv = torch.zeros((batch, heads * (group + 2), dim), dtype=torch.bfloat16, device="cuda")
    lengths, after = torch.zeros(batch, dtype=torch.int32, device="cuda"), torch.zeros(batch, dtype=torch.int32, device="cuda")
    positions = torch.zeros((batch, heads, width * page), dtype=torch.int32, device="cuda")
    weights = torch.zeros((batch, heads, width * page), device="cuda")
    seen = torch.zeros(batch, dtype=torch.int32, device="cuda")
    ws = torch.empty(8 << 20, dtype=torch.uint8, device="cuda")
    att = (torch.empty((batch, heads * group, dim), dtype=torch.bfloat16, device="cuda"), torch.empty((batch, heads * group), device="cuda"))
    evi = (torch.empty((batch, heads, 60), dtype=torch.int32, device="cuda"), lengths, positions, weights)

    def step():
        q, k, v = qkv[:, :heads * group], qkv[:, heads * group:heads * (group + 1)], qkv[:, heads * (group + 1):]
        cache.append(k, v, table, lengths, first=seen, positions=positions, weights=weights)
        torch.add(lengths, 1, out=after)
        seen.add_(1)
        cache.attend(q, table, after, first=seen - 1, positions=positions, weights=weights, weights_out=weights, out=att, workspace=ws)
        cache.evict(table, after, weights, 60, sinks=4, recent=10, positions=positions, seen=seen, out=evi, workspace=ws)

    def load(seed):
        r = np.random.default_rng(seed)
        for t, s in zip(bufs, start):
            t.copy_(s)
        qkv.copy_(torch.from_numpy(r.normal(size=tuple(qkv.shape))).to(torch.bfloat16))
        lengths.copy_(torch.from_numpy(r.integers(1, 100, batch).astype(np.int32)))
        seen.fill_(200)
        positions.copy_(torch.from_numpy(np.stack([np.stack([r.permutation(200)[:width * page] for _ in range(heads)]) for _ in range(batch)]).astype(np.int32)))
        weights.copy_(torch.from_numpy(r.random(tuple(weights.shape), dtype=np.float32)))

    state = lambda: [t.clone() for t in (*bufs, *att, evi[0], lengths, positions, weights, seen)]  # noqa: E731
    load(0)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    load(0)
    with torch.cuda.graph(graph):
        step()
    for seed in range(1, 6):
        load(seed)
        step()
        want = state()
        load(seed)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(state(), want):
            assert torch.equal(x, y)


def test_the_example_runs(monkeypatch, capsys):
    import json
    import sys

    from paper_1609_01882_amd.benchmarks import decode
    monkeypatch.setattr(sys, "argv", "decode --batch 2 --kv-heads 2 --group 3 --prompt 301 --chunk 100 --budget 120 --recent 30 --slack 8 --tokens 30".split())
    decode.main()
    res = json.loads(capsys.readouterr().out)
    assert 0.0 < res["first_chunk_off_by"] < 0.3 and res["token_ms"] > 0
