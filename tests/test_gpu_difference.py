"""Differential attention over the attention memory (`psc_kv_difference`, needs an MI355X) against its definition in 64 bits on the host."""
import numpy as np
import pytest
import torch

import kv_util as U
import layer_util as L

pytestmark = pytest.mark.gpu


def _cuda(x):
    return None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda()


def _case(seed, dtype, dim, pairs, group, page, lengths, rows, window=0, sinks=0, causal=True, evicted=False, weights=True, first=None, missing=(),
          scale=None, poison=(), q_scale=2.0, norm=True, lam_rows=False, factor=0.4, nobody=(0, 0)):
    """One call against the definition.  Slots behind the lengths hold NaN scales; `nobody` rows stand before and behind the sequences'."""
    import paper_1609_01882_amd as psc
    rng = np.random.default_rng(seed)
    heads, lengths, rows = 2 * pairs, np.array(lengths, np.int32), np.array(rows)
    batch = len(lengths)
    buffers, table, _ = L.random_memory(rng, batch, heads, dim, page, np.maximum(lengths, 1))
    width = table.shape[1]
    for b in range(batch):
        for s in range(max(0, int(lengths[b])), width * page):
            if table[b, s // page] >= 0:
                for buf in (buffers[1], buffers[3]):
                    buf[table[b, s // page], :, s % page] = 255
    for b, s, h in poison:  # what append makes of a token that is not finite
        buffers[1][table[b, s // page], h, s % page] = 255
        buffers[2][table[b, s // page], h, s % page] = 0
    for b, p, value in missing:
        table[b, p] = value
    positions = None
    if evicted:
        positions = np.zeros((batch, heads, width * page), np.int32)
        for b in range(batch):
            for j in range(pairs):
                positions[b, 2 * j] = rng.permutation(3 * width * page)[:width * page]
                positions[b, 2 * j + 1] = -1 if seed % 2 else positions[b, 2 * j]      # (the odd head's are not read)
        if first is None:
            first = (3 * np.maximum(lengths, 1) - rows).astype(np.int32)
    offsets = (nobody[0] + np.concatenate([[0], np.cumsum(rows)])).astype(np.int32)
    n = int(offsets[-1]) + nobody[1]
    qkv = torch.from_numpy(rng.normal(size=(n, heads * group + 2 * heads, dim)) * q_scale).to(U.TYPES[dtype]).cuda()
    q = qkv[:, :heads * group]
    scale = scale or 1.0 / np.sqrt(dim)
    lam = rng.uniform(0.1, 0.9, (n if lam_rows else 1, heads * group // 2)).astype(np.float32)
    lam[:, 0] = -0.3
    weight = (1.0 + 0.2 * rng.normal(size=2 * dim)).astype(np.float32) if norm else None
    given = rng.random((batch, heads, width * page)).astype(np.float32)
    uniform = len(set(rows)) == 1 and nobody == (0, 0)
    received = torch.full((batch, heads, width * page), np.nan, device="cuda") if weights else None
    cache = psc.KvCache(*(_cuda(x) for x in buffers))
    print(f"difference {dtype} d={dim} pairs={pairs}x{group} page={page} n={lengths.tolist()} rows={rows.tolist()}", flush=True)
    wide = _cuda(np.pad(lam, ((0, 0), (0, 3)))) if lam_rows else None
    got, lse = cache.attend_difference(q, wide[:, :-3] if lam_rows else _cuda(lam[0]), _cuda(table), _cuda(lengths), offsets=None if uniform else _cuda(offsets),
                                       max_rows=max(int(rows.max()), -(-n // batch)), first=_cuda(None if first is None else np.asarray(first, np.int32)),
                                       positions=_cuda(positions), scale=scale, causal=causal, window=window, sinks=sinks, norm=_cuda(weight), eps=1e-5,
                                       factor=factor, weights=_cuda(given) if weights else None, weights_out=received)
    ref, tol = L.difference(q.double().cpu().numpy(), np.broadcast_to(lam, (n, lam.shape[1])), buffers, table, lengths, offsets, first, positions,
                            float(np.float32(scale)), causal, window, sinks, weight, 1e-5, float(np.float32(factor)), dtype)
    mine = np.zeros(n, bool)
    mine[offsets[0]:offsets[-1]] = True
    assert bool(torch.isnan(got[_cuda(~mine)]).all()) and bool(torch.isnan(lse[_cuda(~mine)]).all())
    for x, y, t, name in ((got, ref[0], tol[0], "out"), (lse, ref[1], tol[1], "lse")):
        worst = L.finite_or_same(x.double().cpu().numpy()[mine], y[mine], t[mine])
        assert worst <= 1.0, (name, worst)
    if weights:
        worst = L.finite_or_same(received.double().cpu().numpy(), ref[2] + given, tol[2] + 2.0 ** -23 * (ref[2] + given))
        assert worst <= 1.0, ("weights", worst)
    return got, lse, received


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("group", [1, 3, 8])
def test_single_tokens(dtype, dim, group):
    _case(group + dim, dtype, dim, 2, group, 16, [1, 31, 32, 33, 500, 77], [1] * 6)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("dim", [64, 128])
def test_chunks_of_rows(dtype, dim):
    _case(dim, dtype, dim, 1, 2, 32, [200, 333, 64, 5], [40, 7, 64, 5], lam_rows=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim,rows", [(64, 1), (128, 1), (64, 9), (128, 5), (64, 50)])
def test_long_memories_in_parts(dtype, dim, rows):
    _case(rows + dim, dtype, dim, 1, 3, 64, [5000, 1700, 2, 3333], [rows, 1, 1, max(1, rows // 2)])


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("window,sinks", [(1, 0), (40, 4), (700, 33), (5000, 1)])
def test_windows(dim, window, sinks):
    _case(window, "bf16", dim, 2, 2, 32, [900, 65, 2000], [1, 1, 1], window=window, sinks=sinks)
    _case(window + 1, "f16", dim, 1, 2, 16, [900, 65, 300], [33, 20, 1], window=window, sinks=sinks)
    _case(window + 2, "f32", dim, 1, 2, 16, [900, 65, 300], [3, 2, 1], window=window, sinks=sinks, evicted=True)


@pytest.mark.parametrize("dim", [64, 128])
def test_memories_in_another_order(dim):
    _case(2, "bf16", dim, 2, 2, 64, [1500, 40, 700], [1, 1, 1], evicted=True)
    _case(3, "bf16", dim, 1, 4, 16, [700, 40], [20, 3], evicted=True)


@pytest.mark.parametrize("norm", [False, True])
def test_rows_that_see_nothing(norm):
    # sequences without tokens, rows before all tokens, tokens on pages that are not there
    got, lse, _ = _case(1, "bf16", 64, 1, 2, 16, [0, 40, 64], [2, 3, 2], norm=norm, first=[0, -3, 62], missing=[(2, 0, -1), (2, 1, 99), (2, 2, -7), (2, 3, 1 << 30)])
    assert bool((got[:2] == 0).all()) and bool((got[5:] == 0).all()) and bool(torch.isinf(lse[:2]).all())
    _case(2, "f32", 128, 1, 1, 16, [0, 0], [1, 1], norm=norm)


def test_not_causal_and_without_a_norm():
    _case(1, "bf16", 128, 1, 2, 32, [300, 100], [5, 5], causal=False, norm=False, factor=1.0)
    _case(2, "f16", 64, 2, 1, 32, [300, 100], [1, 1], weights=False, norm=False, factor=-2.0)


def test_tokens_that_are_not_finite():
    got, lse, received = _case(4, "bf16", 64, 2, 1, 16, [100, 90, 80], [1, 1, 1], poison=[(0, 50, 1), (2, 79, 0)])
    bad = torch.isnan(got).any(-1)
    assert bad.tolist() == [[True, False], [False, False], [True, False]]
    assert bool(torch.isnan(got[bad]).all()) and not bool(torch.isnan(received).any())


def test_large_scores():
    _case(1, "f32", 64, 1, 2, 16, [300], [4], q_scale=200.0, norm=False, factor=1.0)
    import paper_1609_01882_amd as psc
    # scores far beyond 2^24: what neighbouring floats cannot tell apart shares the row; it stays finite
    rng = np.random.default_rng(0)
    buffers, table, lengths = L.random_memory(rng, 1, 2, 64, 16, [100])
    cache = psc.KvCache(*(_cuda(x) for x in buffers))
    q = torch.randn((1, 2, 64), device="cuda") * 1e9
    out, lse = cache.attend_difference(q, torch.full((1,), 0.5, device="cuda"), _cuda(table), _cuda(lengths))
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())


def test_rows_of_nobody_come_out_nan():
    _case(1, "bf16", 64, 1, 2, 16, [60, 70], [3, 2], nobody=(2, 4))
    _case(2, "bf16", 128, 1, 2, 16, [5000, 70], [3, 2], nobody=(1, 3))


# Calls with so many rows that every wave of the card has some of its own: 512 workgroups' worth of 64 rows (128 with 64 coordinates).
def _many(rng, batch, rows):
    """Lengths and rows of sequences: few tokens before the rows or many, ends inside blocks and pages; one without rows, one without tokens, some
    of a single row."""
    rows = [rows + int(r) for r in rng.integers(0, 30, batch)]
    rows[3], rows[7], rows[11] = 1, 0, 2
    lengths = [r + int(t) for r, t in zip(rows, rng.choice([0, 1, 13, 31, 32, 100], batch))]
    lengths[9] = 0
    return lengths, rows


def _fills_the_card(dim, pairs, group, rows):
    assert sum(rows) * group * pairs >= 512 * (64 if dim == 128 else 128)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim,rows,group", [(128, 40, 3), (64, 60, 4)])
def test_rows_of_their_own(dtype, dim, rows, group):
    lengths, rows = _many(np.random.default_rng(dim), 32, rows)
    _fills_the_card(dim, 8, group, rows)
    _case(dim, dtype, dim, 8, group, 16, lengths, rows, lam_rows=True, poison=[(2, lengths[2] - 5, 1)], missing=[(4, 0, -1), (5, 1, 1 << 20)], nobody=(2, 5))


@pytest.mark.parametrize("dim,rows,group", [(128, 40, 3), (64, 60, 4)])
def test_rows_of_their_own_with_windows_and_in_another_order(dim, rows, group):
    lengths, rows = _many(np.random.default_rng(dim + 1), 32, rows)
    _fills_the_card(dim, 8, group, rows)
    _case(1, "bf16", dim, 8, group, 32, lengths, rows, window=20, sinks=3, weights=False)
    _case(2, "f16", dim, 8, group, 16, lengths, rows, evicted=True, window=150, sinks=5, norm=False)
    _case(3, "bf16", dim, 8, group, 16, lengths, rows, causal=False, weights=False)


@pytest.mark.parametrize("dim", [64, 128])
def test_as_many_rows_to_every_sequence(dim):
    # (without offsets; memories of several places of 32 blocks, first positions behind the tokens: a window leaves some rows nothing)
    rows = [256 if dim == 64 else 128] * 4
    _fills_the_card(dim, 8, 8, rows)
    _case(5, "bf16", dim, 8, 8, 64, [2200, 1300, 600, 256], rows, first=[2100, 1172, 900, 0], window=500)


def test_rows_of_their_own_with_large_scores():
    import paper_1609_01882_amd as psc
    rng = np.random.default_rng(0)
    buffers, table, lengths = L.random_memory(rng, 64, 16, 64, 16, [200] * 64)
    cache = psc.KvCache(*(_cuda(x) for x in buffers))
    q = torch.randn((64 * 140, 16, 64), device="cuda").half()
    q[5 * 140 + 3] *= 6e4 / q[5 * 140 + 3].abs().max()
    lam = torch.full((8,), 0.5, device="cuda")
    # a scale that lifts the scores of one row of sequence 5 over 2^24, and leaves those of the others below it
    out, lse = cache.attend_difference(q, lam, _cuda(table), _cuda(lengths), scale=64.0)
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())
    few, few_lse = cache.attend_difference(q[5 * 140:6 * 140].contiguous(), lam, _cuda(table[5:6]), _cuda(lengths[5:6]), scale=64.0)
    # Scores are the same products in both kernels, and so is what a row refers to in the end; probabilities are rounded to float16 against
    # the largest seen so far, which differs: 2^-11 of each in either kernel.  Held values are 3 at most (6 times 2^-1), the maps weigh 1
    # and 0.5: 2 * 1.5 * 3 * 2^-11, and two outputs of up to 4.5 rounded to float16: 2 * 4.5 * 2^-11.  The row beyond 2^24 has
    # scores that 32 bits hardly tell apart: its output is within the held values.
    mine, others = out[5 * 140:6 * 140], torch.arange(140, device="cuda") != 3
    assert float((few_lse - lse[5 * 140:6 * 140]).abs()[others].max()) <= 2.0 ** -9      # (scores of up to 2^14: a step of 2^-10 in either)
    assert float((few[others].float() - mine[others].float()).abs().max()) <= 18 * 2.0 ** -11
    assert float(mine[3].abs().max()) <= 4.5 and float(few[3].abs().max()) <= 4.5


def test_a_prompt_beside_single_tokens():
    # 8 pairs: the prompt fills the card, the others have a row or two over long memories
    _case(4, "bf16", 64, 8, 8, 64, [1030, 3000, 1, 2500, 40], [1030, 1, 1, 2, 3], weights=False)


def test_against_two_attentions():
    """The same maps through `attend` of each key head over each value head."""
    import paper_1609_01882_amd as psc
    rng = np.random.default_rng(5)
    buffers, table, lengths = L.random_memory(rng, 3, 4, 128, 64, [3000, 500, 64])
    k, ks, v, vs = (_cuda(x) for x in buffers)
    q = torch.randn((3, 8, 128), device="cuda")
    lam = torch.rand(4, device="cuda")
    out, lse = psc.KvCache(k, ks, v, vs).attend_difference(q, lam, _cuda(table), _cuda(lengths))
    maps = []
    for value in (0, 1):
        rep = [t[:, value::2].repeat_interleave(2, 1).contiguous() for t in (v, vs)]
        o, l = psc.KvCache(k, ks, *rep).attend(q, _cuda(table), _cuda(lengths))
        assert torch.allclose(l, lse, rtol=0, atol=2e-5)      # (scores of up to 40 with 128 products each)
        maps.append(o.view(3, 2, 2, 2, 128))
    want = torch.cat([m[:, :, 0] for m in maps], -1) - lam.view(2, 2, 1) * torch.cat([m[:, :, 1] for m in maps], -1)
    assert torch.allclose(out, want.view(3, 4, 256), rtol=0, atol=1e-4)


def test_both_heads_receive_the_same_and_are_cut_alike():
    import paper_1609_01882_amd as psc
    rng = np.random.default_rng(6)
    buffers, table, lengths = L.random_memory(rng, 2, 4, 64, 16, [200, 150])
    cache = psc.KvCache(*(_cuda(x) for x in buffers))
    q, lam = torch.randn((2, 4, 64), device="cuda"), torch.rand(2, device="cuda")
    w = torch.zeros((2, 4, table.shape[1] * 16), device="cuda")
    cache.attend_difference(q, lam, _cuda(table), _cuda(lengths), weights=w, weights_out=w)
    assert torch.equal(w[:, 0::2], w[:, 1::2]) and torch.allclose(w.sum(-1), torch.full((2, 4), 2.0, device="cuda"), atol=1e-4)
    kept, after, pos, left = cache.evict(_cuda(table), _cuda(lengths), w, budget=100, sinks=2, recent=8)
    assert torch.equal(kept[:, 0::2], kept[:, 1::2]) and torch.equal(pos[:, 0::2], pos[:, 1::2])
    out, _ = cache.attend_difference(q, lam, _cuda(table)[:, :7].contiguous(), after, first=_cuda(lengths) - 1,
                                     positions=torch.nn.functional.pad(pos, (0, 12), value=1 << 30))
    assert bool(torch.isfinite(out).all())


def test_calls_without_rows_pass_the_weights_on():
    import paper_1609_01882_amd as psc
    rng = np.random.default_rng(8)
    buffers, table, lengths = L.random_memory(rng, 2, 4, 64, 16, [200, 150])
    cache = psc.KvCache(*(_cuda(x) for x in buffers))
    w = torch.rand((2, 4, table.shape[1] * 16), device="cuda")
    out = torch.full_like(w, -1.0)
    q, lam = torch.zeros((0, 4, 64), device="cuda"), torch.zeros(2, device="cuda")
    cache.attend_difference(q, lam, _cuda(table), _cuda(lengths), weights=w, weights_out=out)
    assert torch.equal(out, w)
    cache.attend_difference(q, lam, _cuda(table), _cuda(lengths), weights_out=out)
    assert bool((out == 0).all())


def test_two_calls_at_once():
    import paper_1609_01882_amd as psc
    rng = np.random.default_rng(9)
    buffers, table, lengths = L.random_memory(rng, 2, 2, 64, 16, [6000, 3000])
    cache = psc.KvCache(*(_cuda(x) for x in buffers))
    table, lengths = _cuda(table), _cuda(lengths)
    qs, lam = [torch.randn((2, 4, 64), device="cuda").half() for _ in range(2)], torch.rand(2, device="cuda")
    want = [cache.attend_difference(q, lam, table, lengths) for q in qs]
    streams = [torch.cuda.Stream() for _ in qs]
    got = []
    for q, stream in zip(qs, streams):
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            got.append([cache.attend_difference(q, lam, table, lengths) for _ in range(5)])
    torch.cuda.synchronize()
    for w, many in zip(want, got):
        assert all(torch.equal(w[0], o) and torch.equal(w[1], l) for o, l in many)


def test_captured_graphs_repeat():
    import paper_1609_01882_amd as psc
    rng = np.random.default_rng(7)
    buffers, table, lengths = L.random_memory(rng, 2, 2, 128, 32, [4000, 900])
    cache = psc.KvCache(*(_cuda(x) for x in buffers))
    table, lengths = _cuda(table), _cuda(lengths)
    q, lam = torch.randn((2, 4, 128), device="cuda").bfloat16(), torch.rand(2, device="cuda")
    w = torch.rand((2, 2, table.shape[1] * 32), device="cuda")
    norm = torch.rand(256, device="cuda")
    call = lambda **more: cache.attend_difference(q, lam, table, lengths, norm=norm, weights=w, **more)  # noqa: E731
    bytes_ = cache.attend_difference_workspace_bytes(2, table.shape[1], 2, 1, 4, q.dtype, weights=True)
    # two graphs with a workspace of their own each, replayed in turn
    graphs = []
    for _ in range(2):
        ws, got = torch.empty(bytes_, dtype=torch.uint8, device="cuda"), torch.empty_like(w)
        out = (torch.empty((2, 2, 256), dtype=q.dtype, device="cuda"), torch.empty((2, 4), device="cuda"))
        call(weights_out=got, out=out, workspace=ws)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(weights_out=got, out=out, workspace=ws)
        graphs.append((graph, out, got, ws))
    for turn in range(4):
        q.mul_(1.25)
        lengths.sub_(turn)
        seen = torch.empty_like(w)
        want = call(weights_out=seen)
        for graph, out, got, ws in graphs:
            out[0].zero_()
            ws.fill_(255)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1]) and torch.equal(got, seen)


def test_refusals():
    import paper_1609_01882_amd as psc
    cache = psc.KvCache.empty(4, 2, 64, 16)
    table, lengths = torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    q, lam, norm = torch.zeros((1, 4, 64), device="cuda"), torch.zeros(2, device="cuda"), torch.ones(128, device="cuda")
    ok = cache.attend_difference(q, lam, table, lengths, norm=norm)
    assert ok[0].shape == (1, 2, 128) and ok[1].shape == (1, 4)
    odd, wide = psc.KvCache.empty(4, 3, 64, 16), psc.KvCache.empty(4, 2, 256, 16)
    for call in (lambda: odd.attend_difference(q[:, :3], lam, table, lengths), lambda: wide.attend_difference(q.new_zeros(1, 4, 256), lam, table, lengths),
                 lambda: cache.attend_difference(q[:, :3], lam, table, lengths), lambda: cache.attend_difference(q, lam[:1], table, lengths),
                 lambda: cache.attend_difference(q, lam.half(), table, lengths), lambda: cache.attend_difference(q, lam.expand(2, 2), table, lengths),
                 lambda: cache.attend_difference(q, lam, table, lengths, norm=norm[:64]), lambda: cache.attend_difference(q, lam, table, lengths, norm=norm, eps=-1.0),
                 lambda: cache.attend_difference(q, lam, table, lengths, factor=float("inf")), lambda: cache.attend_difference(q.clone().requires_grad_(), lam, table, lengths),
                 lambda: cache.attend_difference(q, lam.clone().requires_grad_(), table, lengths), lambda: cache.attend_difference(q, lam, table, lengths, window=4, causal=False),
                 lambda: cache.attend_difference(q, lam, table, lengths, weights=torch.zeros((1, 2, 16), device="cuda")),
                 lambda: cache.attend_difference(q, lam, table, lengths, out=(q, ok[1]))):
        with pytest.raises(psc.PscError):
            call()
    empty = cache.attend_difference(q[:0], lam, table, lengths)
    assert empty[0].shape == (0, 2, 128)


def test_a_layer_step():
    """Norm, queries and keys turned into the memory, differential attention, norm: as a layer runs them."""
    import paper_1609_01882_amd as psc
    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    batch, heads, group, dim, width = 2, 2, 2, 64, 128
    rand = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    cache = psc.KvCache.empty(8, heads, dim, 16)
    table = torch.arange(8, dtype=torch.int32, device="cuda").view(2, 4)
    lengths = torch.zeros(batch, dtype=torch.int32, device="cuda")
    rope = psc.Rotary(dim)
    w_in, w_out = rand(width, (heads * group + 2 * heads) * dim) / width ** 0.5, rand(heads * group * dim, width) / 16
    weight, norm, lam = torch.ones(width, device="cuda"), torch.ones(2 * dim, device="cuda"), torch.full((heads * group // 2,), 0.3, device="cuda")
    keys, values = [], []
    for step in range(40):
        x = rand(batch, width)
        x, z = psc.residual_norm(x, before=weight)
        qkv = (z @ w_in).view(batch, heads * group + 2 * heads, dim)
        q, k, v = qkv.split([heads * group, heads, heads], 1)
        turned = cache.append(k, v, table, lengths, rotary=rope, q=q)
        held = cache.read(table, lengths, batch)
        keys.append(held[0])
        values.append(held[1])
        lengths += 1
        o, _ = cache.attend_difference(turned, lam, table, lengths, norm=norm, factor=0.7)
        y = o.flatten(1) @ w_out
        h, z = psc.residual_norm(x, y, after=weight, before=weight)
        k_all, v_all = torch.stack(keys, 2).double(), torch.stack(values, 2).double()            # [batch, heads, tokens, dim]
        s = (k_all.repeat_interleave(group, 1) @ turned.double()[..., None])[..., 0] / dim ** 0.5
        p = torch.softmax(s, -1).view(batch, heads // 2, 2, group, -1)
        both = torch.cat((v_all[:, 0::2], v_all[:, 1::2]), -1)[:, :, None]
        d = (p[:, :, 0] - 0.3 * p[:, :, 1])[..., None, :] @ both
        d = d[..., 0, :]
        d = 0.7 * d / torch.sqrt(d.square().mean(-1, keepdim=True) + 1e-6)
        assert torch.allclose(o.double(), d.reshape(batch, -1, 2 * dim), rtol=1e-4, atol=1e-4)
        want = x.double() + (lambda t: t / torch.sqrt(t.square().mean(-1, keepdim=True) + 1e-6))(y.double())
        assert torch.allclose(h.double(), want, rtol=1e-5, atol=1e-5)


@pytest.mark.parametrize("dtype,dim,group", [("bf16", 64, 8), ("f16", 128, 4), ("f32", 64, 5), ("f32", 128, 3)])
@pytest.mark.parametrize("evicted", [False, True])
def test_weights_of_many_rows(dtype, dim, group, evicted):
    # few tokens and many rows: the rows are cut into parts that are added up in order
    _case(dim, dtype, dim, 1, group, 16, [900, 130, 350], [130, 1, 90], evicted=evicted)
    _case(dim + 1, dtype, dim, 2, group, 32, [400, 0, 33], [77, 2, 33], window=50, sinks=5, evicted=evicted, nobody=(1, 3))
    _case(dim + 2, dtype, dim, 1, group, 64, [300, 500], [100, 100], causal=False, evicted=evicted, first=[200, 399])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_rows_of_workgroups_over_parts_of_the_tokens(dtype):
    # 64 coordinates, workgroups of 128 rows times query heads, cut into parts of the tokens: batches whose longest memory has many blocks
    short = [130, 9, 700, 33, 64, 1000, 31, 250]
    few = dict(weights=False, norm=False, factor=1.0)
    _case(1, dtype, 64, 8, 8, 32, [4200] + short, [9] * 9, weights=False)
    _case(2, dtype, 64, 8, 8, 32, [4200] + short, [9, 40, 1, 2, 33, 17, 16, 0, 31], nobody=(2, 3))
    _case(3, dtype, 64, 16, 8, 64, [300, 4100, 200, 10], [10, 9, 16, 9], evicted=True, lam_rows=True)
    _case(4, dtype, 64, 16, 5, 16, [5200, 1900, 20], [50, 70, 14], window=4000, sinks=40)
    _case(5, dtype, 64, 16, 5, 16, [5200, 1900, 20], [50, 70, 14], window=4000, sinks=40, evicted=True)
    _case(6, dtype, 64, 16, 8, 16, [4100, 64, 128, 99], [9, 20, 16, 11], missing=[(0, 7, -1), (0, 20, 1 << 30), (3, 0, -5)], first=[900, 44, 112, -3], **few)
    _case(7, dtype, 64, 16, 8, 16, [0, 4100, 200, 77], [9, 9, 20, 12], causal=False, weights=False)
    _case(8, dtype, 64, 16, 8, 16, [4100, 64, 128, 99], [9, 20, 16, 11], q_scale=200.0, **few)
    got, _, _ = _case(10, dtype, 64, 16, 8, 16, [4100, 64, 128, 99], [9, 20, 16, 11], poison=[(0, 4095, 4), (2, 0, 1)], weights=False)
    assert torch.isnan(got).any(-1).any(-1).tolist() == [4 <= p < 9 or 29 <= p < 45 for p in range(56)]


def test_rows_of_workgroups_over_parts_with_large_scores():
    import paper_1609_01882_amd as psc
    rng = np.random.default_rng(0)
    buffers, table, lengths = L.random_memory(rng, 1, 32, 64, 16, [4100])
    cache = psc.KvCache(*(_cuda(x) for x in buffers))
    q = torch.randn((80, 256, 64), device="cuda").half()
    q[3] *= 6e4 / q[3].abs().max()
    lam = torch.full((128,), 0.5, device="cuda")
    call = lambda q: cache.attend_difference(q, lam, _cuda(table), _cuda(lengths), first=_cuda(np.array([4020], np.int32)), scale=64.0)  # noqa: E731
    out, lse = call(q)
    few, few_lse = call(q[:8].contiguous())      # (64 rows times query heads: waves share out the tokens)
    # tolerances: as in test_rows_of_their_own_with_large_scores, and 2^-24 for each of up to 64 scaled sums of parts, which 2^-11 dwarfs
    others = torch.arange(8, device="cuda") != 3
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())
    assert float((few_lse - lse[:8]).abs()[others].max()) <= 2.0 ** -9
    assert float((few.float() - out[:8].float())[others].abs().max()) <= 18 * 2.0 ** -11
    assert float(out[3].abs().max()) <= 4.5 and float(few[3].abs().max()) <= 4.5
    again, again_lse = call(q)
    assert torch.equal(again, out) and torch.equal(again_lse, lse)


def test_captured_chunks_repeat():
    # rows' workgroups over parts of the tokens, the weights' parts: a graph replayed between eager calls that have other rows
    import paper_1609_01882_amd as psc
    rng = np.random.default_rng(12)
    buffers, table, lengths = L.random_memory(rng, 1, 32, 64, 16, [4100])
    cache = psc.KvCache(*(_cuda(x) for x in buffers))
    table, lengths = _cuda(table), _cuda(lengths)
    q, lam = torch.randn((80, 256, 64), device="cuda").bfloat16(), torch.rand(128, device="cuda")
    w = torch.rand((1, 32, table.shape[1] * 16), device="cuda")
    call = lambda **more: cache.attend_difference(q, lam, table, lengths, weights=w, **more)  # noqa: E731
    ws = torch.empty(cache.attend_difference_workspace_bytes(1, table.shape[1], 80, 80, 256, q.dtype, weights=True), dtype=torch.uint8, device="cuda")
    got, out = torch.empty_like(w), (torch.empty((80, 128, 128), dtype=q.dtype, device="cuda"), torch.empty((80, 256), device="cuda"))
    call(weights_out=got, out=out, workspace=ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(weights_out=got, out=out, workspace=ws)
    for turn in range(4):
        q.mul_(1.25)
        lengths.sub_(100 * turn)
        seen = torch.empty_like(w)
        want = call(weights_out=seen)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1]) and torch.equal(got, seen), turn
    with pytest.raises(psc.PscError, match="workspace too small"):
        call(weights_out=got, out=out, workspace=ws[:-16])
