"""Rotary positions (`psc_rotary_*`, `psc_kv_append_rotary`; needs an MI355X) against their definition in 64 bits on the host."""
import numpy as np
import pytest
import torch

import kv_util as U
import layer_util as L

pytestmark = pytest.mark.gpu


def _cuda(x):
    return None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda()


def _input(seed, rows, heads, dim, dtype, before=1, behind=2):
    """Heads in the middle of a product's output."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, before + heads + behind, dim), generator=g).to(U.TYPES[dtype]).cuda()
    return x[:, before:before + heads]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rows,heads,dim,dims", [(1, 1, 2, 2), (1, 8, 64, 64), (37, 3, 80, 80), (20, 5, 96, 32), (9, 2, 72, 48), (33, 4, 50, 26),
                                                 (11, 1, 7, 4), (600, 33, 128, 128), (5, 2, 256, 254)])
def test_rows_are_turned(dtype, interleaved, rows, heads, dim, dims):
    import paper_1609_01882_amd as psc
    rng = np.random.default_rng(rows + dim + dims)
    x = _input(rows, rows, heads, dim, dtype)
    positions = rng.integers(-5, 1 << 20, rows).astype(np.int32)
    positions[0] = (1 << 31) - 1
    factor = 1.25 if dims == 48 else 1.0
    rope = psc.Rotary(dims, interleaved=interleaved, factor=factor)
    host = x.double().cpu().numpy()
    for got, back in ((rope(x, _cuda(positions)), False), (rope.inverse(x, _cuda(positions)), True)):
        want = L.turned(host, positions, rope.frequencies, dims, interleaved, factor, back)
        tol = L.turned_tolerance(host, dims, interleaved, factor, dtype)
        assert got.shape == x.shape and got.dtype == x.dtype and got.is_contiguous()
        assert L.finite_or_same(got.double().cpu().numpy(), want, tol) <= 1.0
        assert torch.equal(got[..., dims:], x[..., dims:])


def test_unaligned_rows_are_turned():
    import paper_1609_01882_amd as psc
    whole = torch.randn((10, 3, 131), device="cuda").to(torch.bfloat16)
    x = whole[:, :, 3:]                                       # 6 bytes behind a multiple of 16, rows of 262 bytes
    at = torch.arange(10, dtype=torch.int32, device="cuda") * 1000
    rope = psc.Rotary(128)
    assert torch.equal(rope(x, at), rope(x.contiguous(), at))


def test_in_place_and_into_strides():
    import paper_1609_01882_amd as psc
    for dims in (128, 64, 30):
        rope = psc.Rotary(dims, interleaved=dims == 64)
        qkv = torch.randn((50, 12, 128), device="cuda").half()
        at = torch.arange(50, dtype=torch.int32, device="cuda") * 77
        want = rope(qkv[:, 2:6], at)
        before = qkv.clone()
        assert rope(qkv[:, 2:6], at, out=qkv[:, 2:6]).data_ptr() == qkv[:, 2:6].data_ptr()
        assert torch.equal(qkv[:, 2:6], want) and torch.equal(qkv[:, :2], before[:, :2]) and torch.equal(qkv[:, 6:], before[:, 6:])
        with pytest.raises(psc.PscError):
            rope(before[:20, :4], at[:20], out=before[:20, :4].as_strided((20, 4, 128), (13 * 128, 128, 1)))


def test_rows_of_sequences():
    import paper_1609_01882_amd as psc
    rope = psc.Rotary(64, base=500.0)
    x = torch.randn((23, 2, 64), device="cuda")
    first = torch.tensor([5, 1 << 30, 0, 9], dtype=torch.int32, device="cuda")
    offsets = torch.tensor([2, 2, 10, 11, 19], dtype=torch.int32, device="cuda")      # rows 0, 1 and 19 .. 22 are nobody's
    at = np.zeros(23, np.int64)
    for b, (lo, hi) in enumerate(((2, 2), (2, 10), (10, 11), (11, 19))):
        at[lo:hi] = int(first[b]) + np.arange(hi - lo)
    got = rope(x, first=first, offsets=offsets)
    want = L.turned(x.double().cpu().numpy(), at, rope.frequencies, 64, False)
    want[:2], want[19:] = x[:2].cpu().numpy(), x[19:].cpu().numpy()
    assert L.finite_or_same(got.double().cpu().numpy(), want, L.turned_tolerance(x.double().cpu().numpy(), 64, False, 1.0, "f32")) <= 1.0
    assert torch.equal(got[:2], x[:2]) and torch.equal(got[19:], x[19:])
    # without a first: places; without offsets: equal parts
    even = x[:20]
    assert torch.equal(rope(even, offsets=torch.tensor([0, 20], dtype=torch.int32, device="cuda")), rope(even))
    assert torch.equal(rope(even, first=first), rope(even, (first[:, None] + torch.arange(5, device="cuda")).flatten().int()))
    assert torch.equal(rope(even[:, 0], first=first), rope(even, first=first)[:, 0])
    assert rope(x[:0]).shape == (0, 2, 64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_gradient_is_the_transposed(dtype):
    import paper_1609_01882_amd as psc
    rope = psc.Rotary(48, interleaved=True, factor=0.8)
    x = _input(3, 21, 4, 64, dtype).detach().requires_grad_()
    at = torch.arange(21, dtype=torch.int32, device="cuda") * 31
    dy = torch.randn((21, 4, 64), device="cuda").to(x.dtype)
    y = rope(x, at)
    for grad in (dy, dy.transpose(0, 1).contiguous().transpose(0, 1), dy[:, :1].expand(21, 4, 64), dy.transpose(1, 2).contiguous().transpose(1, 2)):
        dx, = torch.autograd.grad(y, x, grad, retain_graph=True)
        host = grad.double().cpu().numpy()
        want = L.turned(host, at.cpu().numpy(), rope.frequencies, 48, True, 0.8, back=True)
        assert L.finite_or_same(dx.double().cpu().numpy(), want, L.turned_tolerance(host, 48, True, 0.8, dtype)) <= 1.0
    # and by differences: the map is linear, so that one of any size will do
    if dtype == "f32":
        v = torch.randn_like(dy)
        left = ((rope(x.detach() + v, at) - rope(x.detach() - v, at)).double() / 2 * dy.double()).sum()
        dx, = torch.autograd.grad(y, x, dy)
        # 5376 products of two normal numbers with errors of a few steps each
        assert abs(float(left - (dx.double() * v.double()).sum())) < 5376 * 16 * L.EPS32


def test_gradients_as_autograd_hands_them_over():
    import paper_1609_01882_amd as psc
    rope = psc.Rotary(32)
    x = torch.randn((6, 2, 64), device="cuda", requires_grad=True)
    at = torch.arange(6, dtype=torch.int32, device="cuda")
    y = rope(x, at)
    dx, = torch.autograd.grad(y.sum(), x)
    assert torch.equal(dx, rope.inverse(torch.ones((6, 2, 64), device="cuda"), at))
    first, = torch.autograd.grad((rope(x, at) ** 2).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(first.sum(), x)
    y = rope(x, at)
    at += 1
    with pytest.raises(RuntimeError):
        y.sum().backward()
    # on another stream than the tensors' own
    want = rope(x.detach(), at)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        leaf = x.detach().clone().requires_grad_()
        y = rope(leaf, at)
        dx, = torch.autograd.grad(y, leaf, torch.ones_like(y))
    torch.cuda.synchronize()
    assert torch.equal(y, want) and torch.equal(dx, rope.inverse(torch.ones_like(want), at))


def test_frequencies_for_long_contexts():
    import paper_1609_01882_amd as psc
    x = torch.randn((40, 2, 128), device="cuda")
    at = torch.arange(40, dtype=torch.int32, device="cuda") * 25_000
    for more in (dict(stretch=4.0), dict(stretch=8.0, trained=8192), dict(stretch=16.0, trained=4096, low=1.0, high=32.0, blend="pairs")):
        f = psc.rotary_frequencies(128, 10000.0, **more)
        rope = psc.Rotary(128, frequencies=f, factor=1.1)
        want = L.turned(x.double().cpu().numpy(), at.cpu().numpy(), f, 128, False, float(np.float32(1.1)))
        assert L.finite_or_same(rope(x, at).double().cpu().numpy(), want, L.turned_tolerance(x.double().cpu().numpy(), 128, False, 1.1, "f32")) <= 1.0


# ------------------------------------------------------------------------------------------- into the memory
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,dims,heads,group,page", [(64, 64, 1, 3, 16), (64, 16, 3, 1, 32), (128, 128, 2, 4, 64), (128, 96, 4, 0, 16), (256, 192, 1, 2, 128)])
def test_keys_are_turned_on_their_way(dtype, interleaved, dim, dims, heads, group, page):
    import paper_1609_01882_amd as psc
    rng = np.random.default_rng(dim + dims)
    rows, lengths = np.array([1, 0, 33, 70]), np.array([0, 5, 3, page - 1], np.int32)
    batch, width = 4, -(-(page + 70) // page) + 1
    table = rng.permutation(batch * width).reshape(batch, width).astype(np.int32)
    offsets = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    n = int(offsets[-1])
    first = np.array([7, 8, 123_456, 1 << 30], np.int32)
    at = np.concatenate([first[b] + np.arange(rows[b]) for b in range(batch)])
    q_heads = heads * group
    qkv = torch.from_numpy(rng.normal(size=(n, q_heads + 2 * heads, dim))).to(U.TYPES[dtype])
    qkv[5, q_heads, 3] = float("nan")                          # a key and a value that are not finite
    qkv[9, -1, dim - 1] = float("inf")
    rope = psc.Rotary(dims, interleaved=interleaved)
    host = qkv.double().numpy()
    k = L.turned(host[:, q_heads:q_heads + heads], at, rope.frequencies, dims, interleaved).astype(np.float32).astype(np.float64)
    kc, ks, vc, vs = U.round_to_4_bits(k, host[:, q_heads + heads:])
    cache = psc.KvCache.empty(batch * width, heads, dim, page)
    positions = torch.full((batch, heads, width * page), -5, dtype=torch.int32, device="cuda")
    weights = torch.full((batch, heads, width * page), 3.0, device="cuda")
    x = qkv.cuda()
    q = x[:, :q_heads] if group else None
    got = cache.append(x[:, q_heads:q_heads + heads], x[:, q_heads + heads:], _cuda(table), _cuda(lengths), offsets=_cuda(offsets), first=_cuda(first),
                       positions=positions, weights=weights, rotary=rope, q=q)
    if group:
        want = L.turned(host[:, :q_heads], at, rope.frequencies, dims, interleaved)
        assert L.finite_or_same(got.double().cpu().numpy(), want, L.turned_tolerance(host[:, :q_heads], dims, interleaved, 1.0, dtype)) <= 1.0
        assert torch.equal(got, rope(q, _cuda(at.astype(np.int32))))
    else:
        assert got is None
    k_got, v_got = cache.read(_cuda(table), _cuda(lengths), n, offsets=_cuda(offsets))
    assert np.array_equal(k_got.double().cpu().numpy(), U.values(U.pack(kc), ks), equal_nan=True)
    assert np.array_equal(v_got.double().cpu().numpy(), U.values(U.pack(vc), vs))
    pos, w = positions.cpu().numpy(), weights.cpu().numpy()
    for b in range(batch):
        s = slice(lengths[b], lengths[b] + rows[b])
        assert (pos[b, :, s] == first[b] + np.arange(rows[b])).all() and (w[b, :, s] == 0).all()
        pos[b, :, s], w[b, :, s] = -5, 3.0
    assert (pos == -5).all() and (w == 3.0).all()


def test_append_without_a_first_and_rows_of_nobody():
    import paper_1609_01882_amd as psc
    cache = psc.KvCache.empty(4, 2, 64, 16)
    table = torch.tensor([[1, -1], [3, 0]], dtype=torch.int32, device="cuda")
    lengths = torch.tensor([10, 4], dtype=torch.int32, device="cuda")
    offsets = torch.tensor([1, 9, 12], dtype=torch.int32, device="cuda")       # rows 0, 12, 13 are nobody's; slots 16, 17 of 0 have no page
    x = torch.randn((14, 8, 64), device="cuda")
    rope = psc.Rotary(64)
    got = cache.append(x[:, 4:6], x[:, 6:], table, lengths, offsets=offsets, rotary=rope, q=x[:, :4])
    want = x[:, :4].contiguous()
    at = torch.tensor([10 + i for i in range(8)] + [4, 5, 6], dtype=torch.int32, device="cuda")
    want[1:12] = rope(x[1:12, :4], at)
    assert torch.equal(got, want)
    plain = psc.KvCache.empty(4, 2, 64, 16)
    keys = x[:, 4:6].contiguous()
    keys[1:12] = rope(keys[1:12], at)
    plain.append(keys, x[:, 6:], table, lengths, offsets=offsets)
    # (rounded from float32 here and from 64 bits there: scales alike, codes but for those next to a border)
    assert torch.equal(cache.k_scales, plain.k_scales) and torch.equal(cache.v_codes, plain.v_codes)
    assert (cache.k_codes != plain.k_codes).float().mean() < 1e-3


def test_captured_and_on_another_stream():
    import paper_1609_01882_amd as psc
    cache = psc.KvCache.empty(8, 2, 128, 16)
    table = torch.arange(8, dtype=torch.int32, device="cuda").view(2, 4)
    lengths, first = (torch.tensor(t, dtype=torch.int32, device="cuda") for t in ([3, 20], [3, 500]))
    x = torch.randn((2, 12, 128), device="cuda").bfloat16()
    rope = psc.Rotary(128)
    want = cache.append(x[:, 8:10], x[:, 10:], table, lengths, first=first, rotary=rope, q=x[:, :8])
    codes = cache.k_codes.clone()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    out, turned = torch.empty_like(want), torch.empty_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        cache.append(x[:, 8:10], x[:, 10:], table, lengths, first=first, rotary=rope, q=x[:, :8], q_out=out)
    torch.cuda.current_stream().wait_stream(stream)
    assert torch.equal(out, want)
    with torch.cuda.graph(graph):
        cache.append(x[:, 8:10], x[:, 10:], table, lengths, first=first, rotary=rope, q=x[:, :8], q_out=out)
        rope(x[:, :8], first=first, out=turned)
    for step in range(4):
        cache.k_codes.zero_()
        out.zero_()
        turned.zero_()
        first += step
        want = rope(x[:, :8], first=first)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(turned, want)
        assert step > 0 or torch.equal(cache.k_codes, codes)


def test_refusals():
    import paper_1609_01882_amd as psc
    rope = psc.Rotary(64)
    x = torch.zeros((6, 2, 64), device="cuda")
    at = torch.zeros(6, dtype=torch.int32, device="cuda")
    first = torch.zeros(4, dtype=torch.int32, device="cuda")
    for call in (lambda: rope(x.cpu()), lambda: rope(x.double()), lambda: rope(x[..., :32]), lambda: rope(x, at[:5]), lambda: rope(x, at.long()),
                 lambda: rope(x, first=first), lambda: rope(x, at, first=first[:1]), lambda: rope(x.transpose(0, 2)), lambda: rope(x, at, out=x.half()),
                 lambda: rope(x, offsets=at[:0]), lambda: rope(x, first=first[:2], offsets=at[:2]),
                 lambda: rope(x.clone().requires_grad_(), at, out=torch.empty_like(x)), lambda: rope.inverse(x.clone().requires_grad_(), at)):
        with pytest.raises(psc.PscError):
            call()
    cache = psc.KvCache.empty(4, 2, 64, 16)
    table, lengths = torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    ask = x.clone().requires_grad_()
    for call in (lambda: cache.append(x, x, table, lengths, q=x), lambda: cache.append(x, x, table, lengths, rotary=psc.Rotary(24)),
                 lambda: cache.append(x, x, table, lengths, rotary=psc.Rotary(80)), lambda: cache.append(x, x, table, lengths, rotary=rope, q=x[:5]),
                 lambda: cache.append(x, x, table, lengths, rotary=rope, q=x.half()), lambda: cache.append(x, x, table, lengths, rotary=rope, q_out=x),
                 lambda: cache.append(x, x, table, lengths, rotary=rope, q=x, q_out=x), lambda: cache.append(ask, x, table, lengths, rotary=rope),
                 lambda: cache.append(x, x, table, lengths, rotary=rope, q=ask)):
        with pytest.raises(psc.PscError):
            call()
    with torch.no_grad():
        cache.append(x, x, table, lengths, rotary=rope, q=ask)
