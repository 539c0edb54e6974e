"""Norms around a block (`psc_residual_norm_*`, needs an MI355X) against their definition in 64 bits on the host."""
import numpy as np
import pytest
import torch

import layer_util as L

pytestmark = pytest.mark.gpu
NAMES = ("x", "y", "gate", "after", "before")


def _given(seed, rows, width, stream, block, weights, gates, has):
    g = torch.Generator().manual_seed(seed)
    t = {"x": 3.0 * torch.randn((rows, width), generator=g), "y": torch.randn((rows, width), generator=g),
         "gate": 2.0 * torch.randn((max(gates, 1), width), generator=g), "after": 1.0 + 0.3 * torch.randn(width, generator=g),
         "before": 1.0 + 0.3 * torch.randn(width, generator=g)}
    types = {"x": stream, "y": block, "gate": block, "after": weights, "before": weights}
    return {n: t[n].to(L.TYPES[types[n]]).cuda() if n in has else None for n in NAMES}


def _tolerances(given, activation, a, b, eps, dh, dz, types):
    """What float32 arithmetic may be off by, from the sizes of what is added.  Sums of squares of up to 16384 positive terms,
    16 in a row to a lane, then halves: 40 roundings at most; 64 of them cover roots, products and the gate's exponential too."""
    c = 64 * L.EPS32
    t = {n: None if v is None else v.double().cpu() for n, v in given.items()}
    rms = lambda v: torch.sqrt((v * v).mean(-1, keepdim=True) + eps)  # noqa: E731
    share = 0.0
    if t["y"] is not None:
        share = t["y"].abs() if t["after"] is None else (t["y"] / rms(t["y"]) * t["after"]).abs()
    open_ = slope = None
    if t["gate"] is not None:
        each = share.shape[0] // t["gate"].shape[0]
        g = t["gate"].repeat_interleave(each, 0)
        s = 1 / (1 + torch.exp(-g))
        open_ = L.act(activation, g).abs()
        slope = torch.ones_like(g) if activation == "none" else s * (1.0 + g.abs())     # (no less than its parts)
    u = share if open_ is None else share * open_
    size = abs(b) * u + (0.0 if t["x"] is None else (a * t["x"]).abs())
    h, z, grads = L.residual_norm(given, activation, a, b, eps, dh, dz)
    root = rms(h)
    more = torch.clamp(rms(size) / root, min=1.0)                         # what cancels in h weighs the more in its norm
    tol = {"h": types["x"] * h.abs() + c * size}
    if z is not None:
        tol["z"] = types["y"] * z.abs() + c * t["before"].abs() * (size + h.abs() * more) / root
    if dh is None and dz is None:
        return h, z, grads, {n: 1.01 * v + 1e-30 for n, v in tol.items()}
    m = torch.zeros_like(h) if dh is None else dh.double().cpu().abs()
    c = 4 * c * more
    rows = h.shape[0]
    added = lambda v, unit, k: unit * v.sum(0).abs() + ((c + rows * L.EPS32) * k).sum(0)  # noqa: E731
    if dz is not None:
        d = (dz.double().cpu() * t["before"]).abs()
        normed = size / root
        tol["before"] = types["before"] * grads["before"].abs() + ((c + rows * L.EPS32) * dz.double().cpu().abs() * normed).sum(0)
        m = m + (d + normed * (normed * d).mean(-1, keepdim=True)) / root
    if "x" in grads:
        tol["x"] = types["x"] * grads["x"].abs() + c * abs(a) * m
    if t["y"] is not None:
        m = abs(b) * m
        if t["gate"] is not None:
            k = c * m * share * slope
            if t["gate"].shape[0] < rows:
                k = ((c + rows * L.EPS32) * m * share * slope).view(t["gate"].shape[0], -1, k.shape[1]).sum(1)
            tol["gate"] = types["y"] * grads["gate"].abs() + k
            m = m * open_
        if t["after"] is not None:
            normed = (t["y"] / rms(t["y"])).abs()
            tol["after"] = types["after"] * grads["after"].abs() + ((c + rows * L.EPS32) * m * normed).sum(0)
            m = m * t["after"].abs()
            m = (m + normed * (normed * m).mean(-1, keepdim=True)) / rms(t["y"])
        tol["y"] = types["y"] * grads["y"].abs() + c * m
    return h, z, grads, {n: 1.01 * v + 2.0 ** -24 * (types["y"] == L.UNIT["f16"]) + 1e-30 for n, v in tol.items()}


def _check(given, activation, a, b, eps, stream, block, weights, train, want_dh=True, want_dz=True):
    import paper_1609_01882_amd as psc
    some = given["x"] if given["x"] is not None else given["y"]
    g = torch.Generator().manual_seed(1)
    dh = torch.randn(some.shape, generator=g).to(some.dtype).cuda() if train and want_dh else None
    dz = torch.randn(some.shape, generator=g).to((given["y"] if given["y"] is not None else some).dtype).cuda() if train and given["before"] is not None and want_dz else None
    block = block if given["y"] is not None else stream
    types = {"x": L.UNIT[stream if given["x"] is not None else block], "y": L.UNIT[block], "after": L.UNIT[weights], "before": L.UNIT[weights]}
    h, z, grads, tol = _tolerances(given, activation, a, b, eps, dh, dz, types)
    leaf = {n: None if t is None else t.detach().requires_grad_(train) for n, t in given.items()}
    got_h, got_z = psc.residual_norm(leaf["x"], leaf["y"], gate=leaf["gate"], activation=activation, after=leaf["after"], before=leaf["before"],
                                     residual_scale=a, block_scale=b, eps=eps)
    assert got_h.dtype == some.dtype and (got_z is None) == (z is None)
    pairs = [("h", got_h, h)] + ([] if z is None else [("z", got_z, z)])
    if train:
        names = [n for n in NAMES if given[n] is not None]
        outs, ups = zip(*((o, d) for o, d in ((got_h, dh), (got_z, dz)) if d is not None))
        for n, t in zip(names, torch.autograd.grad(outs, [leaf[n] for n in names], ups, allow_unused=True)):
            if t is None:
                assert n == "before" and dz is None
                continue
            assert t.dtype == given[n].dtype and t.shape == given[n].shape
            pairs.append((n, t, grads[n]))
            tol.setdefault(n, torch.full_like(grads[n], 1e-30))
    for n, x, y in pairs:
        worst = L.finite_or_same(x.detach().double().cpu().numpy(), y.numpy(), tol[n].numpy())
        assert worst <= 1.0, (n, worst)


SHAPES = [(1, 1), (5, 7), (3, 64), (70, 65), (33, 128), (9, 500), (40, 512), (17, 520), (6, 1003), (2, 2048), (3, 4096), (2, 5001), (2, 8192), (2, 12_345), (1, 16_384)]


@pytest.mark.parametrize("stream,block,weights", [("bf16", "bf16", "f32"), ("f32", "bf16", "bf16"), ("f16", "f16", "f16"), ("f32", "f16", "f32"), ("f32", "f32", "f32")])
@pytest.mark.parametrize("rows,width", SHAPES)
def test_all_of_it(rows, width, stream, block, weights):
    print(f"norm {rows} x {width} {stream} {block} {weights}", flush=True)
    _check(_given(rows + width, rows, width, stream, block, weights, rows, NAMES), "sigmoid", 1.0, 0.7, 1e-6, stream, block, weights, True)


@pytest.mark.parametrize("has", [("x", "before"), ("y", "after"), ("y", "after", "gate"), ("x", "y"), ("x", "y", "before"), ("x", "y", "after", "before"),
                                 ("x", "y", "gate", "before"), ("y", "before"), ("x", "y", "gate")])
@pytest.mark.parametrize("rows,width", [(13, 96), (5, 1003), (4, 4096)])
def test_parts_of_it(rows, width, has):
    _check(_given(7, rows, width, "bf16", "bf16", "f32", rows, has), "silu", 0.5, -1.5, 1e-5, "bf16", "bf16", "f32", True)
    _check(_given(8, rows, width, "f32", "f32", "f32", rows, has), "none", 1.0, 1.0, 0.0, "f32", "f32", "f32", True)


@pytest.mark.parametrize("activation", ["none", "sigmoid", "silu"])
@pytest.mark.parametrize("rows,gates,width", [(12, 1, 72), (12, 3, 200), (700, 1, 1003), (4800, 6, 64), (3000, 1500, 40), (4000, 2000, 1032), (60, 60, 33), (6, 2, 8200)])
def test_gates_that_rows_share(rows, gates, width, activation):
    print(f"gates {rows} / {gates} x {width}", flush=True)
    _check(_given(rows, rows, width, "f32", "bf16", "f32", gates, NAMES), activation, 1.0, 1.0, 1e-6, "f32", "bf16", "f32", True)


@pytest.mark.parametrize("rows,width", [(5000, 64), (3001, 1000), (1500, 4096)])
def test_many_rows(rows, width):
    _check(_given(rows, rows, width, "f32", "f32", "f32", rows, NAMES), "silu", 1.0, 1.0, 1e-6, "f32", "f32", "f32", True)


def test_only_one_gradient_flows():
    given = _given(1, 9, 300, "f32", "bf16", "f32", 3, NAMES)
    _check(given, "sigmoid", 1.0, 0.5, 1e-6, "f32", "bf16", "f32", True, want_dh=False)
    _check(given, "sigmoid", 1.0, 0.5, 1e-6, "f32", "bf16", "f32", True, want_dz=False)


def test_gradients_by_differences():
    import paper_1609_01882_amd as psc
    given = _given(3, 6, 40, "f32", "f32", "f32", 2, NAMES)
    dh, dz = torch.randn((6, 40), device="cuda"), torch.randn((6, 40), device="cuda")

    def f(t):
        h, z = psc.residual_norm(t["x"], t["y"], gate=t["gate"], activation="silu", after=t["after"], before=t["before"], block_scale=0.5)
        return (h.double() * dh.double()).sum() + (z.double() * dz.double()).sum()

    leaf = {n: t.requires_grad_() for n, t in given.items()}
    grads = dict(zip(NAMES, torch.autograd.grad(f(leaf), [leaf[n] for n in NAMES])))
    step = 2.0 ** -7
    for n in NAMES:
        v = torch.randn_like(given[n])
        with torch.no_grad():
            left = (f({**given, n: given[n] + step * v}) - f({**given, n: given[n] - step * v})) / (2 * step)
        right = (grads[n].double() * v.double()).sum()
        # the third derivative's share, step^2 / 6 of up to some tens of the first's size; roundings of 480 sums over 2 steps
        assert abs(float(left - right)) < 40 * step ** 2 * float(grads[n].norm() * v.norm()) + 480 * 64 * L.EPS32 / step, n


def test_large_and_special_values():
    import paper_1609_01882_amd as psc
    x = torch.randn((6, 100), device="cuda")
    x[1] = 0.0
    x[2, 5] = float("nan")
    x[3, 7] = float("inf")
    y, w = torch.randn((6, 100), device="cuda"), torch.ones(100, device="cuda")
    y[1] = 0.0
    g = torch.full((6, 100), 200.0, device="cuda")
    g[4] = -200.0
    h, z = psc.residual_norm(x, y, gate=g, activation="sigmoid", after=w, before=w)
    assert bool((h[1] == 0).all()) and bool((z[1] == 0).all())
    assert bool(z[2].isnan().all()) and not bool(z[0].isnan().any())
    assert torch.equal(h[4], x[4])                                            # the gate is shut
    assert bool(h[3].isinf().sum() == 1)


def test_strides_and_shapes():
    import paper_1609_01882_amd as psc
    whole = torch.randn((4, 5, 3 * 96), device="cuda").bfloat16()
    x, y, g = whole[..., :96], whole[..., 96:192], whole[..., 192:]
    w = torch.randn(96, device="cuda")
    h, z = psc.residual_norm(x, y, gate=g, activation="silu", after=w, before=w)
    h2, z2 = psc.residual_norm(x.contiguous(), y.contiguous(), gate=g.contiguous(), activation="silu", after=w, before=w)
    assert h.shape == x.shape and torch.equal(h, h2) and torch.equal(z, z2)
    same, z3 = psc.residual_norm(x, before=w)
    assert same is x and torch.equal(z3, psc.residual_norm(x.contiguous(), before=w, residual_scale=1.0)[1])
    assert psc.residual_norm(x, None) == (x, None)
    none = psc.residual_norm(x[:0], y[:0], before=w)
    assert none[0].shape == (0, 5, 96) and none[1].shape == (0, 5, 96)
    empty = [t.detach().requires_grad_() for t in (x[0, :0], y[0, :0], w)]
    h, z = psc.residual_norm(empty[0], empty[1], before=empty[2])
    assert torch.equal(torch.autograd.grad(z.sum(), empty[2])[0], torch.zeros_like(w))


def test_gradients_as_autograd_hands_them_over():
    import paper_1609_01882_amd as psc
    x, y, w = (torch.randn(s, device="cuda", requires_grad=True) for s in ((5, 4, 40), (5, 4, 40), (40,)))
    h, z = psc.residual_norm(x, y, after=w, before=w)
    # sums hand over one value, expanded; transposed products a transposed one
    got = torch.autograd.grad(h.sum() + (z.transpose(0, 2) * 2.0).sum(), (x, y, w), retain_graph=True)
    ones = torch.ones_like(h)
    want = torch.autograd.grad((h, z), (x, y, w), (ones, 2.0 * ones), retain_graph=True)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    # the sum of a weight that stands in two places is that of both
    a, b = w.detach().clone().requires_grad_(), w.detach().clone().requires_grad_()
    h, z = psc.residual_norm(x, y, after=a, before=b)
    ga, gb = torch.autograd.grad((h, z), (a, b), (ones, 2.0 * ones))
    assert torch.equal(ga + gb, want[2])
    # one stream tensor as both
    h, z = psc.residual_norm(x, x, before=w, block_scale=0.5)
    gx, = torch.autograd.grad((h, z), x, (ones, ones))
    x1, x2 = x.detach().clone().requires_grad_(), x.detach().clone().requires_grad_()
    g1, g2 = torch.autograd.grad(psc.residual_norm(x1, x2, before=w, block_scale=0.5), (x1, x2), (ones, ones))
    assert torch.equal(gx, g1 + g2)
    # no second derivative, and no gradient of what has been overwritten
    h, z = psc.residual_norm(x, y, after=w, before=w)
    first, = torch.autograd.grad(z.sum(), y, create_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(first.sum(), y)
    v = y * 1.0
    h, z = psc.residual_norm(x, v, after=w, before=w)
    v.mul_(2.0)
    with pytest.raises(RuntimeError):
        z.sum().backward()


def test_results_repeat_and_graphs_replay():
    import paper_1609_01882_amd as psc
    given = _given(5, 900, 1000, "f32", "bf16", "f32", 3, NAMES)
    dh, dz = torch.randn((900, 1000), device="cuda"), torch.randn((900, 1000), device="cuda").bfloat16()

    def step(leaf):
        h, z = psc.residual_norm(leaf["x"], leaf["y"], gate=leaf["gate"], activation="sigmoid", after=leaf["after"], before=leaf["before"])
        return [h.detach(), z.detach(), *torch.autograd.grad((h, z), [leaf[n] for n in NAMES], (dh, dz))]

    eager = {n: t.detach().clone().requires_grad_() for n, t in given.items()}
    want = step(eager)
    assert all(torch.equal(a, b) for a, b in zip(want, step(eager)))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    leaf = {n: t.detach().clone().requires_grad_() for n, t in given.items()}
    with torch.cuda.stream(stream):
        assert all(torch.equal(a, b) for a, b in zip(want, step(leaf)))
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = step(leaf)
    for turn in range(3):
        with torch.no_grad():
            for n in NAMES:
                eager[n].mul_(1.0 + 0.1 * turn)
                leaf[n].copy_(eager[n])
        want = step(eager)
        for t in res:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, res))


def test_refusals():
    import paper_1609_01882_amd as psc
    x, w = torch.zeros((6, 32), device="cuda"), torch.ones(32, device="cuda")
    h = x.half()
    for call in (lambda: psc.residual_norm(None), lambda: psc.residual_norm(x, gate=x), lambda: psc.residual_norm(x, after=w),
                 lambda: psc.residual_norm(x, x[:5]), lambda: psc.residual_norm(h, x), lambda: psc.residual_norm(h, x.bfloat16()), lambda: psc.residual_norm(x.cpu(), before=w.cpu()),
                 lambda: psc.residual_norm(x.double(), before=w), lambda: psc.residual_norm(x, x, gate=x[:4]), lambda: psc.residual_norm(x, x, gate=h),
                 lambda: psc.residual_norm(x, x, gate=x[:0]), lambda: psc.residual_norm(x, h, after=w, before=w.half()), lambda: psc.residual_norm(x, h, before=w.bfloat16()),
                 lambda: psc.residual_norm(x, x, before=w[:31]), lambda: psc.residual_norm(x, x, gate=x, activation="tanh"),
                 lambda: psc.residual_norm(x.t(), x.t(), before=w[:6]), lambda: psc.residual_norm(torch.zeros((2, 16_385), device="cuda"), before=torch.zeros(16_385, device="cuda")),
                 lambda: psc.residual_norm(x.view(2, 3, 32).transpose(0, 1), before=w), lambda: psc.residual_norm(x, x, eps=-1.0, before=w),
                 lambda: psc.residual_norm(x, x, block_scale=float("nan"))):
        with pytest.raises(psc.PscError):
            call()
