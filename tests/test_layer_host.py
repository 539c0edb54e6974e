"""Refusals of the calls around the attention memory, frequencies, and the definitions that their tests go by (no GPU: nothing is launched)."""
import ctypes as C
import math
import os
from fractions import Fraction

import numpy as np
import pytest
import torch

import kv_util as U
import layer_util as L


@pytest.fixture(scope="module")
def lib():
    import paper_1609_01882_amd as p
    from paper_1609_01882_amd import binding
    if not os.path.exists(p.lib_path()):
        import __graft_entry__ as g
        g.build()
    return binding._load()


A = 4096  # stands for an aligned device address: refused calls do not look at it


def _ids(d):
    return "-".join(f"{k}={v}" for k, v in d.items())


# ------------------------------------------------------------------------------------------- rotary positions
def _pi():
    """pi to 500 bits, from 16 arctan(1/5) - 4 arctan(1/239)."""
    one = 1 << 520

    def arctan(x):
        term, total, n, sign = one // x, one // x, 3, -1
        while term:
            term //= x * x
            total += sign * (term // n)
            n, sign = n + 2, -sign
        return total

    return Fraction(4 * (4 * arctan(5) - arctan(239)), one)


def test_turns_are_exact(lib):
    radians = [1.0, 0.1, 1e-4, 3.3, 1000.0, 1024.0, -1024.0, 1e-12, 5e-324, -0.7, 1e-30, math.pi, 2 * math.pi, 0.0, -0.0, 10000.0 ** (-126 / 128)]
    turns = (C.c_uint64 * len(radians))()
    assert lib.psc_rotary_turns((C.c_double * len(radians))(*radians), len(radians), turns) == 0
    pi = _pi()
    for f, t in zip(radians, turns):
        assert t == round(Fraction(f) / (2 * pi) * 2 ** 64) % 2 ** 64, f
    for bad in (float("nan"), float("inf"), 1025.0, -1e300):
        assert lib.psc_rotary_turns((C.c_double * 1)(bad), 1, turns) == -1
    assert lib.psc_rotary_turns(None, 1, turns) == -1 and lib.psc_rotary_turns(None, -1, None) == -1 and lib.psc_rotary_turns(None, 0, None) == 0


def test_frequencies():
    import paper_1609_01882_amd as psc
    plain = psc.rotary_frequencies(8, 100.0)
    assert plain == [1.0, 100.0 ** -0.25, 0.1, 100.0 ** -0.75]
    assert psc.rotary_frequencies(8, 100.0, stretch=4.0) == [f / 4.0 for f in plain]
    f = psc.rotary_frequencies(128, stretch=8.0, trained=8192)
    turns = [8192 * x / (2 * math.pi) for x in psc.rotary_frequencies(128)]
    for x, y, t in zip(f, psc.rotary_frequencies(128), turns):
        keep = min(max((t - 1.0) / 3.0, 0.0), 1.0)
        assert x == pytest.approx(y * keep + y / 8.0 * (1 - keep), rel=1e-15)
    assert f[0] == 1.0 and f[-1] == pytest.approx(10000.0 ** (-126 / 128) / 8, rel=1e-15)
    by_pairs = psc.rotary_frequencies(128, stretch=16.0, trained=4096, low=1.0, high=32.0, blend="pairs")
    assert by_pairs[:20] == psc.rotary_frequencies(128)[:20] and by_pairs[-10:] == [x / 16.0 for x in psc.rotary_frequencies(128)[-10:]]
    assert all(a > b for a, b in zip(by_pairs, by_pairs[1:]))
    for bad in (dict(dims=7), dict(dims=0), dict(dims=8, base=1.0), dict(dims=8, stretch=0.0), dict(dims=8, trained=0), dict(dims=8, trained=10, low=4.0, high=4.0),
                dict(dims=8, trained=10, blend="?"), dict(dims=8, base=float("inf"))):
        with pytest.raises(psc.PscError):
            psc.rotary_frequencies(**bad)


def _rotary(**other):
    from paper_1609_01882_amd.layer import _Rotary
    f = dict(turns=A, dims=64, interleaved=0, factor=1.0)
    f.update(other)
    return _Rotary(*f.values())


def _rows(lib, rotary=None, dtype=0, x=A, xs=(256, 64), n=6, heads=4, dim=64, positions=None, batch=3, offsets=None, first=None, out=2 * A, os_=(256, 64)):
    return lib.psc_rotary_rows(C.byref(rotary or _rotary()), 0, dtype, x, *xs, n, heads, dim, positions, batch, offsets, first, out, *os_, None)


@pytest.mark.parametrize("bad", [dict(dtype=3), dict(dtype=-1), dict(x=None), dict(out=None), dict(x=A + 1), dict(out=A + 1), dict(n=-1), dict(n=7), dict(heads=0),
                                 dict(heads=65537), dict(dim=62), dict(dim=1), dict(dim=65537), dict(batch=0), dict(positions=A, first=A), dict(positions=A, offsets=A),
                                 dict(positions=A + 2), dict(offsets=A + 1), dict(first=A + 1), dict(xs=(1 << 40, 64)), dict(os_=(256, -(1 << 40))), dict(out=A, os_=(512, 64)),
                                 dict(n=1 << 30, heads=64, dim=512, offsets=A)], ids=_ids)
def test_bad_rows_are_refused(lib, bad):
    assert _rows(lib, **bad) == -1 and lib.psc_last_error()


@pytest.mark.parametrize("bad", [dict(turns=None), dict(turns=A + 4), dict(dims=0), dict(dims=63), dict(dims=66), dict(dims=-2), dict(factor=float("nan"))], ids=_ids)
def test_bad_rotaries_are_refused(lib, bad):
    assert _rows(lib, _rotary(**bad)) == -1
    assert _append(lib, rotary=_rotary(**bad)) == -1


def test_no_rows_are_no_call(lib):
    assert _rows(lib, n=0) == 0 and _rows(lib, n=0, x=None, out=None) == 0
    assert _append(lib, n=0) == 0


# ------------------------------------------------------------------------------------------- the memory's calls
def _cache(**other):
    from paper_1609_01882_amd.kv import _Cache
    f = dict(k_codes=4096, k_scales=4096, v_codes=4096, v_scales=4096, pages=8, kv_heads=2, head_dim=128, page=32, table=4096, batch=3, table_width=4, lengths=4096)
    f.update(other)
    return _Cache(**f)


def _append(lib, cache=None, rotary=None, dtype=0, k=A, ks=(256, 128), v=A, vs=(256, 128), q=A, qs=(512, 128), q_heads=4, q_out=2 * A, n=6, offsets=None, first=None,
            positions=None, weights=None):
    return lib.psc_kv_append_rotary(C.byref(cache or _cache()), C.byref(rotary or _rotary()), dtype, k, *ks, v, *vs, q, *qs, q_heads, q_out, n, offsets, first,
                                    positions, weights, None)


@pytest.mark.parametrize("bad", [dict(dtype=3), dict(k=None), dict(v=None), dict(q=None), dict(q_out=None), dict(q_out=A), dict(k=A + 8), dict(q=A + 8), dict(q_out=A + 8),
                                 dict(ks=(260, 128)), dict(vs=(256, 4)), dict(qs=(512, 4)), dict(n=7), dict(n=-1), dict(q_heads=-1), dict(q_heads=65537), dict(offsets=A + 2),
                                 dict(first=A + 2), dict(positions=A + 4), dict(weights=A + 4), dict(rotary=None, n=3 << 28, q_heads=64)], ids=_ids)
def test_bad_appends_are_refused(lib, bad):
    assert _append(lib, **bad) == -1 and lib.psc_last_error()


def test_dimensions_in_sixteens_for_the_memory(lib):
    assert _append(lib, rotary=_rotary(dims=24)) == -1 and _append(lib, _cache(head_dim=64), rotary=_rotary(dims=80)) == -1
    assert lib.psc_kv_append_rotary(C.byref(_cache()), None, 0, A, 256, 128, A, 256, 128, A, 512, 128, 4, 2 * A, 6, None, None, None, None, None) == -1


def _difference(lib, cache=None, dtype=0, q=A, qs=(512, 128), n=6, most=2, heads=4, offsets=None, first=None, positions=None, scale=0.1, causal=1, window=0, sinks=0,
                lam=A, lam_stride=0, norm=None, eps=1e-6, factor=1.0, out=A, lse=A, w_in=None, w_out=None, ws=A, size=1 << 30):
    return lib.psc_kv_difference(C.byref(cache or _cache()), dtype, q, *qs, n, most, heads, offsets, first, positions, scale, causal, window, sinks, lam, lam_stride,
                                 norm, eps, factor, out, lse, w_in, w_out, ws, size, None)


@pytest.mark.parametrize("bad", [dict(cache=dict(kv_heads=3), heads=3), dict(cache=dict(head_dim=256)), dict(cache=dict(head_dim=96)), dict(cache=dict(k_codes=None)), dict(dtype=3),
                                 dict(q=None), dict(q=A + 8), dict(qs=(510, 128)), dict(n=7), dict(n=-1), dict(most=0, offsets=A), dict(most=1, offsets=A), dict(heads=3),
                                 dict(heads=0), dict(heads=65538), dict(offsets=A + 1), dict(first=A + 1), dict(positions=A + 4), dict(scale=0.0), dict(scale=float("nan")),
                                 dict(scale=float("inf")), dict(window=-1), dict(sinks=-1), dict(window=4, causal=0), dict(lam=None), dict(lam=A + 2), dict(lam_stride=1 << 40),
                                 dict(norm=A + 2), dict(norm=A, eps=-1.0), dict(norm=A, eps=float("nan")), dict(factor=float("inf")), dict(out=None), dict(out=A + 8),
                                 dict(lse=A + 2), dict(w_in=A), dict(w_out=A + 4), dict(w_out=A, size=16), dict(w_out=A, ws=None), dict(ws=A + 8)], ids=_ids)
def test_bad_differences_are_refused(lib, bad):
    bad = dict(bad)
    if "cache" in bad:
        bad["cache"] = _cache(**bad["cache"])
    assert _difference(lib, **bad) == -1 and lib.psc_last_error()


def test_workspaces_of_differences(lib):
    size = lambda n, most, heads=8, dtype=0, weights=0, **c: lib.psc_kv_difference_workspace_bytes(C.byref(_cache(**c)), dtype, n, most, heads, 0, 0, 0, weights)  # noqa: E731
    long = dict(table_width=4096, kv_heads=8)
    assert size(0, 0) == 0 and size(3, 1, kv_heads=3) == 0 and size(3, 1, head_dim=256) == 0 and size(3, 1, heads=7) == 0
    assert size(3, 1, **long) > 0 and size(3, 1, weights=1, **long) > size(3, 1, **long)
    # enough with offsets and without, whatever most was
    assert size(6, 6, **long) >= size(6, 2, **long)
    # a call with many rows needs none but for its weights
    assert size(3 * 4096, 4096, heads=64, batch=3, **{**long, "kv_heads": 8}) == 0


# ------------------------------------------------------------------------------------------- norms
def _norm(**other):
    from paper_1609_01882_amd.layer import _Norm
    f = dict(rows=6, width=64, stream_dtype=0, block_dtype=0, weight_dtype=2, x=A, x_stride=64, y=A, y_stride=64, gate=A, gate_stride=64, gate_rows=3, activation=1, after=A,
             before=A, residual_scale=1.0, block_scale=1.0, eps=1e-6)
    f.update(other)
    return _Norm(*f.values())


BAD_NORMS = [dict(rows=-1), dict(rows=1 << 30, gate=None), dict(width=0), dict(width=16385), dict(stream_dtype=3), dict(block_dtype=-1), dict(weight_dtype=1), dict(weight_dtype=5), dict(stream_dtype=1),
             dict(stream_dtype=0, block_dtype=2), dict(x=None, y=None), dict(y=None), dict(y=None, gate=None), dict(y=None, after=None), dict(activation=3), dict(activation=-1),
             dict(gate_rows=4), dict(gate_rows=0), dict(gate_rows=-3), dict(x=A + 1), dict(y=A + 1), dict(gate=A + 1), dict(after=A + 2), dict(before=A + 2),
             dict(x_stride=1 << 40), dict(gate_stride=-(1 << 40)), dict(residual_scale=float("nan")), dict(block_scale=float("inf")), dict(eps=-1e-6), dict(eps=float("nan"))]


@pytest.mark.parametrize("bad", BAD_NORMS, ids=_ids)
def test_bad_norms_are_refused(lib, bad):
    n = _norm(**bad)
    assert lib.psc_residual_norm_forward(C.byref(n), A, A, None, None) == -1 and lib.psc_last_error()
    assert lib.psc_residual_norm_workspace_bytes(C.byref(n)) == 0
    assert lib.psc_residual_norm_backward(C.byref(n), A, A, A, A, A, A, A, A, A, 1 << 30, None) == -1


def test_bad_gradients_are_refused(lib):
    size = lib.psc_residual_norm_workspace_bytes(C.byref(_norm()))
    assert size > 0

    def back(norm=None, stat=A, dh=A, dz=A, dx=A, dy=A, dgate=A, dafter=A, dbefore=A, ws=A, size=size):
        return lib.psc_residual_norm_backward(C.byref(norm or _norm()), stat, dh, dz, dx, dy, dgate, dafter, dbefore, ws, size, None)

    for bad in (dict(stat=None), dict(stat=A + 4), dict(ws=None), dict(ws=A + 8), dict(size=size - 1), dict(dh=A + 1), dict(dx=A + 1), dict(dafter=A + 2),
                dict(norm=_norm(before=None)), dict(norm=_norm(before=None), dz=None), dict(norm=_norm(gate=None)), dict(norm=_norm(x=None)),
                dict(norm=_norm(after=None)), dict(norm=_norm(rows=0))):
        assert back(**bad) == -1, bad
    assert lib.psc_residual_norm_forward(C.byref(_norm(before=None)), A, A, None, None) == -1
    assert lib.psc_residual_norm_forward(C.byref(_norm()), A + 1, A, None, None) == -1 and lib.psc_residual_norm_forward(C.byref(_norm()), A, A, A + 4, None) == -1
    assert lib.psc_residual_norm_forward(C.byref(_norm(rows=0)), None, None, None, None) == 0


def test_the_package_refuses_host_tensors():
    import paper_1609_01882_amd as psc
    with pytest.raises(psc.PscError):
        psc.residual_norm(torch.zeros(2, 4), before=torch.ones(4))
    with pytest.raises(psc.PscError):
        psc.residual_norm(None)
    with pytest.raises(psc.PscError):
        psc.Rotary(8, frequencies=[1.0], device="cpu")
    with pytest.raises(psc.PscError):
        psc.Rotary(8, factor=float("inf"), device="cpu")


# ------------------------------------------------------------------------------------------- the definitions themselves
def test_turned_is_a_rotation():
    rng = np.random.default_rng(1)
    x, at = rng.normal(size=(5, 2, 12)), rng.integers(0, 1 << 20, 5)
    f = [1.0, 0.3, 0.01, 1e-4]
    for interleaved in (False, True):
        y = L.turned(x, at, f, 8, interleaved)
        assert np.allclose(np.linalg.norm(y, axis=-1), np.linalg.norm(x, axis=-1), rtol=1e-12) and np.array_equal(y[..., 8:], x[..., 8:])
        assert np.allclose(L.turned(y, at, f, 8, interleaved, back=True), x, rtol=0, atol=1e-12)
        # products of rows depend on the distance of their positions alone
        a, b = (L.turned(x[:1], np.array([p]), f, 8, interleaved)[0, 0] @ L.turned(x[1:2], np.array([p + 7]), f, 8, interleaved)[0, 0] for p in (3, 100_000))
        assert abs(a - b) < 1e-9


def test_the_difference_of_two_equal_maps():
    rng = np.random.default_rng(2)
    buffers, table, lengths = L.random_memory(rng, 1, 2, 64, 16, [40])
    for buf in buffers[:2]:
        buf[:, 1] = buf[:, 0]                                # the same keys on both sides
    q = rng.normal(size=(1, 1, 64)).repeat(2, 1)
    args = (buffers, table, lengths, np.array([0, 1]), None, None, 0.125, True, 0, 0, None, 1e-6, 1.0, "f32")
    (whole, lse, got), _ = L.difference(q, np.zeros((1, 1)), *args)
    (half, _, _), _ = L.difference(q, np.full((1, 1), 0.5), *args)
    (none, _, _), _ = L.difference(q, np.ones((1, 1)), *args)
    assert np.allclose(half, whole / 2) and np.abs(none).max() < 1e-12 and lse[0, 0] == lse[0, 1]
    assert np.array_equal(got[0, 0], got[0, 1]) and got.sum() == pytest.approx(4.0)
    k, v, _ = U.held(buffers, table, 0, 0, 40)
    p = np.exp(0.125 * (k @ q[0, 0]) - lse[0, 0])
    assert np.allclose(whole[0, 0, :64], p @ v)


def test_gradients_of_the_definition_by_differences():
    g = torch.Generator().manual_seed(3)
    given = {n: torch.randn(s, generator=g, dtype=torch.float64) for n, s in (("x", (4, 6)), ("y", (4, 6)), ("gate", (2, 6)), ("after", (6,)), ("before", (6,)))}
    dh, dz = (torch.randn((4, 6), generator=g, dtype=torch.float64) for _ in range(2))
    for activation in ("none", "sigmoid", "silu"):
        grads = L.residual_norm(given, activation, 0.7, 1.3, 1e-6, dh, dz)[2]

        def f(t):
            h, z, _ = L.residual_norm(t, activation, 0.7, 1.3, 1e-6)
            return float((h * dh).sum() + (z * dz).sum())

        for n, t in given.items():
            v = torch.randn(t.shape, generator=g, dtype=torch.float64)
            left = (f({**given, n: t + 1e-5 * v}) - f({**given, n: t - 1e-5 * v})) / 2e-5
            assert abs(left - float((grads[n] * v).sum())) < 1e-6 * (1 + abs(left)), n
