"""Refusals of the attention memory's calls and the definition that its tests go by (no GPU: nothing is launched)."""
import ctypes as C
import os

import numpy as np
import pytest

import kv_util as U


@pytest.fixture(scope="module")
def lib():
    import paper_1609_01882_amd as p
    from paper_1609_01882_amd import binding
    if not os.path.exists(p.lib_path()):
        import __graft_entry__ as g
        g.build()
    return binding._load()


def _cache(**other):
    from paper_1609_01882_amd.kv import _Cache
    f = dict(k_codes=4096, k_scales=4096, v_codes=4096, v_scales=4096, pages=8, kv_heads=2, head_dim=128, page=32, table=4096, batch=3,
             table_width=4, lengths=4096)
    f.update(other)
    return _Cache(**f)


A = 4096  # stands for an aligned device address: refused calls do not look at it


def _append(lib, cache=None, dtype=0, k=A, ks=(256, 128), v=A, vs=(256, 128), n=6, offsets=None, first=None, positions=None, weights=None):
    return lib.psc_kv_append(C.byref(cache or _cache()), dtype, k, *ks, v, *vs, n, offsets, first, positions, weights, None)


def _attend(lib, cache=None, dtype=0, q=A, qs=(512, 128), n=6, most=2, heads=4, offsets=None, first=None, positions=None, scale=0.1, causal=1,
            window=0, sinks=0, out=A, lse=A, w_in=None, w_out=None, ws=A, size=1 << 30):
    return lib.psc_kv_attention(C.byref(cache or _cache()), dtype, q, *qs, n, most, heads, offsets, first, positions, scale, causal, window, sinks,
                                out, lse, w_in, w_out, ws, size, None)


def _evict(lib, cache=None, w=A, positions=None, seen=None, budget=16, sinks=4, recent=8, kept=A, lengths=A, p_out=A, w_out=2 * A, stride=16, ws=A,
           size=1 << 30):
    return lib.psc_kv_evict(C.byref(cache or _cache()), w, positions, seen, budget, sinks, recent, kept, lengths, p_out, w_out, stride, ws, size, None)


BAD_CACHES = [dict(head_dim=96), dict(head_dim=0), dict(page=48), dict(page=8), dict(page=512), dict(kv_heads=0), dict(batch=0), dict(batch=40_000),
              dict(pages=0), dict(pages=1 << 31), dict(pages=1 << 29, page=64), dict(table_width=0), dict(table_width=1 << 26), dict(k_codes=None), dict(v_scales=None),
              dict(k_codes=4104), dict(table=None), dict(lengths=None), dict(lengths=4097)]


@pytest.mark.parametrize("bad", BAD_CACHES, ids=lambda d: "-".join(f"{k}={v}" for k, v in d.items()))
def test_bad_caches_are_refused(lib, bad):
    assert _append(lib, _cache(**bad)) == -1 and lib.psc_last_error()
    assert _attend(lib, _cache(**bad)) == -1
    assert _evict(lib, _cache(**bad)) == -1
    assert lib.psc_kv_read(C.byref(_cache(**bad)), 0, 6, None, A, A, None) == -1


@pytest.mark.parametrize("bad", [dict(dtype=3), dict(dtype=-1), dict(k=None), dict(v=None), dict(k=4100), dict(ks=(260, 128)), dict(vs=(256, 4)),
                                 dict(n=7), dict(n=-3), dict(offsets=4097), dict(positions=4100), dict(weights=4104), dict(dtype=2, ks=(258, 128))])
def test_bad_appends_are_refused(lib, bad):
    assert _append(lib, **bad) == -1 and lib.psc_last_error()


@pytest.mark.parametrize("bad", [dict(dtype=9), dict(q=None), dict(q=4098), dict(qs=(516, 128)), dict(heads=3), dict(heads=0), dict(n=7), dict(n=-1),
                                 dict(offsets=A, most=0), dict(offsets=A, most=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
                                 dict(scale=float("inf")), dict(window=-1), dict(sinks=-1), dict(causal=0, window=5), dict(out=None), dict(out=4104),
                                 dict(w_in=A), dict(positions=4100), dict(w_out=4104), dict(w_out=A, ws=None, size=0), dict(w_out=A, size=8),
                                 dict(w_out=A, ws=4100), dict(n=1 << 30, heads=4), dict(lse=4097)])
def test_bad_attentions_are_refused(lib, bad):
    assert _attend(lib, **bad) == -1 and lib.psc_last_error()


@pytest.mark.parametrize("bad", [dict(budget=0), dict(budget=-1), dict(sinks=-1), dict(recent=-1), dict(sinks=9, recent=8), dict(w=None), dict(kept=None),
                                 dict(lengths=None), dict(w_out=None), dict(stride=15), dict(w_out=A), dict(positions=A), dict(ws=None),
                                 dict(size=3 * 2 * 16 * 8 - 1), dict(ws=4100), dict(kept=4098)])
def test_bad_evictions_are_refused(lib, bad):
    assert _evict(lib, **bad) == -1 and lib.psc_last_error()


def test_null_cache_and_no_rows(lib):
    assert lib.psc_kv_append(None, 0, A, 256, 128, A, 256, 128, 6, None, None, None, None, None) == -1
    assert lib.psc_kv_attention_workspace_bytes(None, 0, 6, 2, 4, 0, 0, 0, 0) == 0
    assert _append(lib, n=0, k=None, v=None) == 0                     # nothing to do: no device is touched
    assert _attend(lib, n=0, q=None, out=None) == 0
    assert lib.psc_kv_read(C.byref(_cache()), 0, 0, None, None, None, None) == 0


def test_workspaces_grow_with_what_they_hold(lib):
    size = lambda rows, weights, **kw: lib.psc_kv_attention_workspace_bytes(C.byref(_cache(**kw)), 0, rows, rows // 3, 4, 0, 0, 0, weights)  # noqa: E731
    assert size(3, 1) >= 3 * 4 * 8 and size(3, 1) > size(3, 0)
    assert size(3, 0, table_width=4096) > size(3, 0)
    assert lib.psc_kv_evict_workspace_bytes(C.byref(_cache()), 100) >= 3 * 2 * 100 * 8
    assert lib.psc_kv_evict_workspace_bytes(C.byref(_cache()), 0) == 0


def test_the_tests_own_rounding():
    """The host definition on values whose codes are known."""
    x = np.zeros(32)
    x[:9] = [6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.3]
    codes, scales, _, _ = U.round_to_4_bits(x, x)
    assert scales[0] == 127 and codes[:9].tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 9]
    for top, e in ((7.0, 0), (7.001, 1), (4.0, 0), (3.5, -1), (3.51, 0), (0.0, -23), (1e9, 13)):
        x[0] = top
        x[1:] = 0.0
        assert U.round_to_4_bits(x, x)[1][0] == 127 + e, top
    rng = np.random.default_rng(0)
    x = rng.normal(size=(50, 64))
    codes, scales, _, _ = U.round_to_4_bits(x, x)
    err = np.abs(U.values(U.pack(codes), scales) - x).reshape(50, 2, 32)
    assert np.all(err <= 2.0 ** (scales.astype(float) - 127)[..., None])     # at most one step of the coarsest part of the grid


def test_the_tests_own_eviction():
    w = np.array([[[5.0, 1.0, 3.0, 3.0, 9.0, 0.5, 3.0, 2.0]]], np.float32)
    assert U.evict([8], w, None, None, 4, 1, 1)[0, 0].tolist() == [0, 4, 2, 7]
    assert U.evict([3], w, None, None, 4, 1, 1)[0, 0].tolist() == [0, 1, 2, -1]
