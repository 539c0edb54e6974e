"""Sizes and refusals of the attention memory's calls at their limits (no GPU: nothing is launched)."""
import ctypes as C
import os

import pytest

from test_kv_host import A, _append, _attend, _cache, _evict


@pytest.fixture(scope="module")
def lib():
    import paper_1609_01882_amd as p
    from paper_1609_01882_amd import binding
    if not os.path.exists(p.lib_path()):
        import __graft_entry__ as g
        g.build()
    return binding._load()


def _size(lib, rows, most, heads=4, weights=0, window=0, **cache):
    return lib.psc_kv_attention_workspace_bytes(C.byref(_cache(**cache)), 0, rows, most, heads, window, 0, 0, weights)


def test_sizes_hold_whether_or_not_the_rows_have_offsets(lib):
    """Without offsets the call takes rows / batch for max_rows, whatever the size was asked with."""
    for width in (4, 100, 4096):
        for rows in (3, 60, 600, 60_000):
            need = _size(lib, rows, rows // 3, table_width=width)
            for most in (0, 1, rows, 100 * rows):
                assert _size(lib, rows, most, table_width=width) >= need, (width, rows, most)


def test_more_rows_than_the_sequences_may_have_are_refused(lib):
    for bad in (dict(n=60, most=19), dict(n=60, most=1), dict(n=4, most=1)):
        assert _attend(lib, offsets=A, **bad) == -1 and b"max_rows" in lib.psc_last_error()


LANES = 1 << 32    # a dimension of a grid has fewer


def test_more_rows_than_a_grid_has_lanes_for_are_refused(lib):
    for dim, heads in ((128, 2), (256, 1), (64, 48)):
        kw = dict(head_dim=dim, kv_heads=heads)
        n = -(-LANES // (heads * dim // 8 * 3)) * 3                  # (a multiple of the three sequences)
        assert _append(lib, _cache(**kw), n=n) == -1 and b"rows" in lib.psc_last_error()
        assert lib.psc_kv_read(C.byref(_cache(**kw)), 0, n, None, A, A, None) == -1 and b"rows" in lib.psc_last_error()


def test_a_budget_that_a_grid_has_no_lanes_for_is_refused(lib):
    budget = -(-LANES // (3 * 2 * 4))
    assert _evict(lib, budget=budget, stride=budget, size=1 << 60) == -1 and b"budget" in lib.psc_last_error()


def test_attention_that_a_grid_has_no_lanes_for_is_refused(lib):
    one = dict(batch=1, kv_heads=1)
    n = (1 << 30) - 32                                               # units of 32 rows, a workgroup of 256 to each
    assert _attend(lib, _cache(**one), n=n, most=n, heads=1, size=1 << 60) == -1 and b"rows" in lib.psc_last_error()
    # weights of many rows: a workgroup to 32 slots of 256 coordinates
    wide = _cache(**one, head_dim=256, page=256, table_width=1 << 21)
    assert _attend(lib, wide, n=100, most=100, heads=1, w_out=A, size=1 << 60) == -1 and b"weights" in lib.psc_last_error()


def test_kept_scores_are_bounded(lib):
    """Eight rows of 64 x 8 memories of a million slots: their scores would take 17 GB."""
    small = _size(lib, 64, 1, heads=64, weights=1, batch=64, kv_heads=8, page=64, table_width=64)
    assert small >= 64 * 8 * 8 * 4096 * 4
    assert _size(lib, 64, 1, heads=64, weights=1, batch=64, kv_heads=8, page=64, table_width=16_384) < 9 << 29
