"""Pages held behind a sequence's length: the oracle by hand, and what a loop without them loses (no GPU)."""
import ctypes

import numpy as np
import pytest

from oracle import pages as op


def test_held_by_hand():
    tab = np.array([[5, 6, -1, -1], [-1, -1, -1, -1], [7, 8, 9, -1]], np.int32)
    got, slots, taken, held = op.reserve_held(tab, [3, 16, 32], [30, 2, 1], np.arange(20, 40), 2, [2, 0, 3], [-1, 2, -1])
    assert got.tolist() == [[5, 6, 22, -1], [7, 23, -1, -1], [7, 8, 9, -1]] and taken == 4 and held == [3, 2, 3]
    assert slots.tolist() == [5 * 16 + t for t in range(3, 16)] + [6 * 16 + t for t in range(16)] + [22 * 16] + \
        [23 * 16, 23 * 16 + 1, 9 * 16]


def test_rows_taken_back():
    """K = 8: a call reserves n_new + 7 rows and keeps one."""
    for known in (False, True):
        tab, taken, held, rows = np.full((1, 40), -1, np.int32), 0, [0], np.arange(1000)
        for length in range(200):
            if known:
                tab, _, taken, held = op.reserve_held(tab, [length], [8], rows, taken, held)
            else:
                tab, _, taken = op.reserve(tab, [length], [8], rows, taken)
        kept = len(set(tab[tab >= 0].tolist()))
        assert (taken == kept) if known else (taken > 5 * kept)


def test_null_context_and_cache():
    import __graft_entry__ as g
    g.build()
    from paper_2609_09338_gb300 import binding as ob
    P, kv = ctypes.c_void_p(256), ctypes.byref(ob.osprey_kv())
    for ctx, c in ((None, kv), (P, None)):
        assert ob._c_kv_reserve_held(ctx, c, 1, P, None, 1, P, 1, P, P, P, None, None) == -1


def test_held_has_to_fit():
    torch = pytest.importorskip("torch")
    import __graft_entry__ as g
    g.build()
    from paper_2609_09338_gb300 import binding as ob
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    pages = torch.zeros((1, 3, 2, 16, 64), dtype=torch.bfloat16)
    kv = ob.KvCache(pages, pages, i32(2, 2), i32(2))
    with pytest.raises(ValueError, match="held"):
        ob.osprey_kv_reserve(None, kv, i32(2), i32(5), i32(1), i32(1), total_rows=0, held=i32(3))
    with pytest.raises(TypeError, match="held"):
        ob.osprey_kv_reserve(None, kv, i32(2), i32(5), i32(1), i32(1), total_rows=0, held=i32(2).float())
