"""Refusals of the cache operators that the host sees, before anything is launched (no GPU)."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def ob():
    import __graft_entry__ as g
    g.build()
    from paper_2609_09338_gb300 import binding
    return binding


def test_null_context_and_cache(ob):
    p = ctypes.c_void_p(256)
    kv, kv8 = ob.osprey_kv(), ob.osprey_kv8()
    assert ob._c_kv_append_rope(None, ctypes.byref(kv), 0, 1, p, 1, p, p, 1, 0, 1, None, None) == -1
    assert ob._c_kv_append_rope(p, None, 0, 1, p, 1, p, p, 1, 0, 1, None, None) == -1
    assert ob._c_kv8_append(None, ctypes.byref(kv8), 0, 1, p, 1, p, p, 1, 0, 1, 1, None, None) == -1
    assert ob._c_kv8_attend(None, ctypes.byref(kv8), 0, 1, 1, p, p, 1, 0, 0, 1, p, None, None) == -1
    assert "null" in ob.osprey_last_error()
