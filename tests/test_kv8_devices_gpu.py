"""Tensors that lie on another device than the current one are refused by the cache operators, whichever tensor it is.
(One device: a tensor's subclass says that it lies on another.)"""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF = torch.bfloat16


class Elsewhere(torch.Tensor):
    def get_device(self):
        return 1


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__ as g
    g.build()


def _away(t):
    return t.as_subclass(Elsewhere)


FIELDS = ["k8", "v8", "k_scale", "v_scale", "k_tail", "v_tail", "page_table", "seq_len"]


def test_cache_operators_refuse_another_device():
    import kv8_cases as kc
    import test_kv8_gpu as t8
    from paper_2609_09338_gb300 import binding as ob
    ctx = kc.make_ctx(8, 4, 64)
    kv, st = t8._cache(ctx, 2, 4, 5)
    tab, n_pages = kc.table(2, 4, 5)
    bf = ob.alloc_kv(ctx.shape, tab, n_pages)
    n = t8._ints([1, 1])
    rows = torch.zeros((1, 2, 4, 64), dtype=BF, device="cuda")
    q = torch.zeros((2, 1, 8, 64), dtype=BF, device="cuda")
    good = {"n_rows": n, "k_rows": rows, "v_rows": rows, "status": st}
    for call, cache in ((ob.osprey_kv_append_rope, bf), (ob.osprey_kv8_append, kv)):
        call(ctx, cache, **good)
        for name, t in good.items():
            with pytest.raises(ValueError):
                call(ctx, cache, **{**good, name: _away(t)})
    good = {"n_rows": n, "q": q, "out": torch.zeros_like(q), "status": st}
    ob.osprey_kv8_attend(ctx, kv, 0, **good)
    for name, t in good.items():
        with pytest.raises(ValueError):
            ob.osprey_kv8_attend(ctx, kv, 0, **{**good, name: _away(t)})
    torch.cuda.synchronize()
    before = kv.seq_len.tolist(), bf.seq_len.tolist()
    for field in FIELDS:
        t = getattr(kv, field)
        setattr(kv, field, _away(t))
        with pytest.raises(ValueError):
            ob.osprey_kv8_attend(ctx, kv, 0, **good)
        with pytest.raises(ValueError):
            ob.osprey_kv8_append(ctx, kv, n, rows, rows, st)
        setattr(kv, field, t)
    for field in ("k_pages", "v_pages", "page_table", "seq_len"):
        t = getattr(bf, field)
        setattr(bf, field, _away(t))
        with pytest.raises(ValueError):
            ob.osprey_kv_append_rope(ctx, bf, n, rows, rows, st)
        setattr(bf, field, t)
    # a cache that has been checked, and another device current since
    now = torch._C._cuda_getDevice
    torch._C._cuda_getDevice = lambda: 1
    try:
        with pytest.raises(ValueError):
            kv.c_struct(ctx.shape)
    finally:
        torch._C._cuda_getDevice = now
    ob.osprey_kv8_attend(ctx, kv, 0, **good)
    torch.cuda.synchronize()
    assert (kv.seq_len.tolist(), bf.seq_len.tolist()) == before and int(st.item()) == 0
