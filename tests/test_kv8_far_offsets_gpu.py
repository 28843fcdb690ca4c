"""Caches whose tensors pass 2^32 bytes and 2^31 elements: pages and ring pages at their far ends hold what near ones do."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__ as g
    g.build()


def test_pages_beyond_32_bits():
    import kv8_cases as kc
    import test_kv8_gpu as t8
    from paper_2609_09338_gb300 import binding as ob
    H, hd, B, n_pages, tail = 8, 128, 4, 280000, 70000
    assert n_pages * H * 16 * hd > 1 << 32 and (B - 1) * tail * H * 16 * hd > 1 << 31
    ctx = kc.make_ctx(16, H, hd)
    gen = torch.Generator(device="cuda").manual_seed(1)
    lens = [40, 16, 1, 300]
    near = np.arange(B * 20, dtype=np.int32).reshape(B, 20)
    far = near + (n_pages - B * 20)
    k, v = (kc.rows(gen, (1, sum(lens), H, hd), BF) for _ in range(2))
    q = kc.rows(gen, (B, 3, 16, hd), BF)
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = []
    for tab, pages, ring in ((near, B * 20, 2), (far, n_pages, tail)):
        kv = ob.alloc_kv8(ctx.shape, tab, pages, ring)
        ob.osprey_kv8_append(ctx, kv, t8._ints(lens), k, v, st)
        out = torch.zeros_like(q)
        ob.osprey_kv8_attend(ctx, kv, 0, t8._ints([3, 2, 1, 3]), q, out, st, rotate=True)
        torch.cuda.synchronize()
        ids = torch.from_numpy(tab.astype(np.int64)).cuda()
        last = [(n - 1) // 16 for n in lens]
        rings = [b * ring + p % ring for b, p in enumerate(last)]
        got.append([x[0, ids].clone() for x in (kv.k8, kv.v8, kv.k_scale, kv.v_scale)] +
                   [x[0, rings].clone() for x in (kv.k_tail, kv.v_tail)] + [out])
        if ring == tail:   # nothing has been written elsewhere
            assert not kv.k8[0, :n_pages - B * 20].any() and int((kv.k_scale != 1).sum()) <= 8 * sum(n // 16 for n in lens)
        del kv
    assert int(st.item()) == 0 and got[0][-1].any()
    assert all(torch.equal(a, b) for a, b in zip(*got))
    del got
    torch.cuda.empty_cache()
    got = []
    for tab, pages in ((near, B * 20), (far, n_pages)):
        kv = ob.alloc_kv(ctx.shape, tab, pages)
        ob.osprey_kv_append_rope(ctx, kv, t8._ints(lens), k, v, st)
        ids = torch.from_numpy(tab.astype(np.int64)).cuda()
        got.append([kv.k_pages[0, ids].clone(), kv.v_pages[0, ids].clone()])
        del kv
        torch.cuda.empty_cache()
    torch.cuda.synchronize()
    assert int(st.item()) == 0 and all(torch.equal(a, b) and a.any() for a, b in zip(*got))
