"""A page id out of range clears every output row of its sequence, those of tiles that end before the page too."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__ as g
    g.build()


@pytest.mark.parametrize("rows,dtype", [(8, BF), (200, BF), (20, F32)])
@pytest.mark.parametrize("page", [0, 5, 15])
def test_all_rows_of_the_sequence_are_zero(rows, dtype, page):
    """256 positions: rows 0 .. 199 of the prompt of 200 stand at 56 .. 255, so that the last page is seen by the last 16."""
    import kv8_cases as kc
    import test_kv8_gpu as t8
    from paper_2609_09338_gb300 import binding as ob
    ctx = kc.make_ctx(8, 2, 64)
    gen = torch.Generator(device="cuda").manual_seed(3)
    kv, st = t8._cache(ctx, 3, 17, 5)
    t8._fill(ctx, kv, st, [256] * 3, gen)
    q = kc.rows(gen, (3, rows, 8, 64), dtype)
    want, got = (torch.full_like(q, 9.0) for _ in range(2))
    n = torch.tensor([rows] * 3, dtype=torch.int32, device="cuda")
    ob.osprey_kv8_attend(ctx, kv, 0, n, q, want, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    for bad in (-1, kv.n_pages):
        kv.page_table[1, page] = bad
        ob.osprey_kv8_attend(ctx, kv, 0, n, q, got, st)
        torch.cuda.synchronize()
        assert int(st.item()) == -4
        st.zero_()
        assert not got[1].any() and torch.equal(got[0], want[0]) and torch.equal(got[2], want[2])
    # an id behind the finished pages is not read
    kv.page_table[1, page] = kv.page_table[1, 16]
    kv.page_table[1, 16] = -1
    ob.osprey_kv8_attend(ctx, kv, 0, n, q, got, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
