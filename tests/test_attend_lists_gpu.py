"""Lists of pages that are none where a row has fewer pages than a list has entries."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__ as g
    g.build()


def _call(S, dtype=BF):
    import kv8_cases as kc
    import pages_cases as pc
    ctx = kc.make_ctx(4, 2, 64)
    lens, n = [11, 300, 32, 17], [1, 2, 2, 1]           # rows that see 1, 18 and 19, 2, 2 pages
    c = pc.Cache(ctx, lens, 7)
    q = pc.queries(ctx, 4, 2, dtype, 5)
    pages = np.full((4, 2, 2, S), -1, np.int32)
    for b, m in enumerate(n):
        for j in range(m):
            have = min(S, (lens[b] - m + j) // 16 + 1)
            pages[b, j, :, :have] = np.arange(have)
    pages = torch.from_numpy(pages).cuda()
    want = pc.attend(c, n, q, pages=pages)
    assert int(c.status.item()) == 0
    pc.check(c, want, n, q, pages=pages.cpu().numpy())
    return c, n, q, pages, want


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("b,j,h,wrong", [
    (0, 0, 1, [0, 3]),                  # a page past the row's own
    (0, 0, 0, [0, 0]), (0, 0, 0, [-1, 0]), (0, 0, 1, [0, -2]), (0, 0, 1, [0, 1 << 30]),
    (2, 0, 0, [0, 1, 1]), (2, 1, 1, [0, -1, 1]), (2, 0, 1, [0, 1, 2]), (3, 0, 0, [0, 1, -1, -1, -1, 0]),
    (3, 0, 0, [-1, -1, 0]), (1, 1, 0, list(range(20)))])
def test_entries_behind_the_rows_pages(b, j, h, wrong, dtype):
    import pages_cases as pc
    c, n, q, pages, want = _call(23, dtype)
    pages[b, j, h] = pc.ints(wrong + [-1] * (23 - len(wrong)))
    got = pc.attend(c, n, q, pages=pages)
    assert int(c.status.item()) == -1
    assert (got[b, :n[b]] == 0).all() and (got[b, n[b]:] == 77).all()
    for x in range(4):
        assert x == b or torch.equal(got[x], want[x])


@pytest.mark.parametrize("S,at", [(65536, 65535), (65536, 40000), (33, 32), (34, 2), (40, 34)])
def test_an_entry_far_behind(S, at):
    import pages_cases as pc
    c, n, q, pages, want = _call(S)
    pages[3, 0, 1, at] = 1
    got = pc.attend(c, n, q, pages=pages)
    assert int(c.status.item()) == -1 and (got[3, :1] == 0).all()
    for x in range(3):
        assert torch.equal(got[x], want[x])
    # a row that is none of the sequence's is not read
    pages[3, 0, 1, at], pages[3, 1, 0, at] = -1, 1
    c.status.zero_()
    assert torch.equal(pc.attend(c, n, q, pages=pages), want) and int(c.status.item()) == 0
