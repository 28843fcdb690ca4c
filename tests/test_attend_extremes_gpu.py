"""Attention over the bf16 cache with values and scores at the ends of their range."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__ as g
    g.build()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("lists", [False, True])
def test_infinite_values_that_every_row_sees(dtype, lists):
    """They are infinite in the output, with their sign: no part of a weight has another one, or is 0."""
    import kv8_cases as kc
    import pages_cases as pc
    lens, n = [300, 700, 20], [1, 3, 2]
    c = pc.Cache(kc.make_ctx(8, 2, 64), lens, 3)
    q = pc.queries(c.ctx, 3, 3, dtype, 4).contiguous()
    q[2] = 0                                           # every weight is 1: one part of three holds all of it
    for b, t, h, d, x in ((0, 7, 0, 5, "inf"), (0, 200, 1, 9, "-inf"), (1, 0, 0, 0, "inf"), (1, 690, 1, 63, "-inf"), (2, 3, 0, 1, "inf")):
        c.v[0, c.tab[b, t // 16], h, t % 16, d] = float(x)
    pages = None
    if lists:
        pages = pc.ints([[[list(range(44)) if (lens[b] - n[b] + min(j, n[b] - 1)) // 16 >= 43 else
                           list(range((lens[b] - n[b] + min(j, n[b] - 1)) // 16 + 1)) +
                           [-1] * (43 - (lens[b] - n[b] + min(j, n[b] - 1)) // 16)] * 2 for j in range(3)] for b in range(3)])
    got = pc.dbl(pc.attend(c, n, q, pages=pages))
    assert int(c.status.item()) == 0
    for b, h, d, x in ((0, 0, 5, np.inf), (0, 1, 9, -np.inf), (1, 0, 0, np.inf), (1, 1, 63, -np.inf), (2, 0, 1, np.inf)):
        assert (got[b, :n[b], 4 * h:4 * h + 4, d] == x).all(), (b, h, d)
        got[b, :n[b], 4 * h:4 * h + 4, d] = 0
    assert np.isfinite(got).all()
