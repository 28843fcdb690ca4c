"""Attention over the bf16 cache with values and scores at the ends of their range."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import pages as op  # noqa: E402

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


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("length", [200, 60000])      # one part, several
def test_scores_of_any_size(length, sign, dtype):
    """Keys along one channel: scores are one product, exact, and equal ones weigh the same however large."""
    import kv8_cases as kc
    import pages_cases as pc
    sizes = [0, 3, 8, 12, 14, 15, 16, 17, 18, 20, 30, 50, 62]
    B = len(sizes)
    c = pc.Cache(kc.make_ctx(8, 2, 64), [length] * B, 3)
    q = torch.zeros((B, 1, 8, 64), dtype=dtype, device="cuda")
    c.k.nan_to_num_(0.0).zero_()
    alike = np.arange(5, length, 7)
    for b, e in enumerate(sizes):
        x = sign * 1.375 * 2.0 ** e
        q[b, :, :, 0] = 1.625 * 2.0 ** e
        rows = torch.from_numpy(c.tab[b, :-(-length // 16)].astype(np.int64)).cuda()
        key = torch.full((len(rows) * 16,), x * (0.5 if sign > 0 else 2), device="cuda").to(BF)   # below the largest
        key[torch.from_numpy(alike).cuda()] = x
        c.k[0, rows, :, :, 0] = key.view(-1, 1, 16).expand(-1, 2, -1)
    out = pc.attend(c, [1] * B, q)
    assert int(c.status.item()) == 0
    for b, e in enumerate(sizes):
        o, spread, size = op.attend(pc.dbl(q[b]), pc.Cache.rows(c, b, c.k), pc.Cache.rows(c, b, c.v), np.ones((1, 2, length), bool))
        # products are exact; from 2^8 on the others are 2^11 and more below, and weigh nothing
        far = np.abs(pc.dbl(out[b]) - o) - pc.tolerance(dtype, o, spread, size if e < 8 else 0)
        assert (far <= 0).all(), (e, far.max())
