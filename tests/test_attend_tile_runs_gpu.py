"""Attention over the bf16 cache where a block's stretch of a unit is longer than a run of tiles (16384 keys; float32
queries: 128), whose outputs are added up in float32."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__ as g
    g.build()


class _Alike:
    """B sequences that all read the same pages, of lengths of their own."""

    def __init__(self, Hq, Hkv, hd, lens, seed):
        import kv8_cases as kc
        import pages_cases as pc
        from paper_2609_09338_gb300 import binding as ob
        one = pc.Cache(kc.make_ctx(Hq, Hkv, hd), [max(lens)], seed)
        self.__dict__.update(one.__dict__, lens=lens, tab=np.repeat(one.tab, len(lens), 0))
        self.kv = ob.KvCache(one.k, one.v, torch.from_numpy(self.tab).cuda(), pc.ints(lens))

    def some(self, which):
        import pages_cases as pc
        d = pc.Cache.__new__(pc.Cache)
        d.__dict__.update(self.__dict__, lens=[self.lens[b] for b in which], tab=self.tab[which])
        return d


@pytest.mark.parametrize("dtype,Hq,Hkv,hd,B,R", [(BF, 8, 2, 64, 200, 1), (BF, 16, 2, 128, 200, 3), (BF, 8, 2, 64, 90, 70),
                                                 (F32, 8, 2, 64, 200, 2), (F32, 4, 2, 128, 90, 40)])
def test_lengths_around_runs(dtype, Hq, Hkv, hd, B, R):
    import pages_cases as pc
    lens = (np.array([16384, 16385, 16383, 16512, 32768, 32769, 16384 + R, 33000, 700])[np.arange(B) % 9]).tolist()
    c = _Alike(Hq, Hkv, hd, lens, 3)
    q = pc.queries(c.ctx, B, R, dtype, 4)
    out = pc.attend(c, [R] * B, q)
    assert int(c.status.item()) == 0
    which = list(range(0, 9)) + [B // 2 + 1, B - 2]
    pc.check(c.some(which), out[which], [R] * len(which), q[which], rows=[0, R // 2, R - 1])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_listed_pages_around_runs(dtype):
    import pages_cases as pc
    B, S = 90, 2100
    lens = (np.array([40000, 34001, 33600, 16384])[np.arange(B) % 4]).tolist()
    c = _Alike(8, 4, 64, lens, 3)
    q = pc.queries(c.ctx, B, 1, dtype, 4)
    rng = np.random.default_rng(1)
    pages = np.full((B, 1, 4, S), -1, np.int32)
    for b in range(B):
        have = -(-lens[b] // 16)
        for h in range(4):
            k = min(have, (1024, 1025, 2048, 2100)[h])
            pages[b, 0, h, :k] = np.sort(rng.permutation(have)[:k])
    out = pc.attend(c, [1] * B, q, pages=torch.from_numpy(pages).cuda())
    assert int(c.status.item()) == 0
    which = [0, 1, 2, 3, 45, 89]
    pc.check(c.some(which), out[which], [1] * 6, q[which], pages=pages[which])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_runs_without_a_finite_score_and_values_that_are_not_finite(dtype):
    """A first run of scores of -inf (float32 queries: -4e36, their planes give NaN for an infinite key) leaves
    nothing behind; a value that is not finite in one of several runs, and the largest score in the last of them."""
    import pages_cases as pc
    from oracle import pages as op
    B, T = 200, 36000
    c = _Alike(8, 2, 64, [T] * B, 3)
    q = pc.queries(c.ctx, B, 1, dtype, 4).contiguous()
    page = lambda t: torch.from_numpy(c.tab[0, t // 16].astype(np.int64)).cuda()  # noqa: E731
    early = np.arange(0, 17008, 16)
    q[..., 0] = 1
    c.k[0, page(early), 0, :, 0] = float("-inf") if dtype == BF else -3e37                # KV head 0: 17008 keys
    c.v[0, int(c.tab[0, 20000 // 16]), 1, 20000 % 16, 5] = float("inf")   # KV head 1: one value, and a key like the query
    last = (35000 // 16, 35000 % 16)
    c.k[0, int(c.tab[0, last[0]]), 1, last[1]] = 2.0
    q[:, :, 4:] = q[:, :, 4:].abs()
    out = pc.attend(c, [1] * B, q)
    assert int(c.status.item()) == 0
    for b in (0, 7, 101, 199):
        k, v, x = pc.Cache.rows(c, b, c.k), pc.Cache.rows(c, b, c.v), pc.dbl(q[b])
        see = np.ones((1, 2, T), bool)
        see[:, 0, :17008] = False
        inf = np.isinf(v[:, 1, 5])
        assert inf.sum() == 1
        v[inf, 1, 5] = 0
        k[:17008, 0, 0] = 0                                             # (not seen there)
        o, spread, size = op.attend(x, k, v, see)
        got = pc.dbl(out[b])
        assert (got[0, 4:, 5] == np.inf).all()
        got[0, 4:, 5], spread[0, 4:, 5] = o[0, 4:, 5], 1
        assert (np.abs(got - o) <= pc.tolerance(dtype, o, spread, size)).all(), b
