"""Attention over the bf16 cache where a block works for seconds."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__ as g
    g.build()


class _Long:
    """B sequences of 2^21 positions and R new rows, which all read the same pages; each channel's values are far from 0."""

    def __init__(self, B, R, dtype=torch.bfloat16):
        import kv8_cases as kc
        import pages_cases as pc
        from paper_2609_09338_gb300 import binding as ob
        ctx = kc.make_ctx(8, 1, 128)
        self.R, P = R, 1 << 17
        gen = torch.Generator(device="cuda").manual_seed(1)
        k = torch.randn((1, P, 1, 16, 128), generator=gen, device="cuda", dtype=torch.bfloat16)
        v = torch.randn((1, P, 1, 16, 128), generator=gen, device="cuda", dtype=torch.bfloat16)
        v += torch.linspace(-3, 3, 128, device="cuda").to(torch.bfloat16)
        table = torch.randperm(P, generator=gen, device="cuda").int().expand(B, -1).contiguous()
        self.lens = [16 * P - 37 * b for b in range(B)]
        c = pc.Cache.__new__(pc.Cache)
        c.ctx, c.lens, c.status = ctx, self.lens, torch.zeros(1, dtype=torch.int32, device="cuda")
        c.kv = ob.KvCache(k, v, table, pc.ints(self.lens))
        self.q = pc.queries(ctx, B, R, dtype, 2)
        self.out = pc.attend(c, [R] * B, self.q)
        torch.cuda.synchronize()
        assert int(c.status.item()) == 0
        self.k, self.v = (x[0, table[0].long(), 0].flatten(0, 1) for x in (k, v))

    def check(self, b, j):
        """A weight's rounding is half a step of bf16, beside a sum of weights that were not rounded: 2^-8 of the values' mean
        magnitude.  An accumulator is cut off for every 16 keys, 2^-23 of what it holds at most, 2^10 times between sums in
        float32; these are some 2^8.  The output's rounding is 2^-8."""
        T = self.lens[b] - self.R + j + 1
        w = torch.softmax(self.q[b, j].double() @ self.k[:T].double().T / 128 ** 0.5, -1)
        want = w @ self.v[:T].double()
        size = w @ self.v[:T].double().abs()
        far = (self.out[b, j].double() - want).abs() - ((2.0 ** -8 + 2.0 ** -13 + 2.0 ** -16) * size + 2.0 ** -8 * want.abs())
        assert (far <= 0).all(), (b, j, float(far.max()))


def test_prompts_behind_two_million_positions():
    """Some 3e9 cycles a block, in units that both of its streams share: no wait's limit is the work's."""
    x = _Long(4, 65536)
    for b, j in ((0, 0), (0, x.R - 1), (1, 40000), (3, 1), (3, x.R - 1)):
        x.check(b, j)


@pytest.mark.parametrize("B,R", [(1, 5000), (320, 1)])     # units of both streams, of one
def test_sums_over_two_million_keys_of_one_block(B, R):
    """What an accumulator cuts off does not add up: with one for all of them, sums were 1.2 % short."""
    x = _Long(B, R)
    for b, j in ((0, 0), (B - 1, R - 1), (B // 2, R // 2)):
        x.check(b, j)
