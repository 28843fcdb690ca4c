"""Attention over the bf16 cache where a block works for seconds."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__ as g
    g.build()


def test_prompts_behind_two_million_positions():
    """Some 3e9 cycles a block, in units that both of its streams share: no wait's limit is the work's.

    The tolerance: a weight's rounding, half a step of bf16, beside a sum of weights that were not rounded (2^-8 of the mean
    magnitude of the values), an accumulator that is cut off for every 16 keys (2^17 times 2^-23 of it at most, of whatever
    sum it holds: a value's magnitude), the output's rounding (2^-8)."""
    import kv8_cases as kc
    import pages_cases as pc
    from paper_2609_09338_gb300 import binding as ob
    ctx = kc.make_ctx(8, 1, 128)
    B, R, P = 4, 65536, 1 << 17
    gen = torch.Generator(device="cuda").manual_seed(1)
    k = torch.randn((1, P, 1, 16, 128), generator=gen, device="cuda", dtype=torch.bfloat16)
    v = torch.randn((1, P, 1, 16, 128), generator=gen, device="cuda", dtype=torch.bfloat16)
    v += torch.linspace(-3, 3, 128, device="cuda").to(torch.bfloat16)       # each channel's sum is far from 0
    table = torch.randperm(P, generator=gen, device="cuda").int().expand(B, -1).contiguous()   # all read the same pages
    lens = [16 * P - 37 * b for b in range(B)]
    c = pc.Cache.__new__(pc.Cache)
    c.ctx, c.lens, c.status = ctx, lens, torch.zeros(1, dtype=torch.int32, device="cuda")
    c.kv = ob.KvCache(k, v, table, pc.ints(lens))
    q = pc.queries(ctx, B, R, torch.bfloat16, 2)
    out = pc.attend(c, [R] * B, q)
    torch.cuda.synchronize()
    assert int(c.status.item()) == 0
    rows = lambda x: x[0, table[0].long(), 0].flatten(0, 1)  # noqa: E731
    kk, vv = rows(k), rows(v)
    for b, j in ((0, 0), (0, R - 1), (1, 40000), (3, 1), (3, R - 1)):
        T = lens[b] - R + j + 1
        w = torch.softmax(q[b, j].double() @ kk[:T].double().T / 128 ** 0.5, -1)
        want = w @ vv[:T].double()
        size = w @ vv[:T].double().abs()
        far = (out[b, j].double() - want).abs() - ((2.0 ** -8 + 2.0 ** -6) * size + 2.0 ** -8 * want.abs())
        assert (far <= 0).all(), (b, j, float(far.max()))
