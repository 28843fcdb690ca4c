"""Attention over blocks whose scales appending makes at the ends of bf16's range."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__ as g
    g.build()


@pytest.mark.parametrize("k_exp,v_exp", [(0, 100), (0, 60), (0, -45), (0, -80), (80, 0), (-80, 0), (90, 90), (-90, -30)])
@pytest.mark.parametrize("R,dtype", [(1, BF), (3, BF), (12, BF), (1, F32)])
def test_keys_and_values_of_any_size(k_exp, v_exp, R, dtype):
    """Keys 2^k_exp and queries 2^-k_exp of the usual, so that scores are the usual ones; values 2^v_exp.

    Blocks of scale under 2^-60 (values of 2^-80) have weights in steps of their own: half a step is 2^-26 of the largest
    weight times 2^-60, a code at most 448, and the largest weight at most 2^7 of the mean here (scores of deviation 1, 2048
    keys): 2^(-26 - 60 + 9 + 7) = 2^-70, as the header says."""
    import kv8_cases as kc
    import test_kv8_gpu as t8
    from paper_2609_09338_gb300 import binding as ob
    ctx = kc.make_ctx(8, 2, 128)
    gen = torch.Generator(device="cuda").manual_seed(R)
    lens = [300, 17 + R, 2048]
    kv, st = t8._cache(ctx, 3, 130, 5)
    k, v = (kc.rows(gen, (1, sum(lens), 2, 128), BF) for _ in range(2))
    k *= 2.0 ** k_exp
    v *= 2.0 ** v_exp
    ob.osprey_kv8_append(ctx, kv, t8._ints(lens), k, v, st, rotate=False)
    q = kc.rows(gen, (3, R, 8, 128), dtype) * 2.0 ** -k_exp
    out = torch.zeros_like(q)
    ob.osprey_kv8_attend(ctx, kv, 0, t8._ints([R] * 3), q, out, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    if v_exp == -80:
        want = t8._seen(v[0], lens)
        for b, T in enumerate(lens):
            w = t8.o8.attend(t8._dbl(q[b]), t8._seen(k[0], lens)[b], want[b])
            assert (abs(t8._dbl(out[b]) - w) <= 2.0 ** -70).all()
        return
    t8._check(q, out, [R] * 3, lens, t8._seen(k[0], lens), t8._seen(v[0], lens), dtype, 0.0)
    # the same numbers with the sizes taken out: everything is a power of two apart
    kv2, _ = t8._cache(ctx, 3, 130, 5)
    ob.osprey_kv8_append(ctx, kv2, t8._ints(lens), k * 2.0 ** -k_exp, v * 2.0 ** -v_exp, st, rotate=False)
    plain = torch.zeros_like(q)
    ob.osprey_kv8_attend(ctx, kv2, 0, t8._ints([R] * 3), q * 2.0 ** k_exp, plain, st)
    torch.cuda.synchronize()
    got, want = out.double() * 2.0 ** -v_exp, plain.double()
    # scores differ by the order of their scalings' roundings: 2^-20 of a weight, then the output's rounding on each side
    tol = 2.0 ** -18 * max(float(x.abs().max()) for x in v.double() * 2.0 ** -v_exp) + (2.0 ** -7 if dtype is BF else 2.0 ** -22) * want.abs()
    assert ((got - want).abs() <= tol).all()


@pytest.mark.parametrize("R,dtype", [(1, BF), (12, BF), (1, F32)])
def test_a_block_of_huge_values_beside_others(R, dtype):
    """One page's values are 2^100: outputs go by it, and stay right relative to it."""
    import kv8_cases as kc
    import test_kv8_gpu as t8
    from paper_2609_09338_gb300 import binding as ob
    ctx = kc.make_ctx(8, 2, 64)
    gen = torch.Generator(device="cuda").manual_seed(R)
    kv, st = t8._cache(ctx, 1, 40, 5)
    k, v = (kc.rows(gen, (1, 500, 2, 64), BF) for _ in range(2))
    v[0, 160:176] *= 2.0 ** 100
    ob.osprey_kv8_append(ctx, kv, t8._ints([500]), k, v, st, rotate=False)
    q = kc.rows(gen, (1, R, 8, 64), dtype)
    out = torch.zeros_like(q)
    ob.osprey_kv8_attend(ctx, kv, 0, t8._ints([R]), q, out, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    t8._check(q, out, [R], [500], t8._seen(k[0], [500]), t8._seen(v[0], [500]), dtype, 0.0)
