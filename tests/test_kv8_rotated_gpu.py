"""Attention over the 8-bit cache with queries turned on the way: every form of the kernel (4, 8, 16, 32 queries a unit,
float32, whole prompts) against float64, to what its planes hold."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import kv8 as o8  # noqa: E402

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__ as g
    g.build()


def _ints(n):
    return torch.tensor(n, dtype=torch.int32, device="cuda")


def _check(q, out, n, lens, ks, vs, dtype):
    """A turned query's planes keep 16 bits of each element in bf16 calls, 24 in float32 ones, whose turn itself is off by
    2^-22 of its pair; the score's sum 2^-20 of its magnitudes (float32, with room).  Errors d_j of the scores move an
    output by sum w_j d_j |V_j - out|, to first order (a hundredth more for the second).  A weight's planes (2^-16 or 2^-24)
    and its exponential (2^-20) are off in the numerator, the exponential in the sum too."""
    import kv8_cases as kc
    planes, turn = (2.0 ** -16, 2.0 ** -22) if dtype is BF else (2.0 ** -24, 2.0 ** -22)
    Hq, hd = q.shape[2:]
    H = ks[0].shape[1]
    G = Hq // H
    worst = 0.0
    for b, (m, T) in enumerate(zip(n, lens)):
        if not m:
            continue
        turned = o8.rotate_rows(q[b, :m].double().cpu().numpy(), T - m, kc.THETA)
        pair = np.abs(turned).reshape(m, Hq, 2, hd // 2).sum(2)
        size = planes * np.abs(turned) + turn * np.concatenate([pair, pair], -1)
        got = out[b, :m].double().cpu().numpy()
        for j in range(m):
            t = T - m + j + 1
            for h in range(H):
                K, V = ks[b][:t, h], vs[b][:t, h]
                qq = turned[j, h * G:(h + 1) * G]
                s = K @ qq.T / np.sqrt(hd)
                w = np.exp(s - s.max(0))
                w /= w.sum(0)
                err = np.abs(K) @ (size[j, h * G:(h + 1) * G] + 2.0 ** -20 * np.abs(qq)).T / np.sqrt(hd)
                want = w.T @ V
                tol = np.stack([1.01 * (w[:, i] * err[:, i]) @ np.abs(V - want[i]) for i in range(G)])
                tol += (planes + 2.0 ** -19) * (w.T @ np.abs(V)) + (2.0 ** -8 if dtype is BF else 2.0 ** -23) * np.abs(want)
                worst = max(worst, (np.abs(got[j, h * G:(h + 1) * G] - want) / np.maximum(tol, 1e-30)).max())
    assert worst <= 1, worst


FORMS = [(1, BF), (2, BF), (5, BF), (8, BF), (17, BF), (64, BF), (200, BF), (1, F32), (2, F32), (17, F32), (100, F32)]


@pytest.mark.parametrize("R,dtype", FORMS)
@pytest.mark.parametrize("hd", [64, 128])
def test_random_rows(R, dtype, hd):
    import kv8_cases as kc
    import test_kv8_gpu as t8
    from paper_2609_09338_gb300 import binding as ob
    ctx = kc.make_ctx(8, 2, hd)
    gen = torch.Generator(device="cuda").manual_seed(R + hd)
    lens, n = [R + 300, R, R + 37, 500], [R, R, max(1, R // 2), 0]
    kv, st = t8._cache(ctx, 4, 40, 5)
    k, v = t8._fill(ctx, kv, st, lens, gen)
    q = kc.rows(gen, (4, R, 8, hd), dtype, width=12 * hd)
    out = torch.full((4, R, 8, hd), 9.0, dtype=dtype, device="cuda")
    ob.osprey_kv8_attend(ctx, kv, 0, _ints(n), q, out, st, rotate=True)
    torch.cuda.synchronize()
    assert int(st.item()) == 0 and (out[3] == 9).all()
    _check(q, out, n, lens, t8._seen(k[0], lens), t8._seen(v[0], lens), dtype)


@pytest.mark.parametrize("R,dtype", FORMS)
@pytest.mark.parametrize("hd", [64, 128])
def test_two_dims_decide(R, dtype, hd):
    """Queries of the first pair of dims alone, scores of tens: half of the keys read the one dim and have the value 1,
    half the other and -1.  The turned query's two numbers are nearly the same: the output is what they leave of each
    other, with nothing to average their errors."""
    import kv8_cases as kc
    import test_kv8_gpu as t8
    from paper_2609_09338_gb300 import binding as ob
    ctx = kc.make_ctx(8, 2, hd)
    gen = torch.Generator(device="cuda").manual_seed(R + hd)
    T = R + 256 + 5
    kv, st = t8._cache(ctx, 1, 40, 5)
    k = torch.zeros((1, T, 2, hd), dtype=BF, device="cuda")
    v = torch.ones_like(k)
    k[0, 0::2, :, 0] = 256.0
    k[0, 1::2, :, hd // 2] = 256.0
    v[0, 1::2] = -1.0
    ob.osprey_kv8_append(ctx, kv, _ints([T]), k, v, st, rotate=False)
    q = torch.zeros((1, R, 8, hd), device="cuda")
    size = 1 + torch.rand((1, R, 8), generator=gen, device="cuda")
    angle = torch.pi / 4 + 0.02 * (torch.rand((1, R, 8), generator=gen, device="cuda") - 0.5)
    angle = angle - torch.arange(T - R, T, device="cuda")[None, :, None]
    q[..., 0], q[..., hd // 2] = size * torch.cos(angle), size * torch.sin(angle)
    q = q.to(dtype)
    out = torch.zeros_like(q)
    ob.osprey_kv8_attend(ctx, kv, 0, _ints([R]), q, out, st, rotate=True)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    _check(q, out, [R], [T], t8._seen(k[0], [T]), t8._seen(v[0], [T]), dtype)


@pytest.mark.parametrize("R", [1, 2, 5, 17])
@pytest.mark.parametrize("rotate", [False, True])
def test_elements_of_unlike_sizes(R, rotate):
    """Queries whose elements lie between their largest and 2^-20 of it, keys that even them out."""
    import kv8_cases as kc
    import test_kv8_gpu as t8
    from paper_2609_09338_gb300 import binding as ob
    hd, T = 128, 300
    ctx = kc.make_ctx(8, 2, hd)
    gen = torch.Generator(device="cuda").manual_seed(R)
    kv, st = t8._cache(ctx, 1, 40, 5)
    size = torch.exp2(-20 * torch.arange(hd // 2, device="cuda") / (hd // 2))
    size = torch.cat([size, size])
    k, v = (kc.rows(gen, (1, T, 2, hd), BF) for _ in range(2))
    ob.osprey_kv8_append(ctx, kv, _ints([T]), k, v, st, rotate=False)
    q = (kc.rows(gen, (1, R, 8, hd), F32) * size * 4).to(BF)
    out = torch.zeros_like(q)
    ob.osprey_kv8_attend(ctx, kv, 0, _ints([R]), q, out, st, rotate=rotate)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    ks, vs = t8._seen(k[0], [T]), t8._seen(v[0], [T])
    if rotate:
        _check(q, out, [R], [T], ks, vs, BF)
    else:   # exact, or 2^-21 of the row's largest element for those under 2^-13 of it
        qd, got = q[0].double().cpu().numpy(), out[0].double().cpu().numpy()
        want = o8.attend(qd, ks[0], vs[0])
        a = np.abs(ks[0]).sum(2).max() * np.abs(qd).max() / np.sqrt(hd)
        tol = 2 * (2.0 ** -20 * a + 2.0 ** -16 + 2.0 ** -20) * np.abs(vs[0]).max() + 2.0 ** -8 * np.abs(want)
        assert (np.abs(got - want) <= tol).all()
