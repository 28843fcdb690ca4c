"""Attention over the 8-bit cache where one key takes nearly all of the weight and its value is 0: the output is what the
others' small weights make, and has to be right relative to itself."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import kv8 as o8  # noqa: E402

BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__ as g
    g.build()


def _decoded(kv, T, hd):
    """K and V [T, Hkv, hd] float64 of sequence 0 and layer 0 as attention reads them (T a multiple of 16)."""
    ids = kv.page_table[0, :T // 16].long()
    value = torch.from_numpy(o8.e4m3_decode(torch.arange(256).numpy())).cuda()
    H = kv.k8.shape[2]
    k = value[kv.k8[0, ids].long()].view(-1, H, 2, hd // 16, 8, 16).permute(0, 2, 4, 1, 3, 5).reshape(-1, 16, H, hd)
    v = value[kv.v8[0, ids].long()].view(-1, H, hd, 16).permute(0, 3, 1, 2)
    return [(x * s[0, ids].double()[:, None, :, None]).reshape(T, H, hd)
            for x, s in ((k, kv.k_scale), (v, kv.v_scale))]


def _sink_case(Hq, Hkv, hd, R, dtype, T, share, at, mean, rotate=False):
    """Queries of the last R positions.  The key at `at` takes `share` of each row's weight; its value is 0, the others'
    `mean` and deviation 1, their scores' deviation 1.  The sink lies in the slowest pair of dims."""
    import kv8_cases as kc
    from paper_2609_09338_gb300 import binding as ob
    ctx = kc.make_ctx(Hq, Hkv, hd)
    gen = torch.Generator(device="cuda").manual_seed(T + R + hd)
    tab, n = kc.table(1, T // 16 + 3, 1)
    kv = ob.alloc_kv8(ctx.shape, tab, n)
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    k, v = (kc.rows(gen, (1, T, Hkv, hd), BF) for _ in range(2))
    v += mean
    q = kc.rows(gen, (1, R, Hq, hd), dtype)
    dim = hd // 2 - 1
    q[..., dim], q[..., hd - 1] = 4.0, 0.0
    k[..., dim], k[..., hd - 1] = 0.0, 0.0
    # Sum of the others' weights: T e^(1/2)
    score = float(torch.log(torch.tensor(share / (1 - share) * T * 1.65)))
    k[0, at], v[0, at] = 0.0, 0.0
    k[0, at, :, dim] = score * hd ** 0.5 / 4.0
    ob.osprey_kv8_append(ctx, kv, torch.tensor([T], dtype=torch.int32, device="cuda"), k, v, st, rotate=False)
    out = torch.zeros_like(q)
    ob.osprey_kv8_attend(ctx, kv, 0, torch.tensor([R], dtype=torch.int32, device="cuda"), q, out, st, rotate=rotate)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    K, V = _decoded(kv, T, hd)
    qd = q[0].double()
    if rotate:
        qd = torch.from_numpy(o8.rotate_rows(qd.cpu().numpy(), T - R, kc.THETA)).cuda()
    return qd, K, V, out[0].double()


def _check(qd, K, V, got, at, dtype):
    """Errors of a weight: the score's float32 sum and exponential, d relative (2^-17 of |q| sum |k| / sqrt(hd), natural
    units, and 2^-20), of numerator and denominator: 2 d.  Planes: half their last step, 2^-26 (float32 queries: 2^-34)
    of the reference that the key's tile goes by, which is the sink's for at most two tiles, 255 others, and no more than
    the largest of the others' weights elsewhere.  Sums: a float32 rounding a tile.  Then the output's rounding."""
    R, Hq, hd = qd.shape
    T, H, _ = K.shape
    G = Hq // H
    step = 2.0 ** -34 if dtype is F32 else 2.0 ** -26
    worst = 0.0
    for h in range(H):
        a = float(qd[:, h * G:(h + 1) * G].abs().max() * K[:, h].abs().sum(1).max()) / hd ** 0.5
        d = 2.0 ** -17 * a + 2.0 ** -20 + T / 128 * 2.0 ** -24
        for j in range(R):
            n = T - R + j + 1
            s = K[:n, h] @ qd[j, h * G:(h + 1) * G].T / hd ** 0.5
            w = torch.softmax(s, 0)                                    # [n, G]
            want, size = w.T @ V[:n, h], w.T @ V[:n, h].abs()
            rest = w.clone()
            rest[at] = 0
            planes = step * (255 * w[at] + n * rest.max(0).values)[:, None] * V[:n, h].abs().max(0).values
            tol = 2 * d * size + planes + (2.0 ** -8 if dtype is BF else 2.0 ** -23) * want.abs()
            err = (got[j, h * G:(h + 1) * G] - want).abs()
            worst = max(worst, float((err / tol).max()))
    assert worst <= 1, worst


# queries a unit: 4, 8, 16 to 32 and more (kernels of their own), and float32
@pytest.mark.parametrize("R,dtype", [(1, BF), (2, BF), (6, BF), (20, BF), (1, F32), (2, F32), (5, F32)])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("mean", [0.0, 0.5])
def test_a_key_of_most_weight_and_no_value(R, dtype, hd, mean):
    _check(*_sink_case(8, 2, hd, R, dtype, 16384 + 256, 0.99, 0, mean), 0, dtype)


@pytest.mark.parametrize("R,dtype", [(1, BF), (6, BF), (20, BF), (1, F32)])
def test_in_the_middle_of_a_long_context(R, dtype):
    T, at = 1 << 19, 200000
    _check(*_sink_case(4, 1, 64, R, dtype, T, 0.99, at, 0.5), at, dtype)


@pytest.mark.parametrize("R", [1, 6, 20])
def test_rotated_queries(R):
    qd, K, V, got = _sink_case(8, 2, 128, R, BF, 8192, 0.99, 3, 0.5, rotate=True)
    _check(qd, K, V, got, 3, BF)


@pytest.mark.parametrize("R,dtype", [(1, BF), (6, BF), (20, BF), (1, F32)])
def test_weight_that_falls_step_by_step(R, dtype):
    """Scores that fall by 30 from the first tile to the last and values that grow from 0: each tile's weights are far
    below the tile's before, and the sums are those of the first."""
    import kv8_cases as kc
    from paper_2609_09338_gb300 import binding as ob
    T, hd, Hq, Hkv = 4096, 128, 8, 2
    ctx = kc.make_ctx(Hq, Hkv, hd)
    gen = torch.Generator(device="cuda").manual_seed(R)
    tab, n = kc.table(1, T // 16 + 3, 1)
    kv = ob.alloc_kv8(ctx.shape, tab, n)
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    k, v = (kc.rows(gen, (1, T, Hkv, hd), BF) for _ in range(2))
    q = kc.rows(gen, (1, R, Hq, hd), dtype)
    q[..., 0] = 4.0
    k[0, :, :, 0] = (torch.linspace(15, -15, T, device="cuda") * hd ** 0.5 / 4.0)[:, None].to(BF)
    v[0, :, :, :8] = (torch.linspace(0, 1, T, device="cuda") ** 4)[:, None, None].to(BF)
    ob.osprey_kv8_append(ctx, kv, torch.tensor([T], dtype=torch.int32, device="cuda"), k, v, st, rotate=False)
    out = torch.zeros_like(q)
    ob.osprey_kv8_attend(ctx, kv, 0, torch.tensor([R], dtype=torch.int32, device="cuda"), q, out, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    K, V = _decoded(kv, T, hd)
    qd, got = q[0].double(), out[0].double()
    for h in range(Hkv):
        a = float(qd.abs().max() * K[:, h].abs().sum(1).max()) / hd ** 0.5
        for j in range(R):
            m = T - R + j + 1
            w = torch.softmax(K[:m, h] @ qd[j, h * 4:h * 4 + 4].T / hd ** 0.5, 0)
            want, size = w.T @ V[:m, h], w.T @ V[:m, h].abs()
            # planes: half a step of the largest weight of the 17 tiles before (a reference may be that old)
            top = torch.nn.functional.max_pool1d(torch.nn.functional.pad(w.T[None], (17 * 128 + 127, 0)), 17 * 128 + 128, 1)[0]
            planes = (2.0 ** -34 if dtype is F32 else 2.0 ** -26) * (top @ V[:m, h].abs())
            tol = 2 * (2.0 ** -17 * a + 2.0 ** -19) * size + planes + (2.0 ** -8 if dtype is BF else 2.0 ** -23) * want.abs()
            assert ((got[j, h * 4:h * 4 + 4] - want).abs() <= tol).all(), (h, j)
