"""The cache operators one after another, each step held to what one rounding allows: turned keys to half a step of bf16,
codes to those of the rows cached, attention to its planes over what the cache holds.  Page tables far wider than the
sequences, whose calls are cut into clusters with nothing to do, among them."""
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


def _bf16(x):
    return torch.from_numpy(x).to(F32).to(BF).double().numpy()


def _rounded_once(got, raw, first, theta):
    """Each value of got is the bf16 next to the turned row, whose float32 turn is off by 2^-22 of its pair's magnitudes
    (angle, cosine and sine 2^-24 each, two products and a sum): never a step further."""
    want = o8.rotate_rows(raw, first, theta)
    half = raw.shape[-1] // 2
    off = 2.0 ** -22 * np.tile(np.abs(raw[..., :half]) + np.abs(raw[..., half:]), 2)
    assert ((_bf16(want - off) <= got) & (got <= _bf16(want + off))).all()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("eight", [False, True])
def test_turned_keys_are_rounded_once(hd, dtype, eight):
    import kv8_cases as kc
    from paper_2609_09338_gb300 import binding as ob
    ctx = kc.make_ctx(8, 4, hd)
    gen = torch.Generator(device="cuda").manual_seed(hd)
    tab, n_pages = kc.table(3, 300, 2)
    kv = ob.alloc_kv8(ctx.shape, tab, n_pages, tail_pages=8) if eight else ob.alloc_kv(ctx.shape, tab, n_pages)
    start, n = np.array([0, 1000, 4700]), [40, 17, 100]
    kv.seq_len.copy_(torch.from_numpy(start.astype(np.int32)))
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    k, v = (kc.rows(gen, (1, sum(n), 4, hd), dtype) for _ in range(2))
    call = ob.osprey_kv8_append if eight else ob.osprey_kv_append_rope
    call(ctx, kv, torch.tensor(n, dtype=torch.int32, device="cuda"), k, v, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    r = 0
    for b, m in enumerate(n):
        pos = np.arange(start[b], start[b] + m)
        if eight:
            kc_, vc_ = (t.double().cpu().numpy()[0][b * 8 + pos // 16 % 8, :, pos % 16] for t in (kv.k_tail, kv.v_tail))
        else:
            kc_, vc_ = (t.double().cpu().numpy()[0][tab[b][pos // 16], :, pos % 16] for t in (kv.k_pages, kv.v_pages))
        _rounded_once(kc_, k[0, r:r + m].double().cpu().numpy(), int(start[b]), kc.THETA)
        np.testing.assert_array_equal(vc_, v[0, r:r + m].to(BF).double().cpu().numpy())
        r += m


@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("rows", [1, 3])
@pytest.mark.parametrize("width", [8, 8192])
def test_decoding(graph, rows, width):
    """A prompt, then `rows` positions at a time: append with the rotation, attend with turned queries."""
    import kv8_cases as kc
    import test_kv8_gpu as t8
    import test_kv8_rotated_gpu as tr
    from paper_2609_09338_gb300 import binding as ob
    Hq, H, hd, B = 8, 2, 128, 3
    ctx = kc.make_ctx(Hq, H, hd)
    gen = torch.Generator(device="cuda").manual_seed(rows)
    kv, st = t8._cache(ctx, B, width, 5)
    lens = np.array([30, 1, 63])
    T = kv.tail_pages
    model = kc.Model(1, B)

    def take(at, n):
        """Rows at .. at + n - 1 of every sequence as the tail holds them, into the model."""
        tails = [t.double().cpu().numpy()[0] for t in (kv.k_tail, kv.v_tail)]
        for b in range(B):
            for x, t in zip((model.k, model.v), tails):
                x[0][b] += [t[b * T + p // 16 % T, :, p % 16] for p in range(at[b], at[b] + n[b])]

    at = np.zeros(B, int)     # the prompt, no more rows at a time than the tail keeps
    while (at < lens).any():
        n = np.minimum(lens - at, 16)
        k, v = (kc.rows(gen, (1, int(n.sum()), H, hd), BF) for _ in range(2))
        ob.osprey_kv8_append(ctx, kv, t8._ints(n.tolist()), k, v, st)
        torch.cuda.synchronize()
        take(at, n)
        r = 0
        for b in range(B):
            if n[b]:
                _rounded_once(np.array(model.k[0][b][at[b]:]), k[0, r:r + n[b]].double().cpu().numpy(), int(at[b]), kc.THETA)
            r += n[b]
        at += n
    count = t8._ints([rows] * B)
    qkv = torch.zeros((B, rows, (Hq + 2 * H) * hd), dtype=BF, device="cuda")
    q = qkv[..., :Hq * hd].unflatten(-1, (Hq, hd))
    kn = qkv.view(B * rows, -1)[:, Hq * hd:(Hq + H) * hd].unflatten(-1, (H, hd))
    vn = qkv.view(B * rows, -1)[:, (Hq + H) * hd:].unflatten(-1, (H, hd))
    out = torch.zeros((B, rows, Hq, hd), dtype=BF, device="cuda")

    def step():
        ob.osprey_kv8_append(ctx, kv, count, kn, vn, st, layer=0)
        ob.osprey_kv8_attend(ctx, kv, 0, count, q, out, st, rotate=True)

    if graph:
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            step()
    for i in range(20):
        qkv.copy_(torch.randn(qkv.shape, generator=gen, device="cuda"))
        g.replay() if graph else step()
        torch.cuda.synchronize()
        take(lens, [rows] * B)
        for b in range(B):
            _rounded_once(np.array(model.k[0][b][lens[b]:]), kn[b * rows:(b + 1) * rows].double().cpu().numpy(),
                          int(lens[b]), kc.THETA)
            np.testing.assert_array_equal(np.array(model.v[0][b][lens[b]:]), vn[b * rows:(b + 1) * rows].double().cpu().numpy())
        lens = lens + rows
        assert int(st.item()) == 0 and kv.seq_len.tolist() == lens.tolist()
        model.check(kv, lens)
        seen = [t8._seen(torch.from_numpy(np.concatenate([np.array(x[0][b]) for b in range(B)])), lens) for x in (model.k, model.v)]
        tr._check(q, out, [rows] * B, lens, *seen, BF)


@pytest.mark.parametrize("R,dtype", [(1, BF), (2, BF), (6, BF), (20, BF), (1, F32), (5, F32)])
@pytest.mark.parametrize("rotate", [False, True])
def test_page_tables_wider_than_the_sequences(R, dtype, rotate):
    """Room for 131072 positions, at most 2100 of them held: most of a cluster's blocks have no page, or one."""
    import kv8_cases as kc
    import test_kv8_gpu as t8
    import test_kv8_rotated_gpu as tr
    from paper_2609_09338_gb300 import binding as ob
    ctx = kc.make_ctx(8, 2, 128)
    gen = torch.Generator(device="cuda").manual_seed(R)
    lens = [R, 16 + R, 140, 700, 2100]
    n = [R, R, max(1, R - 1), R, R]
    B = len(lens)
    tab, n_pages = kc.table(B, 140, 5)
    wide = np.full((B, 8192), -1, np.int32)      # behind the sequences: no page
    wide[:, :140] = tab
    kv = ob.alloc_kv8(ctx.shape, wide, n_pages)
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    k, v = t8._fill(ctx, kv, st, lens, gen)
    q = kc.rows(gen, (B, R, 8, 128), dtype)
    out = torch.full_like(q, 9.0)
    ob.osprey_kv8_attend(ctx, kv, 0, t8._ints(n), q, out, st, rotate=rotate)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    ks, vs = t8._seen(k[0], lens), t8._seen(v[0], lens)
    if rotate:
        tr._check(q, out, n, lens, ks, vs, dtype)
        assert all((out[b, m:] == 9).all() for b, m in enumerate(n))
    else:
        t8._check(q, out, n, lens, ks, vs, dtype, 9.0)
