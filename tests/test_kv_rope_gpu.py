"""osprey_kv_append_rope: rows land turned to their positions, once rounded, where the table says; its refusals."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import kv8 as o8  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__ as g
    g.build()


def _cache(ctx, B, max_pages, seed):
    import kv8_cases as kc
    from paper_2609_09338_gb300 import binding as ob
    tab, n = kc.table(B, max_pages, seed)
    return ob.alloc_kv(ctx.shape, tab, n), torch.zeros(1, dtype=torch.int32, device="cuda")


def _gathered(kv, b, n):
    """[L, n, Hkv, hd] float64 of sequence b's first n positions."""
    t = np.arange(n)
    tab = kv.page_table.cpu().numpy()[b]
    out = []
    for pages in (kv.k_pages, kv.v_pages):
        p = pages.double().cpu().numpy()
        out.append(np.moveaxis(p[:, tab[t // 16], :, t % 16], 0, 1))
    return out


@pytest.mark.parametrize("Hq,Hkv,hd,L", [(4, 2, 64, 1), (16, 8, 128, 1), (4, 1, 128, 2), (12, 3, 64, 2)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("wide", [False, True])
def test_rows_are_rotated_and_placed(Hq, Hkv, hd, L, dtype, wide):
    import kv8_cases as kc
    from paper_2609_09338_gb300 import binding as ob
    ctx = kc.make_ctx(Hq, Hkv, hd, L)
    gen = torch.Generator(device="cuda").manual_seed(hd + Hkv)
    counts = [[0, 1, 15, 16, 17, 100, 33], [5, 16, 1, 0, 40, 2, 15]]
    B = len(counts[0])
    kv, st = _cache(ctx, B, 16, 7)
    width = (Hq + 2 * Hkv) * hd if wide else None
    at = np.zeros(B, int)
    for n in counts:
        k, v = (kc.rows(gen, (L, sum(n), Hkv, hd), dtype, width) for _ in range(2))
        ob.osprey_kv_append_rope(ctx, kv, torch.tensor(n, dtype=torch.int32, device="cuda"), k, v, st)
        torch.cuda.synchronize()
        assert int(st.item()) == 0
        r = 0
        for b, m in enumerate(n):
            gk, gv = (x[:, at[b]:] for x in _gathered(kv, b, at[b] + m))
            for l in range(L):
                raw = k[l, r:r + m].double().cpu().numpy()
                want = o8.rotate_rows(raw, at[b], kc.THETA)
                # one rounding to bf16 (2^-8), and the float32 turn: angle 2^-22.3, cos and sin 2 ulp, two products
                mag = np.abs(raw[..., :hd // 2]) + np.abs(raw[..., hd // 2:])
                tol = 1.01 * 2.0 ** -8 * np.abs(want) + 2.0 ** -20 * np.concatenate([mag, mag], -1)
                assert (np.abs(gk[l] - want) <= tol).all()
                np.testing.assert_array_equal(gv[l], v[l, r:r + m].to(torch.bfloat16).double().cpu().numpy())
            r += m
        at += np.array(n)
        np.testing.assert_array_equal(kv.seq_len.cpu().numpy(), at)


def test_far_positions_keep_their_angles():
    """Position 2^20 - 20: a float32 angle would be 0.06 off."""
    import kv8_cases as kc
    from paper_2609_09338_gb300 import binding as ob
    ctx = kc.make_ctx(4, 2, 64)
    tab = np.zeros((1, 1 << 16), np.int32)
    tab[0, -2:] = [1, 2]
    kv = ob.alloc_kv(ctx.shape, tab, 3)
    L0 = (1 << 20) - 20
    kv.seq_len.fill_(L0)
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(1)
    k = kc.rows(gen, (1, 20, 2, 64), torch.float32)
    ob.osprey_kv_append_rope(ctx, kv, torch.tensor([20], dtype=torch.int32, device="cuda"), k, k, st)
    torch.cuda.synchronize()
    raw = k[0].double().cpu().numpy()
    want = o8.rotate_rows(raw, L0, kc.THETA)
    mag = np.abs(raw[..., :32]) + np.abs(raw[..., 32:])
    t = np.arange(L0, L0 + 20)
    ids = tab[0][t // 16]
    pages = kv.k_pages[0].double().cpu().numpy()
    got = pages[ids, :, t % 16]
    assert int(st.item()) == 0 and int(kv.seq_len.item()) == 1 << 20
    assert (np.abs(got - want) <= 1.01 * 2.0 ** -8 * np.abs(want) + 2.0 ** -20 * np.concatenate([mag, mag], -1)).all()


def test_one_layer_at_a_time_is_all_layers_at_once():
    import kv8_cases as kc
    from paper_2609_09338_gb300 import binding as ob
    ctx = kc.make_ctx(8, 4, 64, 3)
    gen = torch.Generator(device="cuda").manual_seed(4)
    n = torch.tensor([3, 0, 20], dtype=torch.int32, device="cuda")
    k, v = (kc.rows(gen, (3, 23, 4, 64), torch.bfloat16) for _ in range(2))
    (a, st), (b, _) = _cache(ctx, 3, 4, 2), _cache(ctx, 3, 4, 2)
    ob.osprey_kv_append_rope(ctx, a, n, k, v, st)
    for l in range(3):
        ob.osprey_kv_append_rope(ctx, b, n, k[l], v[l], st, layer=l, advance=l == 2)
        torch.cuda.synchronize()
        assert b.seq_len.tolist() == ([3, 0, 20] if l == 2 else [0, 0, 0])
    assert torch.equal(a.k_pages, b.k_pages) and torch.equal(a.v_pages, b.v_pages) and int(st.item()) == 0


@pytest.mark.parametrize("advance", [True, False])
def test_device_errors_leave_the_sequence(advance):
    import kv8_cases as kc
    from paper_2609_09338_gb300 import binding as ob
    ctx = kc.make_ctx(4, 2, 64)
    gen = torch.Generator(device="cuda").manual_seed(4)
    # sequence 1 has a page id out of range among its new pages, sequence 2 runs past its table
    for n, bad in (([20, 20, 20], "page"), ([20, 20, 65], "table")):
        kv, st = _cache(ctx, 3, 4, 2)
        if bad == "page":
            kv.page_table[1, 1] = kv.n_pages
        k = kc.rows(gen, (1, sum(n), 2, 64), torch.bfloat16)
        ob.osprey_kv_append_rope(ctx, kv, torch.tensor(n, dtype=torch.int32, device="cuda"), k, k, st, advance=advance)
        torch.cuda.synchronize()
        assert int(st.item()) == -4
        left = 1 if bad == "page" else 2
        assert kv.seq_len.tolist() == [20 if advance and b != left else 0 for b in range(3)]
        tab = kv.page_table.cpu().numpy()
        own = [p for p in tab[left] if 0 <= p < kv.n_pages]
        assert not kv.k_pages[:, own].any() and kv.k_pages[:, tab[0, :2]].any()


def test_counts_that_do_not_add_up():
    import kv8_cases as kc
    from paper_2609_09338_gb300 import binding as ob
    ctx = kc.make_ctx(4, 2, 64)
    for n in ([3, 4], [9, -1], [0, 0]):
        kv, st = _cache(ctx, 2, 4, 2)
        k = torch.ones((1, 8, 2, 64), dtype=torch.bfloat16, device="cuda")
        ob.osprey_kv_append_rope(ctx, kv, torch.tensor(n, dtype=torch.int32, device="cuda"), k, k, st, advance=False)
        torch.cuda.synchronize()
        assert int(st.item()) == -1 and not kv.k_pages.any()
