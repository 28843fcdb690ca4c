"""Positions taken back after a draft call: 16 (tail_pages - 1) of them from the last row that the call wrote, its chain's
rows among them."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2609_09338_gb300 import synthetic as syn  # noqa: E402
from paper_2609_09338_gb300.workloads import TINY  # noqa: E402

BF = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__ as g
    g.build()


@pytest.mark.parametrize("K,max_new", [(3, 1), (1, 1), (6, 4), (16, 3)])
def test_rows_taken_back_after_a_draft_call(K, max_new):
    """Lengths of every offset in a page; each goes back as far as it may, attends there, and goes on with other rows."""
    import kv8_cases as kc
    import test_kv8_gpu as t8
    from paper_2609_09338_gb300 import binding as ob
    from paper_2609_09338_gb300.binding import to_device_bf16
    from paper_2609_09338_gb300.session import Kv8DraftSession
    B = 16
    ctx = np.arange(40, 40 + B, dtype=np.int32)
    kv = syn.make_kv_prefix(TINY, ctx, 64, 6)
    sess = Kv8DraftSession(TINY, syn.make_weights(TINY, 5), kv["page_table"], kv["n_pages"], K, max_new)
    sess.append(ctx, kv["k_rows"], kv["v_rows"])
    H, hd = TINY.n_kv_heads, TINY.head_dim
    model = kc.Model(1, B)
    model.append(ctx.tolist(), *(t.double().cpu().numpy() for t in
                                 (to_device_bf16(kv["k_rows"]), to_device_bf16(kv["v_rows"]))))
    di = syn.make_draft_inputs(TINY, B, max_new, K, 7)
    di["n_new"] = np.arange(B, dtype=np.int32) % max_new + 1
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    sess.draft(dev(di["n_new"]), dev(di["tokens"]), to_device_bf16(di["feats"]), 1.0, dev(di["u_draft"]),
               sess.draft_buffers())
    torch.cuda.synchronize()
    assert int(sess.status.item()) == 0
    T = sess.kv.tail_pages
    tails = [t.double().cpu().numpy()[0] for t in (sess.kv.k_tail, sess.kv.v_tail)]
    for b in range(B):
        for j in range(di["n_new"][b]):
            p = ctx[b] + j
            for x, t in zip((model.k, model.v), tails):
                x[0][b].append(t[b * T + p // 16 % T, :, p % 16])
    back = 16 * (T - 1) - (K - 1)
    assert back >= 0 and (back > 0 or T == 1)
    lens = ctx + di["n_new"] - back
    sess.kv.seq_len.copy_(dev(lens))
    for b in range(B):
        model.k[0][b], model.v[0][b] = model.k[0][b][:lens[b]], model.v[0][b][:lens[b]]
    gen = torch.Generator(device="cuda").manual_seed(3)

    def attend():
        q = kc.rows(gen, (B, 1, TINY.n_q_heads, hd), BF)
        out = torch.full_like(q, 9.0)
        ob.osprey_kv8_attend(sess.ctx, sess.kv, 0, t8._ints([1] * B), q, out, sess.status)
        torch.cuda.synchronize()
        at = sess.kv.seq_len.tolist()
        seen = [t8._seen(torch.from_numpy(np.concatenate([np.array(x[0][b]) for b in range(B)])), at)
                for x in (model.k, model.v)]
        t8._check(q, out, [1] * B, at, *seen, BF, 9.0)

    attend()
    n = [20] * B
    k, v = (kc.rows(gen, (1, 20 * B, H, hd), BF) for _ in range(2))
    ob.osprey_kv8_append(sess.ctx, sess.kv, t8._ints(n), k, v, sess.status, rotate=False)
    model.append(n, k.double().cpu().numpy(), v.double().cpu().numpy())
    torch.cuda.synchronize()
    assert int(sess.status.item()) == 0
    attend()
    tab = sess.kv.page_table.cpu().numpy()
    from oracle import kv8 as o8
    for b in range(B):
        x = np.array(model.k[0][b])
        for p in range(len(x) // 16):
            for h in range(H):
                code, s = o8.encode_block(x[p * 16:p * 16 + 16, h])
                assert float(sess.kv.k_scale[0, tab[b, p], h]) == s
                np.testing.assert_array_equal(sess.kv.k8[0, tab[b, p], h].cpu().numpy(), o8.place_k(code))
