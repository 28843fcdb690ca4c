"""The draft call on the 8-bit cache against the oracle drafter, whose prefix is the cache's own rows as attention reads
them: finished pages through 8 bits, the rest bf16.  Two calls in a row, so that the first one's committed rows are read
by the second, finished pages among them."""
from dataclasses import replace

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import drafter as od  # noqa: E402
from oracle import kv8 as o8  # noqa: E402
from oracle.bf16 import widen  # noqa: E402
from paper_2609_09338_gb300 import synthetic as syn  # noqa: E402
from paper_2609_09338_gb300.workloads import TINY  # noqa: E402

LOGIT_TOL = 2e-2   # as the bf16 cache's draft tests: bf16 weights, float32 accumulation

BIG = replace(TINY, n_layers=2, n_q_heads=8, n_kv_heads=2, head_dim=128, d_model=512)


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__ as g
    g.build()


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _ring(kv, l, b, pos, name):
    """Rows at positions pos of sequence b [n, Hkv, hd], float64, from the tail."""
    t = getattr(kv, name + "_tail").double().cpu().numpy()[l]
    pos = np.asarray(pos)
    return t[b * kv.tail_pages + pos // 16 % kv.tail_pages, :, pos % 16]


@pytest.mark.parametrize("shape", [TINY, BIG], ids=["tiny", "two-layer"])
@pytest.mark.parametrize("ctx,n_new", [([128], [1]), ([15, 33], [1, 3]), ([0, 1, 30, 47, 200], [4, 16, 2, 1, 17])])
@pytest.mark.parametrize("T", [0.0, 1.0])
def test_two_calls_follow_the_oracle(shape, ctx, n_new, T):
    import kv8_cases as kc
    from paper_2609_09338_gb300.binding import to_device_bf16
    from paper_2609_09338_gb300.session import Kv8DraftSession
    K, B, max_new = 4, len(ctx), max(n_new)
    ctx = np.array(ctx, np.int32)
    w = syn.make_weights(shape, 5)
    kv = syn.make_kv_prefix(shape, ctx, 2 * max_new + K, 6)
    sess = Kv8DraftSession(shape, w, kv["page_table"], kv["n_pages"], K, max_new)
    sess.append(ctx, kv["k_rows"], kv["v_rows"])
    L = shape.n_layers
    model = kc.Model(L, B)
    model.append(ctx.tolist(), widen(kv["k_rows"]), widen(kv["v_rows"]))
    lens = ctx.copy()
    n_new = np.array(n_new, np.int32)
    for call in range(2):
        di = syn.make_draft_inputs(shape, B, max_new, K, 7 + call)
        di["n_new"] = n_new if call == 0 else n_new[::-1].copy()
        out = sess.draft_buffers(with_logits=True)
        sess.draft(_dev(di["n_new"]), _dev(di["tokens"]), to_device_bf16(di["feats"]), T, _dev(di["u_draft"]), out)
        torch.cuda.synchronize()
        assert int(sess.status.item()) == 0
        toks, logits = out["draft_tokens"].cpu().numpy(), out["draft_logits"].cpu().numpy()
        prefix = [np.stack([np.concatenate([o8.as_cached(np.array(x[l][b]).reshape(-1, shape.n_kv_heads, shape.head_dim),
                                                         lens[b]) for b in range(B)]) for l in range(L)])
                  for x in (model.k, model.v)]
        forced = []
        for b in range(B):
            pos = np.arange(lens[b], lens[b] + di["n_new"][b] + K - 1)
            forced.append([np.stack([_ring(sess.kv, l, b, pos, n) for l in range(L)]) for n in ("k", "v")])
        ref = od.draft_step(w, shape, *prefix, lens, di["tokens"], di["feats"], di["n_new"], K, T, di["u_draft"],
                            forced_tokens=toks, forced_kv=forced)
        err = np.abs(logits - ref["logits"]).max()
        assert err < LOGIT_TOL, err
        for b in range(B):
            for k in range(K):
                if T == 0.0:
                    if ref["margins"][b, k] > 2 * err:
                        assert toks[b, k] == ref["tokens"][b, k]
                else:   # the draw from the call's own logits
                    z = logits[b, k].astype(np.float64)
                    tok, margin = od.inverse_cdf(np.exp(z - z.max()), float(di["u_draft"][b, k]))
                    assert tok == toks[b, k] or margin < 1e-5
            m = di["n_new"][b]
            for l in range(L):
                model.k[l][b] += list(forced[b][0][l, :m])
                model.v[l][b] += list(forced[b][1][l, :m])
        lens = lens + di["n_new"]
        np.testing.assert_array_equal(sess.kv.seq_len.cpu().numpy(), lens)
        # what the call committed, bit for bit (the ring's last rows are the chain's by now)
        tab = sess.kv.page_table.cpu().numpy()
        for l in range(L):
            for b in range(B):
                for p in range(lens[b] // 16):
                    for h in range(shape.n_kv_heads):
                        for x, code, scale, place in ((model.k, sess.kv.k8, sess.kv.k_scale, o8.place_k),
                                                      (model.v, sess.kv.v8, sess.kv.v_scale, o8.place_v)):
                            c, s = o8.encode_block(np.array(x[l][b])[p * 16:p * 16 + 16, h])
                            assert float(scale[l, tab[b, p], h]) == s
                            np.testing.assert_array_equal(code[l, tab[b, p], h].cpu().numpy(), place(c))


def test_a_skipped_sequence_is_left_alone():
    """Sequence 1 has more new rows than the call allows, sequence 2 no page for them."""
    from paper_2609_09338_gb300.binding import to_device_bf16
    from paper_2609_09338_gb300.session import Kv8DraftSession
    K, ctx = 3, np.array([20, 40, 31, 90], np.int32)
    kv = syn.make_kv_prefix(TINY, ctx, 8, 6)
    sess = Kv8DraftSession(TINY, syn.make_weights(TINY, 5), kv["page_table"], kv["n_pages"], K, 2)
    sess.append(ctx, kv["k_rows"], kv["v_rows"])
    sess.kv.page_table[2, 2] = -1
    di = syn.make_draft_inputs(TINY, 4, 2, K, 7)
    n = np.array([1, 3, 2, 2], np.int32)
    out = sess.draft_buffers()
    before = [t.clone() for t in (sess.kv.k8, sess.kv.k_tail)]
    sess.draft(_dev(n), _dev(di["tokens"]), to_device_bf16(di["feats"]), 1.0, _dev(di["u_draft"]), out)
    torch.cuda.synchronize()
    assert int(sess.status.item()) in (-1, -4)
    assert sess.kv.seq_len.tolist() == [21, 40, 31, 92]
    t = out["draft_tokens"].cpu()
    assert (t[1:3] == -1).all() and (t[0] >= 0).all() and (t[3] >= 0).all()
    r = sess.kv.tail_pages
    assert torch.equal(sess.kv.k_tail[:, r:3 * r], before[1][:, r:3 * r])


def test_captured_and_replayed():
    from paper_2609_09338_gb300.binding import to_device_bf16
    from paper_2609_09338_gb300.session import Kv8DraftSession
    K, ctx = 3, np.array([20, 47, 31, 90], np.int32)
    kv = syn.make_kv_prefix(TINY, ctx, 8, 6)
    di = syn.make_draft_inputs(TINY, 4, 1, K, 7)
    outs = []
    for graph in (False, True):
        sess = Kv8DraftSession(TINY, syn.make_weights(TINY, 5), kv["page_table"], kv["n_pages"], K, 1)
        sess.append(ctx, kv["k_rows"], kv["v_rows"])
        out = sess.draft_buffers(with_logits=True)
        args = (_dev(di["n_new"]), _dev(di["tokens"]), to_device_bf16(di["feats"]), 1.0, _dev(di["u_draft"]), out)
        if graph:
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                sess.draft(*args)
            run = g.replay
        else:
            run = lambda: sess.draft(*args)  # noqa: E731
        got = []
        for _ in range(3):
            run()
            torch.cuda.synchronize()
            got.append({k: v.clone() for k, v in out.items()})
        outs.append((got, sess.kv.k8.clone(), sess.kv.seq_len.clone()))
        assert int(sess.status.item()) == 0
    for a, b in zip(outs[0][0], outs[1][0]):
        assert all(torch.equal(a[k], b[k]) for k in a)
    assert torch.equal(outs[0][1], outs[1][1]) and torch.equal(outs[0][2], outs[1][2])


def test_refusals():
    from paper_2609_09338_gb300 import binding as ob
    from paper_2609_09338_gb300.session import Kv8DraftSession
    kv = syn.make_kv_prefix(TINY, np.array([20], np.int32), 8, 6)
    sess = Kv8DraftSession(TINY, syn.make_weights(TINY, 5), kv["page_table"], kv["n_pages"], 4, 1)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    feats = torch.zeros((1, 16, TINY.feat_dim), dtype=torch.bfloat16, device="cuda")
    big = torch.zeros(1 << 28, dtype=torch.uint8, device="cuda")
    with pytest.raises(ob.OspreyError) as e:      # 14 + 16 + 4 rows do not fit a ring of two pages
        ob.osprey_draft_step_kv8(sess.ctx, sess.kv, i32(1), i32(1, 16), feats, 0.0, None, i32(1, 4), workspace=big,
                                 status=sess.status)
    assert e.value.code == -4
    with pytest.raises(ob.OspreyError) as e:      # the bf16 call's workspace lacks the ring's page table
        ob.osprey_draft_step_kv8(sess.ctx, sess.kv, i32(1), i32(1, 1), feats[:, :1].contiguous(), 0.0, None, i32(1, 4),
                                 workspace=sess.workspace[:-1].clone(), status=sess.status)
    assert e.value.code == -4
    assert ob.osprey_draft_kv8_workspace_bytes(sess.ctx, 1, 4, 1, 0) == 0
