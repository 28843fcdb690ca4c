"""Calls of every form of the attention over the 8-bit cache at once, on streams of their own, appends to other caches and
a draft call among them: each result is what the call gives alone."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__ as g
    g.build()


def test_forms_side_by_side():
    import kv8_cases as kc
    import test_kv8_gpu as t8
    from paper_2609_09338_gb300 import binding as ob
    from paper_2609_09338_gb300 import synthetic as syn
    from paper_2609_09338_gb300.binding import to_device_bf16
    from paper_2609_09338_gb300.session import Kv8DraftSession
    from paper_2609_09338_gb300.workloads import TINY
    gen = torch.Generator(device="cuda").manual_seed(1)
    calls = []
    for hd, R, dtype, rotate in ((64, 2, F32, False), (128, 1, BF, False), (64, 3, BF, True), (128, 12, BF, False),
                                 (64, 5, BF, True), (128, 2, F32, True)):
        ctx = kc.make_ctx(8, 2, hd)
        lens = [int(x) for x in torch.randint(max(R, 20), 3000, (12,), generator=gen, device="cuda")]
        kv, st = t8._cache(ctx, 12, 200, hd + R)
        t8._fill(ctx, kv, st, lens, gen)
        q = kc.rows(gen, (12, R, 8, hd), dtype)
        n = t8._ints([R] * 12)
        calls.append((ctx, kv, n, q, st, rotate))
    ctx = calls[0][0]
    grow, gst = t8._cache(ctx, 4, 200, 9)
    rows = [kc.rows(gen, (1, 100, 2, 64), BF) for _ in range(2)]
    cnt = t8._ints([25] * 4)
    # a draft call: tensor-core projections with TMEM of their own between attention launches
    B, K = 8, 4
    dctx = np.arange(100, 100 + B, dtype=np.int32) * 3
    pre = syn.make_kv_prefix(TINY, dctx, K + 1, 6)
    sess = Kv8DraftSession(TINY, syn.make_weights(TINY, 5), pre["page_table"], pre["n_pages"], K, 1)
    sess.append(dctx, pre["k_rows"], pre["v_rows"])
    di = syn.make_draft_inputs(TINY, B, 1, K, 7)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    buf = sess.draft_buffers(with_logits=True)
    args = (dev(di["n_new"]), dev(di["tokens"]), to_device_bf16(di["feats"]), 1.0, dev(di["u_draft"]), buf)
    length = sess.kv.seq_len.clone()

    def draft(stream):
        with torch.cuda.stream(stream):
            sess.kv.seq_len.copy_(length)
            sess.draft(*args)

    want = []
    for ctx_, kv, n, q, st, rotate in calls:
        o = torch.zeros_like(q)
        ob.osprey_kv8_attend(ctx_, kv, 0, n, q, o, st, rotate=rotate)
        want.append(o)
    draft(torch.cuda.current_stream())
    torch.cuda.synchronize()
    logits = buf["draft_logits"].clone()
    buf["draft_logits"].zero_()
    streams = [torch.cuda.Stream() for _ in range(len(calls) + 2)]
    outs = [[torch.zeros_like(w) for _ in range(8)] for w in want]
    torch.cuda.synchronize()
    for i in range(8):
        for j, (ctx_, kv, n, q, st, rotate) in enumerate(calls):
            ob.osprey_kv8_attend(ctx_, kv, 0, n, q, outs[j][i], st, rotate=rotate, stream=streams[j])
        ob.osprey_kv8_append(ctx, grow, cnt, *rows, gst, stream=streams[-2])
        draft(streams[-1])
    torch.cuda.synchronize()
    assert all(int(c[4].item()) == 0 for c in calls) and int(gst.item()) == 0 and int(sess.status.item()) == 0
    for w, os_ in zip(want, outs):
        assert all(torch.equal(o, w) for o in os_)
    assert torch.equal(buf["draft_logits"], logits) and grow.seq_len.tolist() == [200] * 4
