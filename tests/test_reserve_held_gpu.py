"""Pages for new rows where rows are taken back: what a sequence holds behind its length stays its own."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import pages as op  # noqa: E402

BF = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__ as g
    g.build()


class _Server:
    def __init__(self, B, n_pages, max_pages, seed=0):
        import kv8_cases as kc
        import pages_cases as pc
        from paper_2609_09338_gb300 import binding as ob
        self.ob, self.pc, self.ctx = ob, pc, kc.make_ctx(4, 2, 64)
        z = torch.zeros((1, n_pages, 2, 16, 64), dtype=BF, device="cuda")
        self.kv = ob.KvCache(z, z, torch.full((B, max_pages), -1, dtype=torch.int32, device="cuda"), pc.ints([0] * B))
        self.free = np.random.default_rng(seed).permutation(n_pages).astype(np.int32)
        self.free_t = torch.from_numpy(self.free).cuda()
        self.taken, self.status, self.held = pc.ints([0]), pc.ints([0]), pc.ints([0] * B)

    def call(self, n, share=None, held=True, slots=True):
        out = torch.full((sum(n),), -99, dtype=torch.int64, device="cuda") if slots else None
        self.ob.osprey_kv_reserve(self.ctx, self.kv, self.pc.ints(n), self.free_t, self.taken, self.status,
                                  share=None if share is None else self.pc.ints(share), slots=out, total_rows=sum(n),
                                  held=self.held if held else None)
        torch.cuda.synchronize()
        return out.cpu().numpy() if slots else None

    def set(self, lens, held, table):
        self.kv.seq_len.copy_(self.pc.ints(lens))
        self.held.copy_(self.pc.ints(held))
        self.kv.page_table.copy_(torch.from_numpy(table))


@pytest.mark.parametrize("B,hi,ahead", [(1, 5, 3), (7, 40, 5), (64, 1, 2), (100, 9, 40), (200, 30, 4), (3, 9000, 600), (4096, 20, 3)])
@pytest.mark.parametrize("shares", [False, True])
def test_reserve_held(B, hi, ahead, shares):
    rng = np.random.default_rng(B + shares)
    lens, n = rng.integers(0, 200, B).tolist(), rng.integers(0, hi + 1, B).tolist()
    share = [-1] * B
    if shares:
        for b in range(1, B):
            if b % 3:
                share[b] = b - b % 3
                lens[b] = int(rng.integers(0, lens[b - b % 3] // 16 + 1)) * 16
    need = [-(-x // 16) for x in lens]
    most = max(max(-(-(a + m) // 16) for a, m in zip(lens, n)), max(need) + ahead)
    s = _Server(B, B * most + sum(-(-m // 16) + 1 for m in n) + 10, most, B)
    table = np.full((B, most), -1, np.int32)
    ids, held = s.free[-B * most:], []
    for b in range(B):
        more = int(rng.integers(0, ahead + 1))
        # behind the shared pages there are pages of its own, if any
        held.append(need[b] + more if share[b] == -1 or more else int(rng.integers(0, need[b] + 1)))
        table[b, :held[b]] = ids[b * most:b * most + held[b]]
        if share[b] != -1:
            table[b, :need[b]] = -5
    s.set(lens, held, table)
    s.taken.fill_(3)
    want = op.reserve_held(table, lens, n, s.free, 3, held, share)
    got = s.call(n, share)
    assert (s.kv.page_table.cpu().numpy() == want[0]).all() and (got == want[1]).all()
    assert int(s.taken.item()) == want[2] and s.held.tolist() == want[3] and int(s.status.item()) == 0
    # the same call again: everything is held already
    s.call(n, None if not shares else share, slots=False)
    assert (s.kv.page_table.cpu().numpy() == want[0]).all() and s.held.tolist() == want[3] and int(s.taken.item()) == want[2]


def test_refusals():
    lens, n, held = [20, 16, 0, 33], [13, 1, 17, 40], [4, 1, 0, 3]
    s = _Server(4, 200, 6)
    table = np.full((4, 6), -1, np.int32)
    for b in range(4):
        table[b, :held[b]] = 100 + 10 * b + np.arange(held[b])

    def call(code, bad, lens=lens, held=held, table=table, share=None, n_free=200):
        s.set(lens, held, table)
        s.taken.zero_()
        s.status.zero_()
        s.free_t = torch.from_numpy(s.free[:n_free]).cuda()
        slots = s.call(n, share)
        assert int(s.status.item()) == code
        left = lambda x: [0 if b in bad else y for b, y in enumerate(x)]  # noqa: E731
        want = op.reserve_held(table, left(lens), left(n), s.free, 0, left(held))
        stay = [held[b] if b in bad else x for b, x in enumerate(want[3])]
        assert (s.kv.page_table.cpu().numpy() == want[0]).all() and int(s.taken.item()) == want[2] and s.held.tolist() == stay
        at = np.cumsum([0] + n)
        for b in bad:
            assert (slots[at[b]:at[b + 1]] == -1).all()
    call(0, ())
    for x in (-1, 0, 1, 7, 1 << 30, -(1 << 31)):         # fewer than the length needs, past the table
        call(-1, (0,), held=[x, 1, 0, 3])
    for p in (1, 2):                                     # the page that rows continue, one of rows taken back
        for x in (-1, 200):
            t = table.copy()
            t[0, p] = x
            call(-4, (0,), table=t)
    t = table.copy()
    t[0, 3] = -1                                         # no row goes there
    call(0, (), table=t)
    call(-1, (1,), share=[-1, 0, -1, -1], held=[4, -1, 0, 3])
    call(-1, (1,), share=[-1, 0, -1, -1], held=[4, 7, 0, 3])
    call(-4, (3,), n_free=4)                             # the list is at its end: 1 + 2 + 2 pages
    call(-4, (2, 3), n_free=2)
    call(-4, (1, 2, 3), n_free=0)


def _every_page_once(s, B):
    table, held, taken = s.kv.page_table.cpu().numpy(), s.held.tolist(), int(s.taken.item())
    used = np.concatenate([table[b, :held[b]] for b in range(B)] + [s.free_t.cpu().numpy()[taken:]])
    assert sorted(used.tolist()) == sorted(s.free.tolist()), "a page is in two places or in none"


def test_draft_rows_taken_back_lose_no_page():
    """n_new + K - 1 rows reserved and n_new kept, sequences that end and others in their place."""
    B, K = 24, 8
    s = _Server(B, 600, 20)
    rng = np.random.default_rng(2)
    lens = [0] * B
    for step in range(120):
        n_new = rng.integers(1, K + 1, B).tolist() if step else rng.integers(1, 60, B).tolist()
        s.call([x + K - 1 for x in n_new], slots=False)
        assert int(s.status.item()) == 0
        lens = [a + x for a, x in zip(lens, n_new)]
        for b in range(B):
            if lens[b] > 220:          # it ends: its pages go back to the list
                t, h = int(s.taken.item()), int(s.held[b])
                s.free_t[t - h:t] = s.kv.page_table[b, :h]
                s.taken -= h
                s.held[b], lens[b] = 0, 0
                s.kv.page_table[b] = -1
        s.kv.seq_len.copy_(s.pc.ints(lens))
        _every_page_once(s, B)
        assert all(h * 16 >= x for h, x in zip(s.held.tolist(), lens))


def test_drafting_on_reserved_pages():
    """Steps of a drafter that takes its pages from the list as it goes: bit for bit the drafter that has them all."""
    from paper_2609_09338_gb300 import binding as ob
    from paper_2609_09338_gb300 import synthetic as syn
    from paper_2609_09338_gb300.binding import to_device_bf16
    from paper_2609_09338_gb300.session import DraftSession
    from paper_2609_09338_gb300.workloads import TINY
    B, K, most = 5, 4, 3
    ctx = np.array([30, 45, 48, 61, 17], np.int32)
    weights = syn.make_weights(TINY, 5)
    pre = syn.make_kv_prefix(TINY, ctx, 40, 6)
    fixed = DraftSession(TINY, weights, pre["page_table"], pre["n_pages"], K, most)
    moving = DraftSession(TINY, weights, np.full_like(pre["page_table"], -1), pre["n_pages"], K, most)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    free = torch.randperm(pre["n_pages"], device="cuda").int()
    taken, held = dev(np.zeros(1, np.int32)), dev(np.zeros(B, np.int32))

    def reserve(n):
        ob.osprey_kv_reserve(moving.ctx, moving.kv, dev(np.asarray(n, np.int32)), free, taken, moving.status,
                             total_rows=int(sum(n)), held=held)
    reserve(ctx)
    for x in (fixed, moving):
        x.append(ctx, pre["k_rows"], pre["v_rows"])
    for step in range(8):
        di = syn.make_draft_inputs(TINY, B, most, K, 7 + step)
        n_new = np.random.default_rng(step).integers(1, most + 1, B).astype(np.int32)
        reserve(n_new + K - 1)
        out = [x.draft_buffers(with_logits=True) for x in (fixed, moving)]
        for x, o in zip((fixed, moving), out):
            x.draft(dev(n_new), dev(di["tokens"]), to_device_bf16(di["feats"]), 1.0, dev(di["u_draft"]), o)
        for k in out[0]:
            assert torch.equal(out[0][k], out[1][k]), (step, k)
        used = moving.kv.page_table[torch.arange(moving.kv.max_pages, device="cuda")[None] < held[:, None]]
        assert used.unique().numel() == used.numel() == int(taken.item())
        # a verification keeps some of the rows: some steps go back, across pages too
        if step % 3 == 2:
            for x in (fixed, moving):
                x.kv.seq_len -= dev(np.minimum(ctx % 7 + 2, 9).astype(np.int32))
    assert int(fixed.status.item()) == 0 and int(moving.status.item()) == 0


def test_captured_and_on_a_stream_of_its_own():
    """A captured call goes on from what the replay before it left: lengths, held pages and the counter are on the device."""
    B, K = 6, 8
    s = _Server(B, 300, 30)
    n = s.pc.ints([K] * B)

    def call(stream=None):
        s.ob.osprey_kv_reserve(s.ctx, s.kv, n, s.free_t, s.taken, s.status, total_rows=B * K, held=s.held, stream=stream)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    side = torch.cuda.Stream()
    for step in range(40):
        s.kv.seq_len += s.pc.ints([(step + b) % (K + 1) for b in range(B)])
        torch.cuda.synchronize()
        if step % 2:
            graph.replay()
        else:
            call(side)
        torch.cuda.synchronize()
        _every_page_once(s, B)
        lens = s.kv.seq_len.tolist()
        assert all(h >= -(-(t + K) // 16) for h, t in zip(s.held.tolist(), lens)) and int(s.status.item()) == 0
