"""Which sequences the attention over the bf16 cache takes as a run that shares a prefix, and that others are refused."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__ as g
    g.build()


def _refused(share):
    """Sequences that are in no run: share[b] is neither -1 nor b, and somewhere in share[b] + 1 .. b another is named, or
    share[b] itself names another."""
    return [b for b, s in enumerate(share)
            if s not in (-1, b) and not (0 <= s < b and share[s] in (-1, s) and all(share[i] == s for i in range(s + 1, b + 1)))]


def _run(share, dtype, R, seed=5):
    """Every sequence begins with its named first one's 48 positions; the refused are 0, the others are right."""
    import kv8_cases as kc
    import pages_cases as pc
    ctx = kc.make_ctx(4, 2, 64)
    B = len(share)
    rng = np.random.default_rng(seed)
    n = rng.integers(1, R + 1, B).tolist()
    lens = [48 + m + int(x) for m, x in zip(n, rng.integers(0, 40, B))]
    as_built = [s if 0 <= s < b else -1 for b, s in enumerate(share)]
    c = pc.Cache(ctx, lens, 7, as_built, [48] * B)
    q = pc.queries(ctx, B, R, dtype, 6)
    out = pc.attend(c, n, q, share=share, shared_len=[48] * B)
    bad = _refused(share)
    assert int(c.status.item()) == (-1 if bad else 0)
    for b in bad:
        assert (out[b, :n[b]] == 0).all() and (out[b, n[b]:] == 77).all(), f"sequence {b} is refused"
    good = [b for b in range(B) if b not in bad]
    d = pc.Cache.__new__(pc.Cache)
    d.__dict__.update(c.__dict__, lens=[lens[b] for b in good], tab=c.tab[good])
    pc.check(d, out[good], [n[b] for b in good], q[good], rows=[0, 1, R - 1])


CASES = [[0, 0, 0, 0], [-1, 0, 0, -1], [0, 1, 0, 0], [0, 0, 2, 2, 0, 0], [-1, 0, -1, 0, 0], [1, 1, 1], [0, 2, 2, 0, 0],
         [0, 0, 0, 1, 1, 1], [0] * 31 + [31] * 2 + [0] * 33, [0] * 64 + [64] * 33 + [0, 64, 64]]


@pytest.mark.parametrize("R", [2, 70])          # the prefix is read for the run, or by each sequence
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("share", CASES, ids=range(len(CASES)))
def test_sequences_behind_a_gap_are_refused(share, dtype, R):
    _run(share, dtype, R)


def test_random_firsts():
    rng = np.random.default_rng(3)
    for i in range(12):
        B = int(rng.integers(2, 70))
        share, s = [], 0
        for b in range(B):
            x = rng.random()
            s = b if x < 0.2 else int(rng.integers(-1, B)) if x < 0.25 else s
            share.append(s if x > 0.03 else -1)
        _run(share, BF, 3, i)


def test_a_run_over_a_thousand_sequences():
    for share in ([0] * 1500, [0] * 1030 + [1030] * 200 + [0] * 9, [3] * 1040):
        _run(share, BF, 1)
