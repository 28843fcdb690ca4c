"""The barriers of the attention over the 8-bit cache (csrc/attn8.cu), as a model run under random interleavings: the
copying warps, the issuing lane, the tensor pipe and the warpgroups, with mbarrier phases waited for by parity as the
hardware does.  Every buffer's reader finds the tile that it expects and no writer comes too early; nothing waits for
ever; a parity wait never passes on another phase than its own."""
import random

import pytest


class Bar:
    def __init__(self, count):
        self.count, self.left, self.done = count, count, 0

    def arrive(self):
        self.left -= 1
        if self.left == 0:
            self.left, self.done = self.count, self.done + 1

    def passes(self, phase):
        """mbarrier.try_wait.parity for phase `phase`: the current phase's parity is another."""
        if self.done % 2 == phase % 2:
            return False
        assert self.done == phase + 1, "a wait passed on another phase"
        return True


def run(rng, nt, NS, nsb, groups, bad=""):
    kfull, vfull = [Bar(1) for _ in range(NS)], [Bar(1) for _ in range(NS)]
    kfree, vfree = [Bar(1) for _ in range(NS)], [Bar(1) for _ in range(NS)]
    sfull, ofull = [Bar(1) for _ in range(2)], Bar(1)
    sread, pready = Bar(groups), Bar(groups)
    kslot, vslot = [None] * NS, [None] * NS
    S, O = [None] * nsb, None            # tile that a buffer holds
    sseen, oseen = [set() for _ in range(nsb)], set()
    P = [None] * groups
    pipe, copies = [], []                # products in order; copies in any order
    done = []

    def copier(ring, full, free, name):
        def load(t):
            copies.append((ring, full, t))
        for t in range(min(NS, nt)):
            load(t)
            yield None
        for t in range(nt - NS):
            yield (ofull, t) if bad == "slot freed by the output" and name == "v" else (free[t % NS], t // NS)
            load(t + NS)
            yield None

    def issuer():
        def scores(t):
            yield kfull[t % NS], t // NS
            if nsb == 1 and t > 0 and bad != "scores not waited for":
                yield sread, t - 1
            pipe.append(("S", t))
        if nt:
            yield from scores(0)
        for t in range(nt):
            if t + 1 < nt:
                yield from scores(t + 1)
            yield vfull[t % NS], t // NS
            yield pready, t
            pipe.append(("O", t))
            yield None

    def group(g):
        nonlocal O
        for t in range(nt):
            yield sfull[t % nsb], t // nsb
            assert S[t % nsb] == t, "scores of another tile"
            sseen[t % nsb].add(g)
            if nsb == 1:
                sread.arrive()
            yield None
            if t > 0 and bad != "weights before the output":
                yield ofull, t - 1
                assert O == t - 1, "output of another tile"
                oseen.add(g)
            P[g] = t
            yield None
            pready.arrive()
            yield None
            if t > 0 and bad == "weights before the output":
                yield ofull, t - 1
                assert O == t - 1, "output of another tile"
                oseen.add(g)
        if nt:
            yield ofull, nt - 1
            assert O == nt - 1, "output of another tile"
        done.append(g)

    def land():
        ring, full, t = copies.pop(rng.randrange(len(copies)))
        ring[t % NS] = t
        full[t % NS].arrive()

    def compute():
        nonlocal O, oseen
        kind, t = pipe.pop(0)
        if kind == "S":
            assert kslot[t % NS] == t, "K of another tile"
            assert S[t % nsb] is None or len(sseen[t % nsb]) == groups, "scores overwritten before they were read"
            S[t % nsb], sseen[t % nsb] = t, set()
            sfull[t % nsb].arrive()
            kfree[t % NS].arrive()
        else:
            assert vslot[t % NS] == t, "V of another tile"
            assert P == [t] * groups, "weights of another tile"
            assert O is None or len(oseen) == groups, "output overwritten before it was read"
            O, oseen = t, set()
            ofull.arrive()
            vfree[t % NS].arrive()

    actors = [copier(kslot, kfull, kfree, "k"), copier(vslot, vfull, vfree, "v"), issuer()] + [group(g) for g in range(groups)]
    waits = [None] * len(actors)
    alive = list(range(len(actors)))
    favour = rng.random()
    while alive or pipe or copies:
        ready = [i for i in alive if waits[i] is None or waits[i][0].passes(waits[i][1])]
        kinds = (["a"] if ready else []) + (["p"] if pipe else []) + (["c"] if copies else [])
        assert kinds, "every actor waits"
        if len(kinds) > 1 and "a" in kinds and rng.random() < favour:
            kinds = ["a"]
        k = rng.choice(kinds)
        if k == "a":
            i = rng.choice(ready)
            try:
                waits[i] = next(actors[i])
            except StopIteration:
                alive.remove(i)
        elif k == "p":
            compute()
        else:
            land()
    assert len(done) == groups


@pytest.mark.parametrize("NS,nsb,groups", [(3, 2, 1), (2, 2, 1), (6, 2, 1), (3, 2, 2), (2, 2, 2), (4, 2, 4), (4, 1, 4), (8, 2, 4)])
def test_no_tile_is_lost_or_overwritten(NS, nsb, groups):
    for seed in range(400):
        rng = random.Random(seed)
        run(rng, rng.randint(0, 14), NS, nsb, groups)


@pytest.mark.parametrize("bad,args", [("slot freed by the output", (2, 2, 1)), ("scores not waited for", (4, 1, 2)),
                                      ("weights before the output", (3, 2, 2))])
def test_known_mistakes_are_caught(bad, args):
    caught = 0
    for seed in range(400):
        rng = random.Random(seed)
        try:
            run(rng, 12, *args, bad)
        except AssertionError:
            caught += 1
    assert caught
