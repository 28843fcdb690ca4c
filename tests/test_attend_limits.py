"""How long the waits of the attention over the bf16 cache may last (csrc/attn_pages.cu): each ends, or its limit is
renewed, within a bounded number of products, however much work a block has."""
import os
import random
import re

import pytest

from test_attend_protocol import Model


class Watched:
    """A wait whose limit is renewed whenever the block is through with one more tile of both streams."""

    def __init__(self, condition):
        self.condition = condition

    def __call__(self):
        return self.condition()


class Timed(Model):
    """The barriers' model with a clock: a product executed is a step of it."""

    def products(self, me):
        for i, c in enumerate(super().products(me)):
            hand_over = me == 1 and i == 0
            yield Watched(c) if hand_over and self.bad != "one limit for all of the shared units" else c

    def execute(self):
        op = self.queue[0]
        super().execute()
        if op[0] != "commit":
            self.clock += 1
            if op[0] == "O" and op[3][0] and op[1] == 1 and op[4] == 1:
                self.steps += 1

    def longest(self):
        """Runs all of it; the longest time that an actor's wait lasts without an end or a renewal."""
        self.clock = self.steps = 0
        actors = [[a, lambda: True, 0, 0] for a in
                  (self.copies(0), self.copies(1), self.products(0), self.products(1), self.weights(0), self.weights(1))]
        longest = 0
        while actors or self.queue or self.flying:
            ready = []
            for a in actors:
                if a[1]():
                    ready.append(a)
                    continue
                if isinstance(a[1], Watched) and a[3] != self.steps:
                    a[2], a[3] = self.clock, self.steps
                longest = max(longest, self.clock - a[2])
            ready += ["land"] * bool(self.flying) + ["execute"] * bool(self.queue)
            assert ready, "everything waits"
            a = self.rng.choice(ready)
            if a == "land":
                self.land()
            elif a == "execute":
                self.execute()
            else:
                try:
                    a[1] = next(a[0])
                    a[2], a[3] = self.clock, self.steps
                except StopIteration:
                    actors.remove(a)
        return longest


# A tile has six products; a wait for a slot lasts as long as the tiles in the ring, the queue of a stream beside it none more.
def _most(ns):
    return 6 * (ns + 4)


@pytest.mark.parametrize("ns,nss", [(5, 2), (10, 5)])
def test_no_wait_lasts_as_long_as_the_work(ns, nss):
    for seed in range(20):
        m = Timed(random.Random(seed), [60, 1, 90], [[3, 40], [2, 50]], ns, nss)
        assert m.longest() <= _most(ns)


def test_one_limit_for_all_of_the_shared_units_is_caught():
    for seed in range(5):
        m = Timed(random.Random(seed), [60, 1, 90], [[3], [2]], 10, 5, "one limit for all of the shared units")
        assert m.longest() > 3 * _most(10)


class Ending(Model):
    """A wait gives up, then others as they find out; the block leaves.  Thread 0 is one of the first stream's weights'."""

    def leave(self, at):
        """`at`: how many steps come before some wait gives up."""
        actors = {i: [a, lambda: True] for i, a in enumerate(
            [self.copies(0), self.copies(1), self.products(0), self.products(1), self.weights(0), self.weights(1)])}
        abort = seen_by_thread_0 = False
        while actors:
            blocked = [i for i, (_, c) in actors.items() if not c()]
            give_up = blocked if abort or at <= 0 else []
            ready = [i for i in actors if i not in blocked] + ["land"] * bool(self.flying) + ["execute"] * bool(self.queue)
            at -= 1
            i = self.rng.choice(ready + give_up)
            if i == "land":
                self.land()
            elif i == "execute":
                self.execute()
            else:
                if i in blocked:
                    abort = True
                    del actors[i]
                else:
                    try:
                        actors[i][1] = next(actors[i][0])
                        continue
                    except StopIteration:
                        del actors[i]
                if i == 4:
                    seen_by_thread_0 = abort
        told = seen_by_thread_0 if self.bad == "thread 0 looks when it is through" else abort
        while told and (self.queue or self.flying):        # stays until these are through
            self.land() if self.flying else self.execute()
        return abort, told, len(self.queue) + len(self.flying)


def _endings(bad=None):
    for seed in range(300):
        rng = random.Random(seed)
        m = Ending(rng, [3, 1, 2], [[2], [2, 9]], 10, 5, bad)
        yield m.leave(rng.randint(0, 400))


def test_a_wait_that_gives_up_is_told_and_nothing_is_in_flight_when_the_block_leaves():
    ended = list(_endings())
    assert sum(a for a, _, _ in ended) > 100
    for abort, told, left in ended:
        assert told == abort and left == 0


def test_looking_for_it_before_all_are_through_is_caught():
    assert sum(abort and not told for abort, told, _ in _endings("thread 0 looks when it is through")) > 5


def test_a_bad_page_does_not_take_back_that_all_is_cleared():
    """head->bad: 1 of a bad page, 2 of a wait that gave up, from any blocks in any order: every change raises it."""
    src = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_09338_gb300", "csrc", "attn_pages.cu")
    with open(src) as f:
        text = f.read()
    kernel = text[text.index("    attend_kernel(const __grid_constant__"):text.index("void __launch_bounds__(512, 2) attend_join_kernel")]
    assert len(re.findall(r"head->bad", kernel)) == len(re.findall(r"atomicMax\(&w\.head->bad, [12]\)", kernel)) >= 2
