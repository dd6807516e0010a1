"""The model of mla_prefill's barriers with the lock that lets one tile's MMAs be issued at a
time (`turn`): take, give and the rule that it is given back before a wait for keys or values
that are not there yet. It looks for deadlocks, for both threads holding it, and for a wait with
the lock in hand other than that for the second half of a tile's weights, which the softmax
hands over without waiting for anything."""
from __future__ import annotations

import random

import pytest

from test_prefill_protocol_model import GIVE_BACK, Model, random_item


class TurnModel(Model):
    gives_before_waiting = True

    def __init__(self, items, seed):
        super().__init__(items, seed)
        self.holder = None

    def held_wait(self, bar, phase, i, allowed=False):
        for state in self.wait(bar, phase):
            if self.holder == i and not allowed:
                self.problem = f"thread {i} waits for {bar} with the lock in hand"
            yield state

    def take(self, i):
        while self.holder not in (None, i):
            yield "turn"
        self.holder = i

    def give(self, i):
        if self.holder == i:
            self.holder = None
            self.arrive("given")  # (progress, for the search for deadlocks)

    def entry(self, e, i):
        """Waits for a ring entry, the lock given back first if it is not there yet."""
        if self.count.get(f"full{e & 3}", 0) <= e >> 2 and self.gives_before_waiting:
            self.give(i)
        yield from self.held_wait(f"full{e & 3}", e >> 2, i, not self.gives_before_waiting)

    def mma(self, i):
        e = weights = outputs = 0
        loads = [0, 0]
        queue = self.tensor[i]
        for pair in range(1 << 30):
            item = yield from self.next_item(pair)
            if item is None:
                self.give(i)
                return
            n0, n1, dealt, _ = item
            q, both = (0 if dealt else i), max(n0, n1)
            n = (n0 + 1 - i) >> 1 if dealt else (n1 if i else n0)
            rounds = (both + 1) >> 1 if dealt else both
            if n:
                yield from self.held_wait(f"q_full{q}", loads[q], i)
            loads[0] += n0 > 0
            loads[1] += not dealt and n1 > 0
            for x in range(2 * rounds):
                j = x >> 1

                def skip():
                    nonlocal e
                    yield from self.entry(e, i)
                    self.arrive(f"freed{e & 3}")
                    e += 1

                if (i == 1) if dealt else j >= n:
                    yield from skip()
                if j < n:
                    if x & 1 == 0:
                        yield from self.entry(e, i)
                        yield from self.take(i)
                        queue += [f"s_full{i}"]
                        self.give(i)
                        queue += [f"freed{e & 3}"] + [f"q_free{q}"] * (j + 1 == n)
                    else:
                        yield from self.held_wait(f"full{e & 3}", e >> 2, i)
                        if j == 0 and outputs:
                            yield from self.held_wait(f"o_free{i}", outputs - 1, i)
                        for h in range(2):
                            yield from self.held_wait(f"p_full{i}{h}", weights, i, allowed=h == 1)
                            if h == 0:
                                yield from self.take(i)
                        weights += 1
                        queue += [f"freed{e & 3}"] + [f"o_full{i}"] * (j + 1 == n)
                        outputs += j + 1 == n
                        if j + 1 == n:
                            self.give(i)
                    e += 1
                if dealt and i == 0 and 2 * j + 1 < both:
                    yield from skip()
                if x == GIVE_BACK and i == 1 and not dealt and n0:
                    self.arrive("q_free0")


@pytest.mark.parametrize("block", range(6))
def test_no_deadlock_with_the_lock(block):
    for seed in range(block * 120, block * 120 + 120):
        rnd = random.Random(seed)
        items = [random_item(rnd) for _ in range(rnd.randint(0, 10))]
        model = TurnModel(items, seed)
        problem = model.run()
        assert problem is None and model.holder is None, (seed, items, problem)


def test_the_model_sees_a_lock_held_through_a_wait():
    """Kept while keys are late, the lock keeps the other tile from using up what it was given."""
    class Broken(TurnModel):
        gives_before_waiting = False

    rnd = random.Random(1)
    runs = [Broken([random_item(rnd) for _ in range(8)], seed).run() or "" for seed in range(60)]
    assert any("deadlock" in r for r in runs)


def test_the_model_sees_a_lock_that_is_not_given_back():
    class Broken(TurnModel):
        def give(self, i):
            if i == 0:
                super().give(i)

    assert all(Broken([(3, 3, False, 2)] * 4, seed).run() for seed in range(20))
