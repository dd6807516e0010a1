"""A CPU model of tree_pair's synchronisation (csrc/tree_pair.cu): the copies, the arrivals for the
other CTA's copies, the MMA issuer and both CTAs' softmax warps, as their waits, arrivals and
accesses in program order, run in random interleavings with copies that land in any order and MMAs
that complete in theirs. It looks for deadlocks, barriers that run two phases ahead of a waiter
(which a parity wait cannot tell from none), and buffers that are written while something still
reads them or read before they hold what is expected. With a wait taken out it has to find one."""
from __future__ import annotations

import random

import pytest

KEYS, VALUES = 3, 4


class Hazard(Exception):
    pass


class Model:
    def __init__(self, segments, passes, seed, without=""):
        """segments: tiles of each; passes: of QK, a tile; without: a wait to leave out."""
        self.tiles = [(s, i == 0, i == n - 1) for s, n in enumerate(segments) for i in range(n)]
        self.passes = passes
        self.rnd, self.without = random.Random(seed), without
        self.count, self.needs = {}, {"p_full": 8}
        for part in range(KEYS):
            self.needs["k_bar", 0, part] = 2  # (the leader's: its own copy and the other CTA's arrival)
        for part in range(VALUES):
            self.needs["v_bar", 0, part] = 2
        self.holds, self.reading, self.landing = {}, {}, {}
        self.copies, self.tensor = [], []
        self.scores_read = {}

    # ---- barriers
    def arrive(self, bar):
        self.count[bar] = self.count.get(bar, 0) + 1

    def wait(self, bar, phase, name=""):
        if name and name == self.without:
            return
        while True:
            done = self.count.get(bar, 0) // self.needs.get(bar, 1)
            if done > phase + 1:
                raise Hazard(f"{bar} is {done - phase} phases ahead of a waiter")
            if done > phase:
                return
            yield bar

    # ---- buffers
    def write(self, buf, tag):
        if self.reading.get(buf, 0) or self.landing.get(buf, 0):
            raise Hazard(f"{buf} is written while it is read or written")
        self.holds[buf] = tag

    def copy(self, bar, writes):
        for buf, _ in writes:
            if self.reading.get(buf, 0) or self.landing.get(buf, 0):
                raise Hazard(f"a copy to {buf} while it is read or written")
            self.landing[buf] = 1
        self.copies.append((bar, writes))

    def mma(self, reads, write):
        for buf, _ in reads:
            self.reading[buf] = self.reading.get(buf, 0) + 1
        self.tensor.append(("mma", reads, write))

    def commit(self, bar):
        self.tensor.append(("commit", bar, None))

    # ---- roles
    def order(self):
        """(score?, pass or half of PV) in the order of the copies and the issuer."""
        np = nh = 0
        while nh < 2 * len(self.tiles):
            more = np < nh + 3 if self.passes == 2 else np < nh // 2 + 2 and nh % 2 == 0
            if np < self.passes * len(self.tiles) and more:
                yield True, np
                np += 1
            else:
                yield False, nh
                nh += 1

    def load(self, c):
        for score, at in self.order():
            if score:
                n, i = divmod(at, self.passes)
                seg, first, _ = self.tiles[n]
                for part in range(KEYS):
                    if at:
                        yield from self.wait(("k_free", c, part), at - 1, "k_free")
                    writes = [(("K", c, part), (n, i))]
                    if i == 0 and first:
                        writes.append((("Q", c, part), seg))
                    self.copy(("k_bar", c, part), writes)
                    yield "step"
            else:
                n, half = divmod(at, 2)
                for part in (2 * half, 2 * half + 1):
                    if n:
                        yield from self.wait(("v_free", c, part), n - 1, "v_free")
                    self.copy(("v_bar", c, part), [(("V", c, part), n)])
                    yield "step"

    def relay(self):
        for score, at in self.order():
            if score:
                for part in range(KEYS):
                    yield from self.wait(("k_bar", 1, part), at, "relay")
                    self.arrive(("k_bar", 0, part))
                    yield "step"
            else:
                n, half = divmod(at, 2)
                for part in (2 * half, 2 * half + 1):
                    yield from self.wait(("v_bar", 1, part), n)
                    self.arrive(("v_bar", 0, part))
                    yield "step"

    def issue(self):
        for score, at in self.order():
            if score:
                n, i = divmod(at, self.passes)
                seg = self.tiles[n][0]
                if n >= 2 and self.scores_read.get(n - 2, 0) != 8:
                    raise Hazard("scores overwritten before every warp has read them")
                for part in range(KEYS):
                    yield from self.wait(("k_bar", 0, part), at)
                    self.mma([(("K", c, part), (n, i)) for c in (0, 1)] + [(("Q", c, part), seg) for c in (0, 1)],
                             ("S", n & 1, n))
                    for c in (0, 1):
                        self.commit(("k_free", c, part))
                    yield "step"
                if i == self.passes - 1:
                    for c in (0, 1):
                        self.commit(("s_full", c, n & 1))
            else:
                n, half = divmod(at, 2)
                if half == 0:
                    yield from self.wait("p_full", n, "p_full")
                for part in (2 * half, 2 * half + 1):
                    yield from self.wait(("v_bar", 0, part), n)
                    self.mma([(("V", c, part), n) for c in (0, 1)] + [(("P", c, w), n) for c in (0, 1) for w in range(4)],
                             ("O", None, n))
                    for c in (0, 1):
                        self.commit(("v_free", c, part))
                    yield "step"

    def meet(self, c, w, n):
        """The barrier of the two warps that share rows, n-th time."""
        self.arrive(("pair", c, w & 1))
        self.needs["pair", c, w & 1] = 2
        yield from self.wait(("pair", c, w & 1), n)

    def softmax(self, c, w):
        met = 0
        for n, (_, first, last) in enumerate(self.tiles):
            yield from self.wait(("s_full", c, n & 1), n >> 1)
            if self.holds.get(("S", n & 1)) != n:
                raise Hazard(f"scores of tile {n} are not there")
            self.scores_read[n] = self.scores_read.get(n, 0) + 1
            yield from self.meet(c, w, met)
            met += 1
            if n:
                yield from self.wait(("v_free", c, VALUES - 1), n - 1, "wait_pv")
            if n and not first and self.rnd.random() < 0.3:  # the reference is raised: O is scaled
                self.read_output(n - 1)
            self.write(("P", c, w), n)
            yield "step"
            self.arrive("p_full")
            if last:
                yield from self.meet(c, w, met)
                met += 1
                yield from self.wait(("v_free", c, VALUES - 1), n, "end_pv")
                self.read_output(n)
                yield "step"

    def read_output(self, n):
        if any(kind == "mma" and write[0] == "O" for kind, _, write in self.tensor):
            raise Hazard("O is read while an MMA adds to it")
        if self.holds.get(("O", None)) != n:
            raise Hazard(f"O does not hold the tiles up to {n}")

    def complete(self):
        kind, what, write = self.tensor.pop(0)
        if kind == "commit":
            return self.arrive(what)
        for buf, tag in what:
            if self.holds.get(buf) != tag:
                raise Hazard(f"an MMA reads {buf}: {self.holds.get(buf)} instead of {tag}")
            self.reading[buf] -= 1
        self.holds[write[0], write[1]] = write[2]

    def land(self):
        bar, writes = self.copies.pop(self.rnd.randrange(len(self.copies)))
        for buf, tag in writes:
            self.landing[buf] = 0
            self.holds[buf] = tag
        self.arrive(bar)

    def run(self):
        roles = {"load0": self.load(0), "load1": self.load(1), "relay": self.relay(), "issue": self.issue()}
        for c in (0, 1):
            for w in range(4):
                roles[f"softmax{c}{w}"] = self.softmax(c, w)
        slow = self.rnd.choice([1, 1, 4])  # a slow tensor core in some runs
        blocked, idle = {}, 0
        while roles or self.tensor or self.copies:
            pick = list(roles) + ["copies"] * bool(self.copies) + ["tensor"] * (bool(self.tensor) and self.rnd.random() < 1 / slow)
            if not pick:
                continue
            who = self.rnd.choice(pick)
            if who == "tensor":
                self.complete()
                idle = 0
            elif who == "copies":
                self.land()
                idle = 0
            else:
                try:
                    blocked[who] = next(roles[who])
                    idle = 0 if blocked[who] == "step" else idle + 1
                except StopIteration:
                    del roles[who]
                    blocked.pop(who, None)
                    idle = 0
            if idle > 2000 and not self.tensor and not self.copies:
                raise Hazard(f"deadlock: {blocked}")


def segments(rnd):
    return [rnd.choice([1, 1, 2, 3, 5]) for _ in range(rnd.randint(1, 4))]


@pytest.mark.parametrize("block", range(8))
def test_no_hazard_and_no_deadlock(block):
    for seed in range(block * 40, block * 40 + 40):
        Model(segments(random.Random(seed)), 1 + seed % 2, seed).run()


@pytest.mark.parametrize("without", ["k_free", "v_free", "relay", "p_full", "wait_pv", "end_pv"])
def test_a_wait_taken_out_is_seen(without):
    seen = 0
    for seed in range(60):
        try:
            Model(segments(random.Random(seed)) + [3], 1 + seed % 2, seed, without).run()
        except Hazard:
            seen += 1
    assert seen > 20, seen
