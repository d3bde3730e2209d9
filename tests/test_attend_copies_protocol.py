"""Models of the copies in flight of both attention kernels (paper_2609_13692_gb300/csrc/k_attend_few.cu and
k_attend_tile.cu) where a bounded wait gives up, run on random interleavings.

Copies land late and in any order, and any wait may give up at any time.  Checked: while nothing has given
up, every stage that is read holds its own copy; no stage is filled again while a copy into it is in
flight; and when the block ends none is in flight.  The planted mistakes must be caught.
"""

import random

import pytest


class Ring:
    """Barriers "full" (one arrival and the copy's bytes) and "empty" of each stage, by phases."""

    def __init__(self, stages, readers):
        self.stages, self.readers = stages, readers
        self.armed = [0] * stages   # uses whose copy was issued
        self.landed = [0] * stages  # phases of "full"
        self.back = [0] * stages    # arrivals on "empty"
        self.holds = [None] * stages
        self.flying = []

    def issue(self, use):
        s = use % self.stages
        assert self.armed[s] == self.landed[s], f"use {use} fills a stage whose copy is in flight"
        self.armed[s] += 1
        self.flying.append(use)

    def land(self, rng):
        use = self.flying.pop(rng.randrange(len(self.flying)))
        self.landed[use % self.stages] += 1
        self.holds[use % self.stages] = use

    def full(self, use):  # as a parity wait sees it
        n = self.landed[use % self.stages] - use // self.stages
        return n % 2 == 1

    def empty(self, use):  # the stage's use before this one was handed back by every reader
        n = self.back[use % self.stages] // self.readers - (use // self.stages - 1)
        return n % 2 == 1


def run(roles, ring, rng, state):
    """Steps the roles; a role yields None, or (condition, may give up), and gets whether it held."""
    waits = [next(r, "end") for r in roles]
    over = [w == "end" for w in waits]
    eager = rng.random()
    while not all(over):
        choices = [i for i in range(len(roles)) if not over[i] and (waits[i] is None or waits[i][0]())]
        stuck = [i for i in range(len(roles)) if not over[i] and waits[i] is not None and waits[i][1]]
        if ring.flying and (not choices or rng.random() < eager):
            ring.land(rng)
            continue
        held = True
        if stuck and (not choices or rng.random() < state["rate"]):
            i, held = rng.choice(stuck), False
            state["gave_up"] = True
        else:
            assert choices, "deadlock"
            i = rng.choice(choices)
        try:
            waits[i] = roles[i].send(held if waits[i] is not None else None)
        except StopIteration:
            over[i] = True
    assert not ring.flying, f"the block ends with copies {ring.flying} in flight"


def few(rng, uses, stages, copiers, rate, looks=True, drains=lambda ok: True):
    """k_attend_few: copying warps take stages in turn, four warps read every stage, and go on having given up."""
    ring, state = Ring(stages, 4), dict(gave_up=False, rate=rate)

    def copier(me):
        ok, done = True, 0
        for use in range(me, uses, copiers):
            if use >= stages:
                ok = yield (lambda: ring.empty(use)), True
                if looks and state["gave_up"]:
                    ok = False
                if not ok:
                    break
            ring.issue(use)
            done = use + 1
            yield None
        if drains(ok):
            for use in range(max(0, done - stages), done):
                if use % copiers == me:
                    yield (lambda: ring.full(use)), False

    def reader():
        for use in range(uses):
            yield (lambda: ring.full(use) or state["gave_up"]), True
            if not state["gave_up"]:
                assert ring.holds[use % stages] == use
            yield None
            ring.back[use % stages] += 1

    run([copier(i) for i in range(copiers)] + [reader() for _ in range(4)], ring, rng, state)


def tile(rng, tiles, slots, rate, last=None, drains=True):
    """k_attend_tile: keys in uses 2 g, values in uses 2 g + 1, a warp each; the products hand uses back in order
    and stop at the first wait that gives up; both copying warps see to their own copies at the block's end."""
    ring, state = Ring(slots, 1), dict(gave_up=False, rate=rate)
    sent, left = [0, 0], [3]
    last = (slots + 1) // 2 if last is None else last

    def copier(v):
        for g in range(tiles):
            use = 2 * g + v
            if use >= slots and not (yield (lambda: ring.empty(use)), True):
                break
            ring.issue(use)
            sent[v] = g + 1
            yield None
        left[0] -= 1
        yield (lambda: left[0] == 0), False
        if drains and state["gave_up"]:
            for g in range(max(0, sent[v] - last), sent[v]):
                use = 2 * g + v
                # a phase that the other warp has passed reads as not complete: a limit ends that wait
                passed = ring.landed[use % slots] > use // slots
                yield (lambda: ring.full(use) or passed), False

    def products():
        for use in range(2 * tiles):
            if not (yield (lambda: ring.full(use)), True):
                break
            assert ring.holds[use % slots] == use
            yield None
            ring.back[use % slots] += 1
        left[0] -= 1

    run([copier(0), copier(1), products()], ring, rng, state)


FEW = [(3, 1), (4, 1), (3, 3)]
RATES = [0.0, 0.0, 0.02, 0.2]


@pytest.mark.parametrize("stages,copiers", FEW)
def test_small_kernel(stages, copiers):
    rng = random.Random(stages + copiers)
    for _ in range(1500):
        few(rng, rng.randint(1, 20), stages, copiers, rng.choice(RATES))


@pytest.mark.parametrize("slots", [2, 5, 8])
def test_large_kernel(slots):
    rng = random.Random(slots)
    for _ in range(2500):
        tile(rng, rng.randint(1, 20), slots, rng.choice(RATES))


def caught(model, cases, **planted):
    rng = random.Random(9)
    for _ in range(6000):
        try:
            model(rng, rng.randint(1, 16), *rng.choice(cases), rng.choice(RATES), **planted)
        except AssertionError:
            return True
    return False


def test_planted_protocol_mistakes_are_caught():
    # a copying warp that waits for its copies only where it gave up itself
    assert caught(few, FEW, drains=lambda ok: not ok)
    # one that takes a stage back from warps that gave up
    assert caught(few, FEW, looks=False)
    # no wait at the large kernel's end; for too few of the last uses
    assert caught(tile, [(2,), (5,), (8,)], drains=False)
    assert caught(tile, [(8,)], last=3)
    assert caught(tile, [(5,)], last=2)
