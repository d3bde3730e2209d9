"""A model of the large attention kernel's notes on values that are not finite (k_attend_tile in
paper_2609_13692_gb300/csrc/k_attend_tile.cu), run on random interleavings of its roles.

An item has n0 key tiles for its first row tile and n1 for its second (0: it has none).  Per item, the
watching warp waits until both row tiles have read what its set of notes held for the item four before,
where they had a part of that, then writes the set; per key tile it waits until the last phase that it
gave each score buffer has ended and arrives on "P ready" of those that the tile concerns.  The issuing
warp makes the first scores, then per key tile waits for P of each row tile and issues its outputs and
next scores.  A row tile takes its scores, arrives on "P ready", and after its last waits for its
outputs, reads the item's notes (for as long as it takes) and arrives on the set's barrier.

Checked on every interleaving: no deadlock; a parity wait never sees two phases pass; the notes that a
row tile reads are its own item's from its first look to its last.  The planted mistakes must be caught.
"""

import random

import pytest

SETS = 4


def simulate(items, rng, waits_for=lambda s, item: True, sets=SETS):
    need = {"p": 2}  # the rows' arrival and the watching warp's
    done, arrived = {}, {}
    notes = [None] * sets
    reading = {}  # (row tile, set) -> item

    def arrive(bar):
        arrived[bar] = arrived.get(bar, 0) + 1
        if arrived[bar] == need.get(bar[0], 1):
            arrived[bar] = 0
            done[bar] = done.get(bar, 0) + 1

    def passable(bar, phase):
        n = done.get(bar, 0)
        assert n <= phase + 1, f"parity wait on {bar} for phase {phase} after {n}"
        return n > phase

    def watch():
        owed, phase, given, due = {}, {}, [0, 0], []
        for i, n in enumerate(items):
            c = i % sets
            for s in (0, 1):
                if owed.get((s, c)):
                    if waits_for(s, i):
                        yield ("read", s, c), phase.get((s, c), 0)
                    phase[s, c] = phase.get((s, c), 0) + 1
                owed[s, c] = n[s] > 0
            for s in (0, 1):
                assert (s, c) not in reading, f"notes of item {reading.get((s, c))} written over by item {i}"
            notes[c] = i
            yield None
            for j in range(max(n)):
                for s in due:
                    yield ("p", s), given[s] - 1
                due = [s for s in (0, 1) if j < n[s]]
                for s in due:
                    given[s] += 1
                    arrive(("p", s))
                yield None

    def issue():
        ready = [0, 0]
        for n in items:
            for s in (0, 1):
                if n[s]:
                    arrive(("s", s))
            yield None
            for j in range(max(n)):
                for s in (0, 1):
                    if j < n[s]:
                        yield ("p", s), ready[s]
                        ready[s] += 1
                        arrive(("s" if j + 1 < n[s] else "o", s))
                        yield None

    def rows(s):
        scored = out = 0
        for i, n in enumerate(items):
            if n[s] == 0:
                continue
            for _ in range(n[s]):
                yield ("s", s), scored
                scored += 1
                arrive(("p", s))
                yield None
            yield ("o", s), out
            out += 1
            c = i % sets
            reading[s, c] = i
            for _ in range(rng.choice([1, 1, 2, 6])):
                assert notes[c] == i, f"row tile {s} reads item {notes[c]}'s notes for item {i}'s"
                yield None
            del reading[s, c]
            arrive(("read", s, c))
            yield None

    progs = [watch(), issue(), rows(0), rows(1)]
    waits, over = [next(p, "end") for p in progs], [False] * 4
    pace = [rng.choice([1, 1, 8, 60]) for _ in progs]  # some roles far slower than others
    while True:
        for w, at in enumerate(waits):
            over[w] = at == "end"
        ready = [w for w in range(4) if not over[w] and (waits[w] is None or passable(*waits[w]))]
        if not ready:
            assert all(over), f"deadlock: {waits}"
            return
        w = rng.choices(ready, [1 / pace[w] for w in ready])[0]
        waits[w] = next(progs[w], "end")


def lists(rng, count):
    for _ in range(count):
        # a pair of row tiles now and then, most items with one; the second sees as much as the first, or is not there
        out = []
        for _ in range(rng.randint(1, 24)):
            n0 = rng.choice([0, 1, 1, 2, 3])
            n1 = rng.choice([0, 0, 0, n0, n0 + 1])
            if n0 or n1:
                out.append((n0, n1))
        if out:
            yield out


@pytest.mark.parametrize("seed", range(8))
def test_notes_are_their_own_items(seed):
    rng = random.Random(seed)
    for items in lists(rng, 150):
        simulate(items, rng)
    for _ in range(40):  # one pair, then items that the second row tile has no part of
        simulate([(2, 2)] + [(1, 0)] * 12 + [(1, 1)] * 3, rng)


def caught(**planted):
    rng = random.Random(3)
    try:
        for items in lists(rng, 300):
            simulate(items, rng, **planted)
    except AssertionError:
        return True
    return False


def test_planted_protocol_mistakes_are_caught():
    # no wait at all: only the score buffers hold the watching warp back
    assert caught(waits_for=lambda s, i: False)
    # the first row tile alone
    assert caught(waits_for=lambda s, i: s == 0)
    # the second alone
    assert caught(waits_for=lambda s, i: s == 1, sets=1)
