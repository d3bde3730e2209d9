"""A model of the large attention kernel's notes on values that are not finite (k_attend_tile in
paper_2609_13692_gb300/csrc/k_attend_tile.cu), run on random interleavings of its roles.

An item has n0 key tiles for its first row tile and n1 for its second (0: it has none).  Per item, the
warp that copies values waits until both row tiles have read what its set of notes held for the item
four before, arrives on the set's barrier for a row tile that has no part of the item, and copies the
values of its key tiles.  Per key tile the watching warp waits for the values, at the item's first writes
the set, then waits until the last phase that it gave each score buffer has ended and arrives on
"P ready" of those that the tile concerns.  The issuing warp makes the first scores, then per key tile
waits for P of each row tile and issues its outputs and next scores.  A row tile takes its scores,
arrives on "P ready", and after its last waits for its outputs, reads the item's notes (for as long as
it takes) and arrives on the set's barrier.

Checked on every interleaving: no deadlock; a parity wait never sees two phases pass; the notes that a
row tile reads are its own item's from its first look to its last.  The planted mistakes must be caught.
"""

import random

import pytest

SETS = 4


def simulate(items, rng, waits=True, stands_in=True, sets=SETS):
    need = {"p": 2, "read": 2}  # the rows' arrival and the watching warp's; both row tiles'
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

    def copies():
        for i, n in enumerate(items):
            c = i % sets
            if i >= sets and waits:
                yield ("read", c), i // sets - 1
            for s in (0, 1):
                if stands_in and n[s] == 0:
                    arrive(("read", c))
            for j in range(max(n)):
                yield None
                arrive(("v", (i, j)))

    def watch():
        given, due = [0, 0], []
        for i, n in enumerate(items):
            c = i % sets
            for j in range(max(n)):
                yield ("v", (i, j)), 0
                if j == 0:
                    for s in (0, 1):
                        assert (s, c) not in reading, f"notes of item {reading.get((s, c))} written over by item {i}"
                    notes[c] = i
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
            arrive(("read", c))
            yield None

    progs = [copies(), watch(), issue(), rows(0), rows(1)]
    at, over = [next(p, "end") for p in progs], [False] * 5
    pace = [rng.choice([1, 1, 8, 60]) for _ in progs]  # some roles far slower than others
    while True:
        for w, wait in enumerate(at):
            over[w] = wait == "end"
        ready = [w for w in range(5) if not over[w] and (at[w] is None or passable(*at[w]))]
        if not ready:
            assert all(over), f"deadlock: {at}"
            return
        w = rng.choices(ready, [1 / pace[w] for w in ready])[0]
        at[w] = next(progs[w], "end")


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
    # no wait: only the score buffers hold the watching warp back
    assert caught(waits=False)
    # nobody arrives for a row tile that has no part of an item
    assert caught(stands_in=False)
