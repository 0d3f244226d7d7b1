"""A ring of stages between one loader and several consumers, as the kernels of
few rows keep it: barriers are waited for by the parity of their phase alone, and
loads land in any order.  A place of the ring that always belongs to the same
consumer is never taken before its load has landed; a place that changes hands
can be (which is why the kernels hold the number of places to a multiple of
their consumers)."""
import random

import pytest


def run(consumers, places, tiles, seed):
    """Random interleavings; returns the tiles taken before their load landed, and whether the ring came to its end."""
    r = random.Random(seed)
    full, empty = [0] * places, [0] * places          # completed phases of each place's barriers
    issued, flying, landed = 0, [], set()
    at, busy, early = list(range(consumers)), [False] * consumers, 0
    while True:
        acts = []
        if issued < tiles:
            place, turn = issued % places, issued // places
            if turn == 0 or (empty[place] & 1) != ((turn - 1) & 1):   # a parity wait passes once the phase's parity is past
                acts.append(("issue", 0))
        acts += [("land", i) for i in range(len(flying))]
        for c in range(consumers):
            if busy[c]:
                acts.append(("release", c))
            elif at[c] < tiles and (full[at[c] % places] & 1) != ((at[c] // places) & 1):
                acts.append(("take", c))
        if not acts:
            return early, issued == tiles and all(a >= tiles for a in at)
        what, i = r.choice(acts)
        if what == "issue":
            flying.append(issued)
            issued += 1
        elif what == "land":
            t = flying.pop(i)
            full[t % places] += 1
            landed.add(t)
        elif what == "take":
            early += at[i] not in landed
            busy[i] = True
        else:
            empty[at[i] % places] += 1
            busy[i] = False
            at[i] += consumers


@pytest.mark.parametrize("consumers,places", [(3, 6), (3, 3), (2, 6)])
def test_a_place_of_one_consumer(consumers, places):
    for seed in range(200):
        assert run(consumers, places, 40, seed) == (0, True)


def test_a_place_that_changes_hands_is_taken_early():
    assert any(run(4, 6, 60, seed) != (0, True) for seed in range(200))
