"""The deal of the log probabilities' segments to waves, replayed on the CPU: every part of a row
has a place of its own, and the finishing launch reads exactly the row's parts."""
import random

import pytest

BLOCKS, WAVES, ELEMS = 1024, 4, 2048           # kLogBlocks, kLogWaves, elements of a segment


def replay(counts, n, segs):
    """What the pass writes and the finishing launch reads, as the kernels do it: places in
    `masses` and `whole`, `parts`, for sequences with counts[b] of n rows."""
    B, rows = len(counts), sum(counts)
    waves = -(-min(B * n * segs, BLOCKS * WAVES) // WAVES) * WAVES     # whole blocks
    total = rows * segs
    ranges = min(total, waves)
    share = total // ranges if ranges else 0
    longer = total - share * ranges

    def range_of(x):
        of_longer = (share + 1) * longer
        return x // (share + 1) if x < of_longer else longer + (x - of_longer) // share

    first = [(b, i) for b, c in enumerate(counts) for i in range(c)]
    places, parts = {}, {}
    for w in range(ranges):
        x, x1 = share * w + min(w, longer), share * (w + 1) + min(w + 1, longer)
        assert x < x1 and range_of(x) == w == range_of(x1 - 1)
        while x < x1:
            row, g0 = first[x // segs], x % segs
            g1 = min(segs, g0 + x1 - x)
            x += g1 - g0
            begins = g0 == 0
            whole = begins and g1 == segs
            place = ("whole", row) if whole else ("masses", w, begins)
            assert place not in places, (place, "is written twice")
            places[place] = (row, g0, g1)
            if begins:
                parts[row] = (0, -1) if whole else (w, range_of(x + segs - g1 - 1))
    for row in first:
        a, z = parts[row]
        read = [("whole", row)] if z < 0 else [("masses", w, w == a) for w in range(a, z + 1)]
        at = 0
        for place in read:
            got, g0, g1 = places.pop(place)
            assert got == row and g0 == at, (row, place)
            at = g1
        assert at == segs, row
    assert not places


@pytest.mark.parametrize("B,n,V", [(1, 1, 1), (1, 11, 32000), (64, 17, 128256), (4, 2048, 32000), (512, 9, 3000), (64, 65, 128256),
                                   (1, 4096, 300), (1, 4097, 300), (4096, 11, 100), (3, 1365, 4097), (2, 5000, 2048)])
def test_every_part_has_its_place(B, n, V):
    rng = random.Random(B * n + V)
    segs = -(-V // ELEMS)
    replay([n] * B, n, segs)
    replay([rng.choice([0, 1, n // 2, n, rng.randint(0, n)]) for _ in range(B)], n, segs)


def test_every_part_has_its_place_at_random():
    rng = random.Random(7)
    for _ in range(60):
        B, segs = rng.randint(1, 300), rng.choice([1, 1, 2, 3, 5, 16, 63])
        n = rng.randint(1, 1 + 20000 // B)
        replay([rng.randint(0, n) for _ in range(B)], n, segs)
