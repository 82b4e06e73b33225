"""Whether two states of beams share memory, as the reordering call decides it
before it writes, against sets of bytes written out."""
import random

import pytest

from paper_2609_24150_amd import api


def written_out(first, dims, n):
    places = {first}
    for s, c in dims:
        places = {x + s * k for x in places for k in range(c)}
    return {x + i for x in places for i in range(n)}


@pytest.mark.parametrize("seed", range(4))
def test_against_bytes_written_out(seed):
    g = random.Random(seed)

    def regular():
        dims, n = [], g.randint(1, 6)
        end = n
        for _ in range(g.randint(0, 3)):
            s, c = end + g.choice([0, 0, 1, 3, 10]), g.randint(2, 4)
            dims.append((s, c))
            end += s * (c - 1)
        return sorted(dims, reverse=True), n

    for _ in range(1500):
        a, na = regular()
        b, nb = regular()
        if g.random() < 0.5:  # views of one array
            b, nb = [(s, g.randint(2, 4)) for s, _ in a], min(na, g.randint(1, 6))
        d = g.randint(-60, 60)
        assert api._meet(d, a, na, b, nb) == bool(written_out(0, a, na) & written_out(d, b, nb)), (d, a, na, b, nb)


def test_lists_of_states():
    beams = ((4000, 2), (1000, 3))
    one = (0, 7000, True, (2, 100, 500), beams)
    api._check_memory([one, (7000, 7000, True, (2, 100, 500), beams), (100, 6900, True, (2, 100, 500), beams)])
    api._check_memory([(0, 7000, False, (2, 100, 500), beams), (50, 6900, False, (2, 100, 500), beams)])
    for other in (one, (99, 6901, True, (2, 100, 500), beams), (4900, 100, False, (1, 900, 0), ((0, 2), (0, 3)))):
        with pytest.raises(ValueError):
            api._check_memory([(10 ** 6, 50, True, (1, 50, 0), beams), other, one])
