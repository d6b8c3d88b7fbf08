"""Which lists pic_orth_create refuses because an output overlaps something, without a
GPU: matrices of one buffer whose rows are different distances apart."""
import ctypes
import random

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def pic():
    from paper_2609_09020_gb300 import build, pic
    build.build()
    pic.load_library()
    return pic


P = 0x10000  # never followed
F16 = 1


def accepted(pic, *matrices):
    """(first element, rows, columns, distance) each, in place"""
    e = [pic.pic_orth_matrix(P + 2 * at, P + 2 * at, r, c, ld, ld, F16) for at, r, c, ld in matrices]
    return pic.load_library().pic_orth_room_bytes((pic.pic_orth_matrix * len(e))(*e), len(e)) >= 0


# slices of a [6, 20] buffer: columns [0, 7) and [7, 12), all rows, some, every second
LEFT, RIGHT = (0, 6, 7, 20), (7, 6, 5, 20)


@pytest.mark.parametrize("other,ok", [
    ((2 * 20, 1, 7, 7), True),        # one row as _matrices of pic.py has it, in the left columns
    ((2 * 20 + 12, 1, 8, 8), True),   # the rest of a row
    ((2 * 20, 1, 8, 8), False),       # one column more
    ((5 * 20 + 11, 1, 1, 1), False),  # the last element
    ((5 * 20 + 12, 1, 1, 1), True),
    ((12, 3, 8, 40), True),           # every second row
    ((6, 3, 2, 40), False),
    ((20, 3, 7, 40), True),
    ((0, 2, 7, 60), True),
    ((0, 2, 8, 60), False),
    ((12, 2, 10, 60), True),          # the rest of a row and two of the next
    ((1, 3, 6, 19), True),            # rows 1 to 6, 20 to 25, 39 to 44
    ((3, 4, 4, 21), False),           # 3, 24, 45, 66: the second is over one of the right columns
], ids=str)
def test_beside_columns(pic, other, ok):
    assert accepted(pic, RIGHT, other) == ok
    assert accepted(pic, other, RIGHT) == ok


def test_slices_of_one_buffer(pic):
    assert accepted(pic, LEFT, RIGHT, (12, 3, 8, 40), (32, 3, 8, 40))
    assert not accepted(pic, LEFT, RIGHT, (12, 3, 8, 40), (31, 3, 8, 40))


def test_one_row_in_place_at_any_distances(pic):
    e = pic.pic_orth_matrix(P, P, 1, 7, 7, 9, F16)
    assert pic.load_library().pic_orth_room_bytes(ctypes.byref(e), 1) >= 0


def test_against_elements(pic):
    """Random pairs: accepted if and only if they have no element in common."""
    rng = random.Random(0)
    seen = {True: 0, False: 0}
    for _ in range(4000):
        pair = []
        for _ in range(2):
            cols = rng.randint(1, 9)
            pair.append((rng.randint(0, 60), rng.randint(1, 6), cols, cols + rng.choice([0, 0, 3, 11, rng.randint(0, 30)])))
        sets = [{at + i * ld + j for i in range(r) for j in range(c)} for at, r, c, ld in pair]
        ok = not sets[0] & sets[1]
        assert accepted(pic, *pair) == ok, pair
        seen[ok] += 1
    assert min(seen.values()) > 500
