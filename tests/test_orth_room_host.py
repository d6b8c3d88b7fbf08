"""The room of pic_orth_create's matrices, counted without a GPU: up to the largest
sizes, where 32 bits do not hold it."""
import ctypes

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def pic():
    from paper_2609_09020_gb300 import build, pic
    build.build()
    pic.load_library()
    return pic


P = 0x10000  # never followed
F32, F16, BF16 = 0, 1, 2


def entry(pic, at, rows, cols, dtype):
    return pic.pic_orth_matrix(at, at, rows, cols, cols, cols, dtype)


def room(pic, *shapes):
    """The C function's count for (rows, cols, type) matrices that lie apart."""
    entries, at = [], P
    for rows, cols, dtype in shapes:
        entries.append(entry(pic, at, rows, cols, dtype))
        at += rows * cols * 4 + 256
    return pic.load_library().pic_orth_room_bytes((pic.pic_orth_matrix * max(1, len(entries)))(*entries), len(entries))


def want(rows, cols, dtype):
    m = min(rows, cols)
    halves = 1 if dtype == BF16 and m > 64 else 2
    up = lambda n, to: -(-n // to) * to
    x, a = up(2 * rows * up(cols, 64) * 2, 256), up(halves * m * up(m, 64) * 2, 256)
    return 2 * x + 2 * a


LARGE = 2 ** 31 - 257
# the totals of the second and third, in 32 bits, come to less than nothing
BY_TILES = [(2 ** 30, 1), (2 ** 31 - 1257, 1), (LARGE, 1), (1, LARGE), (LARGE, 40), (300, 200), (129, 129), (64, 200000),
            (2 ** 20, 1000)]


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("rows,cols", BY_TILES, ids=str)
def test_room_of_a_matrix(pic, rows, cols, dtype):
    assert room(pic, (rows, cols, dtype)) == want(rows, cols, dtype)


def test_room_of_a_list(pic):
    shapes = [(300, 200, F32), (LARGE, 1, BF16), (500, 900, BF16), (2 ** 30, 1, F16), (150, 200, F16)]
    assert room(pic, *shapes) == sum(want(*s) for s in shapes)
    assert room(pic) == 0
    assert room(pic, (64, 64, F32), (3, 64, F32)) == 0  # by a CTA each
    assert room(pic, (0, 5, F32), (7, 0, F16)) == 0


def test_room_beyond_any_device(pic):
    """Products that leave 64 bits, and sums that would."""
    for shapes in ([(LARGE, LARGE, BF16)], [(2 ** 29, 2 ** 30, F16)] * 3 + [(300, 200, F32)], [(2 ** 28, 2 ** 20, BF16)] * 70):
        assert 2 ** 50 <= room(pic, *shapes) <= 2 ** 50 + 2 ** 20


def test_room_of_refused_lists(pic):
    count = pic.load_library().pic_orth_room_bytes
    make = lambda *m: (pic.pic_orth_matrix * len(m))(*m)
    assert count(make(entry(pic, P, 2 ** 31, 1, F32)), 1) == -1
    assert count(make(entry(pic, P, 4, 5, 3)), 1) == -1
    assert count(make(entry(pic, P, 4, 5, F32), entry(pic, P, 4, 5, F32)), 2) == -1
    assert count(None, 1) == -1
    assert count(None, -1) == -1


@pytest.mark.gpu
def test_room_that_no_device_has_is_refused():
    """Before anything is read, allocated or launched: pointers are never followed."""
    from paper_2609_09020_gb300 import build, pic
    build.build()
    lib, h = pic.load_library(), ctypes.c_void_p()
    torch.zeros(1, device="cuda")
    for rows, cols in ((2 ** 31 - 1257, 1), (LARGE, 1), (LARGE, LARGE)):
        e = pic.pic_orth_matrix(P, P, rows, cols, cols, cols, BF16)
        assert lib.pic_orth_room_bytes(ctypes.byref(e), 1) > 400e9
        assert lib.pic_orth_create(ctypes.byref(e), 1, ctypes.byref(h)) == pic.PIC_ERR_ALLOC
        assert not h.value
