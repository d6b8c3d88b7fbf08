"""Matrices whose last element no address reaches, without a GPU: products of rows and
distances that leave 64 bits do not come back as small ones."""
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
FAR = [(2 ** 24 + 1, 2 ** 40), (2 ** 25 + 1, 2 ** 39), (2 ** 30 + 1, 2 ** 34), (2 ** 30 + 1, 2 ** 40)]  # (rows - 1) * distance is a multiple of 2^64


def grouped(pic, rows, ld, groups=2):
    a = pic.pic_grouped_linear_args()
    a.rows, a.in_features, a.out_features, a.groups = 8, 16, rows, groups
    a.dtype, a.act, a.offsets = pic.PIC_DTYPE_F16, pic.PIC_ACT_NONE, P
    a.x, a.ldx, a.w, a.ldw, a.w_group, a.y, a.ldy = P, 16, P, ld, 2 ** 44, P, rows
    return pic.load_library().pic_grouped_linear_workspace_bytes(ctypes.byref(a))


@pytest.mark.parametrize("rows,ld", FAR, ids=str)
def test_weights(pic, rows, ld):
    assert grouped(pic, rows, ld) == -1
    assert grouped(pic, rows, ld, groups=1) == -1


def test_weights_as_far_apart_as_can_be(pic):
    assert grouped(pic, 2 ** 4 + 1, 2 ** 39) >= 0
    assert grouped(pic, 1, 2 ** 40) >= 0


@pytest.mark.parametrize("rows,ld", FAR, ids=str)
def test_weight_gradients(pic, rows, ld):
    a = pic.pic_grouped_linear_grad_args()
    a.rows, a.in_features, a.out_features, a.groups = 8, 16, rows, 2
    a.dtype, a.act, a.offsets = pic.PIC_DTYPE_F32, pic.PIC_ACT_NONE, P
    a.dy, a.lddy, a.x, a.ldx, a.dw, a.lddw, a.dw_group = P, rows, P, 16, P, ld, 2 ** 44
    assert pic.load_library().pic_grouped_linear_backward_workspace_bytes(ctypes.byref(a)) == -1


@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("rows,ld", FAR, ids=str)
def test_updates(pic, rows, ld, dtype):
    """Their ends would wrap to before their beginnings, and what they overlap would pass."""
    inside = P + 64
    make = lambda *m: (pic.pic_orth_matrix * len(m))(*m)
    room = pic.load_library().pic_orth_room_bytes
    far = pic.pic_orth_matrix(P, P, rows, 16, ld, ld, dtype)
    assert room(make(far), 1) == -1
    assert room(make(pic.pic_orth_matrix(inside, inside, 4, 4, 4, 4, dtype), far), 2) == -1
