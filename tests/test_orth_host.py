"""What pic_orth_create refuses without a GPU, and that the bounds of orth_ref hold
what the described arithmetic loses (on the CPU)."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

import orth_ref as ref


@pytest.fixture(scope="module")
def pic():
    from paper_2609_09020_gb300 import build, pic
    build.build()
    pic.load_library()
    return pic


P = 0x10000  # never followed


def matrix(pic, **kw):
    m = pic.pic_orth_matrix(P, P + 65536, 8, 16, 16, 16, pic.PIC_DTYPE_F16)
    for k, v in kw.items():
        setattr(m, k, v)
    return m


BAD = [dict(grad=None), dict(out=None), dict(grad=P + 1), dict(out=P + 1), dict(dtype=3), dict(dtype=-1), dict(rows=-1),
       dict(cols=-1), dict(rows=2**31), dict(ld_grad=15), dict(ld_out=15), dict(ld_grad=2**41), dict(dtype=0, grad=P + 2),
       dict(out=P + 2), dict(out=P, ld_out=17)]


@pytest.mark.parametrize("bad", BAD, ids=str)
def test_create_refuses(pic, bad):
    h = ctypes.c_void_p()
    assert pic.load_library().pic_orth_create((pic.pic_orth_matrix * 1)(matrix(pic, **bad)), 1,
                                              ctypes.byref(h)) == pic.PIC_ERR_INVALID_ARG
    assert not h.value


def test_overlaps(pic):
    lib, h = pic.load_library(), ctypes.c_void_p()
    make = lambda *m: lib.pic_orth_create((pic.pic_orth_matrix * len(m))(*m), len(m), ctypes.byref(h))
    far = 1 << 20
    for other in (dict(out=P + 65536), dict(out=P + 65536 + 2 * 127), dict(out=P), dict(out=P + 2 * 127),
                  dict(grad=P + 65536)):
        assert make(matrix(pic), matrix(pic, **{"grad": P + far, "out": P + 2 * far, **other})) == pic.PIC_ERR_INVALID_ARG
    # columns of one buffer side by side do not overlap; by one column they do
    side = dict(ld_grad=40, ld_out=40)
    first = matrix(pic, grad=P, out=P, **side)
    for cols, ok in ((16, True), (15, False), (24, True), (25, False)):
        rc = make(first, matrix(pic, grad=P + 2 * cols, out=P + 2 * cols, **side))
        assert (rc != pic.PIC_ERR_INVALID_ARG) == ok, cols
        lib.pic_orth_destroy(h)  # where there is a device
    assert lib.pic_orth_create(None, 1, ctypes.byref(h)) == pic.PIC_ERR_INVALID_ARG
    assert lib.pic_orth_create(None, 0, None) == pic.PIC_ERR_INVALID_ARG
    assert lib.pic_orth_create(None, -1, ctypes.byref(h)) == pic.PIC_ERR_INVALID_ARG


def test_null_handle(pic):
    lib = pic.load_library()
    assert lib.pic_orth(None, 5, 1.0, 0.0, 0.0, 0.0, None) == pic.PIC_ERR_INVALID_ARG
    assert lib.pic_orth_check(None, None) == pic.PIC_ERR_INVALID_ARG
    lib.pic_orth_destroy(None)


def test_emulation_is_near():
    """Five steps in the described arithmetic: within 1e-5 with two halves, 5e-3 with one, of mean size."""
    g = torch.randn(96, 160, generator=torch.Generator().manual_seed(0))
    for dtype, most in ((torch.float32, 1e-5), (torch.float16, 1e-5), (torch.bfloat16, 5e-3)):
        t = g.to(dtype)
        want = ref.exact(t)
        d = ref.emulated(t) - want
        assert float(d.square().mean().sqrt() / want.square().mean().sqrt()) <= most


def test_singular_values_come_to_one():
    s = torch.linalg.svdvals(ref.exact(torch.randn(60, 90, generator=torch.Generator().manual_seed(1))))
    assert 0.6 < float(s.min()) and float(s.max()) < 1.3
