"""What pic.linear, pic.linear_backward and pic.GradClip refuse, without a GPU:
the C entry points return before they touch a device."""
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


def forward_args(pic, **kw):
    a = pic.pic_linear_args()
    a.rows, a.in_features, a.out_features, a.dtype, a.act = 8, 16, 24, pic.PIC_DTYPE_F16, pic.PIC_ACT_NONE
    a.x, a.ldx, a.w, a.ldw, a.y, a.ldy = P, 16, P, 16, P + 4096, 24
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def backward_args(pic, **kw):
    a = pic.pic_linear_grad_args()
    a.rows, a.in_features, a.out_features, a.dtype, a.act = 8, 16, 24, pic.PIC_DTYPE_F16, pic.PIC_ACT_GELU
    a.dy, a.lddy, a.x, a.ldx, a.w, a.ldw, a.pre, a.ldpre = P, 24, P, 16, P, 16, P, 24
    a.dx, a.lddx, a.dw, a.lddw, a.db = P + 4096, 16, P + 8192, 16, P + 16384
    for k, v in kw.items():
        setattr(a, k, v)
    return a


BAD_FORWARD = [dict(rows=-1), dict(in_features=0), dict(out_features=0), dict(rows=2**31), dict(dtype=3),
               dict(dtype=-1), dict(act=3), dict(act=-1), dict(x=None), dict(w=None), dict(y=None), dict(ldx=15),
               dict(ldw=15), dict(ldy=23), dict(x=P + 1), dict(w=P + 1), dict(y=P + 1), dict(bias=P + 1),
               dict(residual=P, ldr=23), dict(residual=P + 1, ldr=24), dict(residual=P + 4096, ldr=25),
               dict(pre=P, ldpre=23), dict(pre=P + 1, ldpre=24), dict(dtype=0, x=P + 2), dict(ldx=2**41)]
BAD_BACKWARD = [dict(rows=-1), dict(in_features=0), dict(out_features=0), dict(dtype=7), dict(act=9), dict(dy=None),
                dict(x=None), dict(w=None), dict(pre=None), dict(dx=None, dw=None, db=None), dict(lddy=23),
                dict(ldpre=23), dict(lddx=15), dict(lddw=15), dict(ldx=15), dict(ldw=15), dict(db=P + 1),
                dict(dx=P + 1), dict(dw=P + 1), dict(dy=P + 1), dict(pre=P + 1)]


@pytest.mark.parametrize("bad", BAD_FORWARD, ids=str)
def test_forward_refuses(pic, bad):
    lib = pic.load_library()
    a = forward_args(pic, **bad)
    assert lib.pic_linear_workspace_bytes(ctypes.byref(a)) == -1
    assert lib.pic_linear(ctypes.byref(a), P, 1 << 30, None) == pic.PIC_ERR_INVALID_ARG


@pytest.mark.parametrize("bad", BAD_BACKWARD, ids=str)
def test_backward_refuses(pic, bad):
    lib = pic.load_library()
    a = backward_args(pic, **bad)
    assert lib.pic_linear_backward_workspace_bytes(ctypes.byref(a)) == -1
    assert lib.pic_linear_backward(ctypes.byref(a), P, 1 << 30, None) == pic.PIC_ERR_INVALID_ARG


def test_null_and_small_workspace(pic):
    lib = pic.load_library()
    assert lib.pic_linear_workspace_bytes(None) == -1
    assert lib.pic_linear(None, None, 0, None) == pic.PIC_ERR_INVALID_ARG
    a = backward_args(pic, rows=100)  # a few rows need none
    need = lib.pic_linear_backward_workspace_bytes(ctypes.byref(a))
    assert need > 0
    for ws, n in ((P, need - 1), (None, need), (P + 128, need)):
        assert lib.pic_linear_backward(ctypes.byref(a), ws, n, None) == pic.PIC_ERR_INVALID_ARG


def test_parts_that_are_not_asked_for_need_no_inputs(pic):
    lib = pic.load_library()
    ok = backward_args(pic, dx=None, w=None)
    assert lib.pic_linear_backward_workspace_bytes(ctypes.byref(ok)) >= 0
    ok = backward_args(pic, dw=None, x=None, act=pic.PIC_ACT_NONE, pre=None)
    assert lib.pic_linear_backward_workspace_bytes(ctypes.byref(ok)) >= 0


def table(pic, *rows):
    t = (pic.pic_clip_tensor * max(len(rows), 1))()
    for i, r in enumerate(rows):
        t[i] = pic.pic_clip_tensor(*r)
    return t


BAD_CLIP = [[(None, P, 4, 0)], [(P, None, 4, 0)], [(P, P, -1, 0)], [(P, P, 4, 3)], [(P + 2, P + 2, 4, 0)],
            [(P + 1, P + 1, 4, 1)], [(P, P + 8, 4, 0)], [(P, P, 4, 0), (P + 8, P + 8, 4, 0)],
            [(P, P + 4096, 4, 0), (P + 64, P + 4096, 4, 0)], [(P, P + 4096, 4, 0), (P + 4096, P + 8192, 4, 0)]]


@pytest.mark.parametrize("rows", BAD_CLIP, ids=range(len(BAD_CLIP)))
def test_clip_refuses(pic, rows):
    lib, h = pic.load_library(), ctypes.c_void_p()
    rc = lib.pic_clip_create(table(pic, *rows), len(rows), ctypes.byref(h))
    if torch.cuda.is_available():
        assert rc == pic.PIC_ERR_INVALID_ARG
    else:
        assert rc in (pic.PIC_ERR_INVALID_ARG, pic.PIC_ERR_UNSUPPORTED)  # overlap is looked for on a device
    assert not h.value


def test_clip_null_arguments(pic):
    lib, h = pic.load_library(), ctypes.c_void_p()
    assert lib.pic_clip_create(None, 1, ctypes.byref(h)) == pic.PIC_ERR_INVALID_ARG
    assert lib.pic_clip_create(None, -1, ctypes.byref(h)) == pic.PIC_ERR_INVALID_ARG
    assert lib.pic_clip_create(None, 0, None) == pic.PIC_ERR_INVALID_ARG
    assert lib.pic_clip(None, 1.0, P, None) == pic.PIC_ERR_INVALID_ARG
    lib.pic_clip_destroy(None)


def test_python_refuses_cpu_tensors(pic):
    x, w = torch.zeros(2, 4), torch.zeros(3, 4)
    with pytest.raises((ValueError, RuntimeError, AssertionError)):
        pic.linear(x, w)
    with pytest.raises((ValueError, RuntimeError, AssertionError)):
        pic.linear_backward(torch.zeros(2, 3), x, w)
    with pytest.raises((ValueError, RuntimeError, AssertionError)):
        pic.GradClip([x])


def test_rows_describes_matrices(pic):
    like = torch.zeros(1, dtype=torch.float16)
    t = torch.zeros(6, 10, dtype=torch.float16)
    assert pic._rows(t, "t", 10, like) == (t.data_ptr(), 10)
    assert pic._rows(t[:, 2:7], "t", 5, like) == (t.data_ptr() + 4, 10)
    assert pic._rows(t[::2], "t", 10, like)[1] == 20
    assert pic._rows(t[3], "t", 10, like, 1) == (t.data_ptr() + 60, 10)
    assert pic._rows(t.view(2, 3, 10), "t", 10, like, 6)[1] == 10
    assert pic._rows(t[:1].expand(4, 10), "t", 10, like, 4, one_row=True)[1] == 0
    for bad in (t.t(), t[:, ::2], t[:1].expand(4, 10), t.view(2, 3, 10)[:, :2], t.float()):
        with pytest.raises(ValueError):
            pic._rows(bad, "t", bad.shape[-1], like)
    with pytest.raises(ValueError):
        pic._rows(t, "t", 11, like)
    with pytest.raises(ValueError):
        pic._rows(t, "t", 10, like, rows=5)


def test_packed_arguments_are_the_structures(pic):
    a = forward_args(pic, bias=P + 64, residual=P + 128, ldr=24, pre=P + 192, ldpre=25)
    b = bytes(pic._LINEAR_ARGS.pack(8, 16, 24, pic.PIC_DTYPE_F16, pic.PIC_ACT_NONE, P, 16, P, 16, P + 64, P + 128, 24,
                                    P + 4096, 24, P + 192, 25))
    assert b == bytes(a) and len(b) == ctypes.sizeof(a)
    a = backward_args(pic)
    b = bytes(pic._LINEAR_GRAD_ARGS.pack(8, 16, 24, pic.PIC_DTYPE_F16, pic.PIC_ACT_GELU, P, 24, P, 16, P, 16, P, 24,
                                         P + 4096, 16, P + 8192, 16, P + 16384))
    assert b == bytes(a) and len(b) == ctypes.sizeof(a)
