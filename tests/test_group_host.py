"""What pic.grouped_linear and pic.grouped_linear_backward refuse, without a GPU:
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
    a = pic.pic_grouped_linear_args()
    a.rows, a.in_features, a.out_features, a.groups = 8, 16, 24, 3
    a.dtype, a.act, a.offsets = pic.PIC_DTYPE_F16, pic.PIC_ACT_NONE, P
    a.x, a.ldx, a.w, a.ldw, a.w_group, a.y, a.ldy = P, 16, P, 16, 16 * 24, P + 4096, 24
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def backward_args(pic, **kw):
    a = pic.pic_grouped_linear_grad_args()
    a.rows, a.in_features, a.out_features, a.groups = 8, 16, 24, 3
    a.dtype, a.act, a.offsets = pic.PIC_DTYPE_F16, pic.PIC_ACT_GELU, P
    a.dy, a.lddy, a.x, a.ldx, a.w, a.ldw, a.w_group, a.pre, a.ldpre = P, 24, P, 16, P, 16, 16 * 24, P, 24
    a.dx, a.lddx, a.dw, a.lddw, a.dw_group, a.db, a.db_group = P + 4096, 16, P + 8192, 16, 16 * 24, P + 16384, 24
    for k, v in kw.items():
        setattr(a, k, v)
    return a


BAD_SIZES = [dict(rows=-1), dict(rows=2**31), dict(in_features=0), dict(out_features=0), dict(groups=0),
             dict(groups=1025), dict(groups=-1), dict(dtype=3), dict(act=3), dict(act=-1), dict(offsets=None),
             dict(offsets=P + 4)]
BAD_FORWARD = BAD_SIZES + [dict(x=None), dict(w=None), dict(y=None), dict(ldx=15), dict(ldw=15), dict(ldy=23),
                           dict(x=P + 1), dict(w=P + 1), dict(y=P + 1), dict(w_group=16 * 24 - 1), dict(w_group=0),
                           dict(bias=P, bias_group=23), dict(bias=P + 1, bias_group=24), dict(pre=P, ldpre=23),
                           dict(pre=P + 1, ldpre=24), dict(dtype=0, x=P + 2), dict(ldx=2**41), dict(w_group=2**45)]
BAD_BACKWARD = BAD_SIZES + [dict(dy=None), dict(x=None), dict(w=None), dict(pre=None), dict(dx=None, dw=None, db=None),
                            dict(lddy=23), dict(ldpre=23), dict(lddx=15), dict(lddw=15), dict(ldx=15), dict(ldw=15),
                            dict(dw_group=16 * 24 - 1), dict(w_group=16 * 24 - 1), dict(db_group=23), dict(db=P + 1),
                            dict(dx=P + 1), dict(dw=P + 1), dict(dy=P + 1), dict(pre=P + 1)]


@pytest.mark.parametrize("bad", BAD_FORWARD, ids=str)
def test_forward_refuses(pic, bad):
    lib = pic.load_library()
    a = forward_args(pic, **bad)
    assert lib.pic_grouped_linear_workspace_bytes(ctypes.byref(a)) == -1
    assert lib.pic_grouped_linear(ctypes.byref(a), P, 1 << 40, None) == pic.PIC_ERR_INVALID_ARG


@pytest.mark.parametrize("bad", BAD_BACKWARD, ids=str)
def test_backward_refuses(pic, bad):
    lib = pic.load_library()
    a = backward_args(pic, **bad)
    assert lib.pic_grouped_linear_backward_workspace_bytes(ctypes.byref(a)) == -1
    assert lib.pic_grouped_linear_backward(ctypes.byref(a), P, 1 << 40, None) == pic.PIC_ERR_INVALID_ARG


def test_null(pic):
    lib = pic.load_library()
    assert lib.pic_grouped_linear_workspace_bytes(None) == -1
    assert lib.pic_grouped_linear(None, None, 0, None) == pic.PIC_ERR_INVALID_ARG
    assert lib.pic_grouped_linear_backward(None, None, 0, None) == pic.PIC_ERR_INVALID_ARG


def test_good_arguments_are_counted(pic):
    lib = pic.load_library()
    for kw in (dict(), dict(groups=1, w_group=0), dict(rows=0, x=None, y=None), dict(w_group=5000, ldw=40),
               dict(bias=P, bias_group=24), dict(groups=1024)):
        assert lib.pic_grouped_linear_workspace_bytes(ctypes.byref(forward_args(pic, **kw))) >= 0
    for kw in (dict(), dict(act=2, pre=None), dict(dx=None, w=None), dict(dw=None, x=None), dict(db=None),
               dict(rows=0), dict(groups=1, w_group=0, dw_group=0, db_group=0)):
        assert lib.pic_grouped_linear_backward_workspace_bytes(ctypes.byref(backward_args(pic, **kw))) >= 0


def test_a_workspace_that_is_too_small_is_refused(pic):
    lib = pic.load_library()
    big = dict(rows=100000, in_features=512, out_features=512, groups=1, x=P, ldx=512, w=P, ldw=512, w_group=0, dy=P,
               lddy=512, pre=P, ldpre=512, lddx=512, lddw=512)
    a = backward_args(pic, **big)
    need = lib.pic_grouped_linear_backward_workspace_bytes(ctypes.byref(a))
    if need > 0:
        assert lib.pic_grouped_linear_backward(ctypes.byref(a), P, need - 1, None) == pic.PIC_ERR_INVALID_ARG
        assert lib.pic_grouped_linear_backward(ctypes.byref(a), P + 16, need, None) == pic.PIC_ERR_INVALID_ARG
        assert lib.pic_grouped_linear_backward(ctypes.byref(a), None, need, None) == pic.PIC_ERR_INVALID_ARG


def test_packed_arguments_have_the_structures_sizes(pic):
    assert pic._GROUPED_ARGS.size == ctypes.sizeof(pic.pic_grouped_linear_args)
    assert pic._GROUPED_GRAD_ARGS.size == ctypes.sizeof(pic.pic_grouped_linear_grad_args)


def test_cpu_tensors_are_refused(pic):
    x, w = torch.zeros(4, 8), torch.zeros(2, 3, 8)
    o = torch.zeros(3, dtype=torch.int64)
    with pytest.raises(ValueError):
        pic.grouped_linear(x, w, o)
    with pytest.raises(ValueError):
        pic.grouped_linear_backward(torch.zeros(4, 3), x, w, o)
    with pytest.raises(ValueError, match="requires a gradient"):
        pic.grouped_linear(x.requires_grad_(), w, o)
