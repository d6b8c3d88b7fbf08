"""First calls of the linear layer from two threads: the tables of types and of C
functions that a first call makes are seen whole or not at all.  The second thread's
call is made where the first is in the middle of making the table."""
import ctypes

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture
def pic():
    from paper_2609_09020_gb300 import build, pic
    build.build()
    pic.load_library()
    return pic


def test_dtype_codes(pic, monkeypatch):
    second = []

    class Slow(dict):
        def items(self):
            for i, item in enumerate(super().items()):
                if i == 1 and not second:
                    second.append(None)  # the second thread's call, which finds the first entry made
                    second[0] = pic._dtype_code(torch.zeros(1, dtype=torch.bfloat16), "t")
                yield item

    monkeypatch.setattr(pic, "DTYPES", Slow(pic.DTYPES))
    monkeypatch.setattr(pic, "_dtype_codes", type(pic._dtype_codes)() if pic._dtype_codes is not None else None)
    assert pic._dtype_code(torch.zeros(1, dtype=torch.float16), "t") == pic.PIC_DTYPE_F16
    assert second == [pic.PIC_DTYPE_BF16]
    for t, code in ((torch.float32, pic.PIC_DTYPE_F32), (torch.float16, pic.PIC_DTYPE_F16), (torch.bfloat16, pic.PIC_DTYPE_BF16)):
        assert pic._dtype_code(torch.zeros(1, dtype=t), "t") == code
    with pytest.raises(ValueError):
        pic._dtype_code(torch.zeros(1, dtype=torch.float64), "t")


def test_c_functions(pic, monkeypatch):
    make, second = ctypes.CFUNCTYPE, []

    def slow(*types):
        kind = make(*types)

        def create(what):
            f = kind(what)
            if what[0] == "pic_linear_backward" and not second:
                second.append(None)  # the second thread's call, while the first has made pic_linear's
                second[0] = refused(pic, "pic_linear_backward")
            return f
        return create

    monkeypatch.setattr(pic.ctypes, "CFUNCTYPE", slow)
    monkeypatch.setattr(pic, "_linear_calls", type(pic._linear_calls)() if pic._linear_calls is not None else None)
    monkeypatch.setattr(pic, "_current_stream", lambda: 0)
    assert refused(pic, "pic_linear") == pic.PIC_ERR_INVALID_ARG
    assert second == [pic.PIC_ERR_INVALID_ARG]


def refused(pic, name):
    """The status with which the C function refuses arguments of zeros."""
    size = ctypes.sizeof(pic.pic_linear_args if name == "pic_linear" else pic.pic_linear_grad_args)
    with pytest.raises(pic.PicError) as e:
        pic._call_with_workspace(name, bytes(size), torch, "cpu")
    return e.value.status
