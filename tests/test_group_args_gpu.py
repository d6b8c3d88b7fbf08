"""What pic.grouped_linear and pic.grouped_linear_backward refuse of CUDA tensors."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pic():
    from paper_2609_09020_gb300 import build, pic
    build.build()
    return pic


def args(**kw):
    z = lambda *s, **o: torch.zeros(s, device="cuda", **o)
    a = dict(x=z(6, 8), weight=z(2, 3, 8), offsets=torch.tensor([0, 2, 6], device="cuda"), bias=z(2, 3))
    a.update(kw)
    return a


def bad_forward():
    z = lambda *s, **o: torch.zeros(s, device="cuda", **o)
    return [dict(x=z(6, 9)), dict(x=z(2, 3, 8)), dict(x=z(6, 8).half()), dict(x=z(6, 8).double()),
            dict(x=z(8, 6).t()), dict(x=z(6, 8).expand(6, 8)[:, :1].expand(6, 8)), dict(weight=z(3, 8)),
            dict(weight=z(2, 0, 8)), dict(weight=z(1, 3, 8).expand(2, 3, 8)), dict(weight=z(2, 8, 3).transpose(1, 2)),
            dict(weight=z(1025, 3, 8)), dict(offsets=torch.tensor([0, 6], device="cuda")),
            dict(offsets=torch.tensor([0, 2, 6], device="cuda", dtype=torch.int32)),
            dict(offsets=torch.tensor([0, 2, 6])), dict(bias=z(3)), dict(bias=z(1, 3).expand(2, 3)),
            dict(bias=z(2, 3).half()), dict(act="tanh"), dict(out=z(5, 3)), dict(out=z(6, 4)),
            dict(out=z(1, 3).expand(6, 3)), dict(weight=z(2, 3, 8).cpu())]


@pytest.mark.parametrize("i", range(len(bad_forward()) if torch.cuda.is_available() else 0))
def test_forward_refuses(pic, i):
    with pytest.raises(ValueError):
        pic.grouped_linear(**args(**bad_forward()[i]))


def test_backward_refuses(pic):
    z = lambda *s, **o: torch.zeros(s, device="cuda", **o)
    good = dict(dy=z(6, 3), x=z(6, 8), weight=z(2, 3, 8), offsets=torch.tensor([0, 2, 6], device="cuda"), act="relu",
                pre=z(6, 3))
    pic.grouped_linear_backward(**good)
    for bad in (dict(dy=z(6, 4)), dict(dy=z(5, 3)), dict(pre=None), dict(pre=z(6, 2)), dict(need=()), dict(need=("w",)),
                dict(dx=z(6, 7)), dict(dweight=z(2, 8, 3)), dict(dweight=z(1, 3, 8).expand(2, 3, 8)), dict(dbias=z(2, 4)),
                dict(dbias=z(1, 3).expand(2, 3)), dict(x=z(6, 8).bfloat16()), dict(offsets=z(3))):
        with pytest.raises(ValueError):
            pic.grouped_linear_backward(**{**good, **bad})


def test_tensors_that_require_gradients(pic):
    a = args()
    a["weight"].requires_grad_()
    with pytest.raises(ValueError, match="grouped_linear_backward"):
        pic.grouped_linear(**a)
    with torch.no_grad():
        assert pic.grouped_linear(**a).shape == (6, 3)
