"""Calls whose derivatives autograd would lose are refused: in reverse and forwards.
(Tensors on the CPU: what is refused for that says so.)"""
import pytest

torch = pytest.importorskip("torch")

from torch.autograd import forward_ad  # noqa: E402

LOST = "autograd does not"
CPU = "current CUDA device"


@pytest.fixture(scope="module")
def pic():
    from paper_2609_09020_gb300 import pic
    return pic


def arguments():
    z = torch.zeros
    offsets = torch.tensor([0, 2, 6])
    return {
        "linear": dict(x=z(6, 8), weight=z(3, 8), bias=z(3), residual=z(6, 3), out=z(6, 3)),
        "grouped_linear": dict(x=z(6, 8), weight=z(2, 3, 8), offsets=offsets, bias=z(2, 3), out=z(6, 3)),
        "grouped_linear_backward": dict(dy=z(6, 3), x=z(6, 8), weight=z(2, 3, 8), offsets=offsets, act="relu", pre=z(6, 3),
                                        dx=z(6, 8), dweight=z(2, 3, 8), dbias=z(2, 3)),
    }


CASES = [(f, k) for f, a in arguments().items() for k, t in a.items() if k not in ("offsets", "act")]


@pytest.mark.parametrize("name,which", [c for c in CASES if c[0] != "grouped_linear_backward"])
def test_reverse(pic, name, which):
    a, call = arguments()[name], getattr(pic, name)
    a[which].requires_grad_()
    with pytest.raises(ValueError, match=f"^{which}: requires a gradient.*{LOST}"):
        call(**a)
    with torch.no_grad(), pytest.raises(ValueError, match=CPU):
        call(**a)


@pytest.mark.parametrize("which", [w for n, w in CASES if n == "grouped_linear_backward"])
def test_gradients_of_what_is_recorded(pic, which):
    """Parameters may be given to it, results of recorded operations not."""
    a = arguments()["grouped_linear_backward"]
    leaf = a[which].requires_grad_()
    with pytest.raises(ValueError, match=CPU):
        pic.grouped_linear_backward(**a)
    a[which] = leaf * 2
    with pytest.raises(ValueError, match=f"^{which}: is part of a graph.*{LOST}"):
        pic.grouped_linear_backward(**a)
    with torch.no_grad(), pytest.raises(ValueError, match=CPU):
        pic.grouped_linear_backward(**a)


@pytest.mark.parametrize("name,which", CASES)
def test_forwards(pic, name, which):
    a, call = arguments()[name], getattr(pic, name)
    with forward_ad.dual_level():
        with pytest.raises(ValueError, match=CPU):  # no tensor has a tangent
            call(**a)
        a[which] = forward_ad.make_dual(a[which], torch.ones_like(a[which]))
        with pytest.raises(ValueError, match=f"^{which}: has a tangent.*{LOST}"):
            call(**a)
        with torch.no_grad(), pytest.raises(ValueError, match=f"^{which}: has a tangent"):
            call(**a)


def test_views_of_parameters(pic):
    """A layer's slice of a buffer of parameters is one; a slice of a result is not."""
    a = arguments()["grouped_linear_backward"]
    blob = torch.zeros(2, 3 * 8 + 3, requires_grad=True)
    weights = lambda t: t[:, :24].unflatten(1, (3, 8))
    a["weight"] = weights(blob)
    assert a["weight"].grad_fn is not None
    with pytest.raises(ValueError, match=CPU):
        pic.grouped_linear_backward(**a)
    a["weight"] = weights(blob * 2)
    with pytest.raises(ValueError, match="^weight: is part of a graph"):
        pic.grouped_linear_backward(**a)
    with pytest.raises(ValueError, match=CPU):
        pic.Orthogonalizer([weights(blob)])
    with pytest.raises(ValueError, match="is part of a graph"):
        pic.Orthogonalizer([weights(blob * 2)])


def test_a_second_derivative(pic):
    """Inside of an autograd.Function whose backward is itself recorded."""
    a = arguments()["grouped_linear_backward"]
    del a["dx"], a["dweight"], a["dbias"]

    class Layer(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x):
            return x.sum(1, keepdim=True).expand(6, 3).clone()

        @staticmethod
        def backward(ctx, dy):
            return pic.grouped_linear_backward(**{**a, "dy": dy})[0]

    x = torch.ones(6, 8, requires_grad=True)
    with pytest.raises(ValueError, match="^dy: is part of a graph"):
        torch.autograd.grad(Layer.apply(x).square().sum(), x, create_graph=True)
    with pytest.raises(ValueError, match=CPU):
        torch.autograd.grad(Layer.apply(x).square().sum(), x)


@pytest.mark.parametrize("which", ["tensors", "out"])
def test_orthogonalizer(pic, which):
    a = {"tensors": [torch.zeros(3, 3)], "out": [torch.zeros(3, 3)]}
    leaf = a[which][0].requires_grad_()
    with pytest.raises(ValueError, match=CPU):
        pic.Orthogonalizer(**a)
    a[which][0] = leaf * 2
    with pytest.raises(ValueError, match=rf"^{which}\[0\]: is part of a graph.*{LOST}"):
        pic.Orthogonalizer(**a)
    with torch.no_grad(), pytest.raises(ValueError, match=CPU):
        pic.Orthogonalizer(**a)
    with forward_ad.dual_level():
        a = {"tensors": [torch.zeros(3, 3)], "out": [torch.zeros(3, 3)]}
        a[which][0] = forward_ad.make_dual(a[which][0], torch.ones(3, 3))
        with pytest.raises(ValueError, match=rf"^{which}\[0\]: has a tangent"):
            pic.Orthogonalizer(**a)
