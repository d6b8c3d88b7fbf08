"""pic.linear is not part of torch's graph: a tensor that requires a gradient is refused
while autograd records, instead of being cut out of the graph without a word."""
import pytest

torch = pytest.importorskip("torch")


def tensors(device="cpu"):
    g = torch.Generator(device=device).manual_seed(1)
    make = lambda *shape: torch.randn(shape, generator=g, device=device)
    return {"x": make(5, 8), "weight": make(6, 8), "bias": make(6), "residual": make(5, 6), "out": make(5, 6)}


@pytest.mark.parametrize("name", ["x", "weight", "bias", "residual", "out"])
def test_refused_while_recording(name):
    from paper_2609_09020_gb300 import pic
    t = tensors()
    t[name].requires_grad_()
    with pytest.raises(ValueError, match=f"^{name}: requires a gradient"):
        pic.linear(**t)
    with torch.no_grad(), pytest.raises((ValueError, RuntimeError, AssertionError)) as e:  # no GPU here, or no CUDA tensor
        pic.linear(**t)
    assert "requires a gradient" not in str(e.value)


@pytest.mark.gpu
def test_taken_where_nothing_is_recorded():
    from paper_2609_09020_gb300 import build, pic
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build()
    t = tensors("cuda")
    del t["out"]
    want = pic.linear(**t)
    w = torch.nn.Parameter(t["weight"])
    with torch.no_grad():
        assert torch.equal(pic.linear(**{**t, "weight": w}), want)
    with torch.inference_mode():
        assert torch.equal(pic.linear(**{**t, "weight": w}), want)
    assert torch.equal(pic.linear(**{**t, "weight": w.detach()}), want)
    with pytest.raises(ValueError):
        pic.linear(**{**t, "weight": w})
    # gradients of parameters are taken outside the graph
    dx, dw, db = pic.linear_backward(want, t["x"], w)
    assert not dw.requires_grad and dw.shape == w.shape
