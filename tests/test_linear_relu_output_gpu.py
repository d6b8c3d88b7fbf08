"""ReLU's gradient from the layer's output instead of its pre-activation: y has z's sign
wherever there is no residual, rounding included, and the gradients are the same bits."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16], ids=["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("M,K,N", [(3, 70, 50), (300, 200, 90), (5000, 64, 64)])
def test_output_for_pre(M, K, N, dtype):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_09020_gb300 import build, pic
    build.build()
    g = torch.Generator(device="cuda").manual_seed(1)
    x, w, dy = (torch.randn(s, generator=g, device="cuda").to(dtype) for s in ((M, K), (N, K), (M, N)))
    w *= 1e-4  # in fp16 some of z and y round to zero
    x[0] *= 1e-4
    y, z = pic.linear(x, w, act="relu", save_pre=True)
    a = pic.linear_backward(dy, x, w, act="relu", pre=z)
    b = pic.linear_backward(dy, x, w, act="relu", pre=y)
    assert all(torch.equal(u, v) for u, v in zip(a, b))
    pic.linear_check()
