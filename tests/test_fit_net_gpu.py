"""The example that trains a synthesis net with the linear layer, its gradient and
gradient clipping: the loss falls, the decoder's image of the trained net is the
net's own output, and one step's gradients are those of fp64 autograd."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_09020_gb300 import build
    build.build()


@pytest.mark.parametrize("dims,act", [((7, 64, 64, 3), "relu"), ((4, 16, 16, 3), "relu"), ((7, 40, 40, 3), "gelu")])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16], ids=["fp32", "fp16", "bf16"])
def test_fit_and_decode(dims, act, dtype):
    from paper_2609_09020_gb300 import fit_net
    H, W, L = 72, 100, dims[0]
    latents, steps, x, target = fit_net.problem(dims, act, H, W, L, 1)
    net = fit_net.Net(dims, act, dtype, seed=1)
    losses = fit_net.fit(net, x.to(dtype), target, 120)
    assert all(l == l for l in losses) and losses[-1] < 0.2 * losses[0]
    # the decoder runs the same net: fp32 sums of other order, features rounded to
    # the training type (half an ulp of up to 32 through a net of gain of order 10)
    y, _ = net.forward(x.to(dtype))
    got = fit_net.decode(net, latents, steps, H, W, L, 1)
    bar = {torch.float32: 1e-4, torch.float16: 0.1, torch.bfloat16: 0.8}[dtype]
    assert float((got - y.float().clamp(0, 1)).abs().max()) <= bar


def test_gradients_are_autograds():
    from paper_2609_09020_gb300 import fit_net
    dims = (7, 64, 64, 3)
    _, _, x, target = fit_net.problem(dims, "gelu", 40, 56, 7, 1)
    net = fit_net.Net(dims, "gelu", torch.float32, seed=3)
    y, kept = net.forward(x)
    net.backward((y - target) * (2.0 / y.numel()), kept)
    p = net.params.double().requires_grad_(True)
    h = x.double()
    layers = net.layers(p)
    for i, (w, b) in enumerate(layers):
        h = torch.nn.functional.linear(h, w, b)
        if i + 1 < len(layers):
            h = torch.nn.functional.gelu(h)
    (h - target.double()).square().mean().backward()
    # fp32 sums over 2240 pixels and three layers: 2^-24 times a few hundred roundings
    assert float((net.grads - p.grad).norm() / p.grad.norm()) < 2e-5


def test_command(capsys):
    from paper_2609_09020_gb300 import fit_net
    fit_net.main(["--steps", "40", "--size", "48x64", "--net", "4-16-16-3"])
    assert "PSNR" in capsys.readouterr().out
