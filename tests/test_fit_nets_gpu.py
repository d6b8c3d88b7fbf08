"""The example that trains several images' nets at once with the grouped layers, their
gradient, clipping and orthogonalised updates: it runs, the decoder's images are the nets'
own outputs, and one step's gradients are those of fp64 autograd and of the single-net example."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_09020_gb300 import build
    build.build()


@pytest.mark.parametrize("dims,act", [((7, 64, 64, 3), "relu"), ((4, 16, 16, 3), "gelu"), ((5, 40, 24, 40, 3), "gelu")])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16], ids=["fp32", "fp16", "bf16"])
def test_fit_and_decode(dims, act, dtype):
    from paper_2609_09020_gb300 import fit_net
    H, W, L, images = 40, 52, dims[0], 5
    latents, steps, x, target, offsets = fit_net.problems(dims, act, H, W, L, 1, images)
    nets = fit_net.Nets(dims, act, dtype, images, seed=1)
    before = nets.master.clone()
    losses = fit_net.fit_many(nets, x.to(dtype), target, offsets, 30)
    assert losses.shape == (30, images) and torch.isfinite(losses).all()
    assert torch.isfinite(nets.master).all() and bool((nets.master != before).any(1).all())
    # the decoder runs the same nets: fp32 sums of other order, features rounded to
    # the training type (half an ulp of up to 32 through a net of gain of order 10)
    y, _ = nets.forward(x.to(dtype), offsets)
    got = fit_net.decode_many(nets, latents, steps, H, W, L, 1)
    bar = {torch.float32: 1e-4, torch.float16: 0.1, torch.bfloat16: 0.8}[dtype]
    assert float((got - y.float().clamp(0, 1)).abs().max()) <= bar


def test_gradients_are_autograds():
    from paper_2609_09020_gb300 import fit_net
    dims, images = (7, 64, 64, 3), 3
    _, _, x, target, _ = fit_net.problems(dims, "gelu", 40, 56, 7, 1, images)
    offsets = [0, 2240, 2300, 6720]  # the images' pixels shared out unevenly
    o = torch.tensor(offsets, device="cuda")
    nets = fit_net.Nets(dims, "gelu", torch.float32, images, seed=3)
    y, kept = nets.forward(x, o)
    nets.backward((y - target) * (2.0 / y.numel()), kept, o)
    p = nets.params.double().requires_grad_(True)
    loss = 0.0
    for g, (i, j) in enumerate(zip(offsets, offsets[1:])):
        h = x[i:j].double()
        layers = nets.layers(p)
        for n, (w, b) in enumerate(layers):
            h = torch.nn.functional.linear(h, w[g], b[g])
            if n + 1 < len(layers):
                h = torch.nn.functional.gelu(h)
        loss = loss + (h - target[i:j].double()).square().sum() / y.numel()
    loss.backward()
    for g in range(images):
        # fp32 sums over up to 4420 pixels and three layers: 2^-24 times a few hundred roundings
        assert float((nets.grads[g] - p.grad[g]).norm() / p.grad[g].norm()) < 2e-5


def test_one_net_is_the_single_example():
    from paper_2609_09020_gb300 import fit_net
    dims = (7, 64, 64, 3)
    _, _, x, target, offsets = fit_net.problems(dims, "relu", 40, 56, 7, 1, 1)
    nets, net = fit_net.Nets(dims, "relu", torch.float32, 1, seed=3), fit_net.Net(dims, "relu", torch.float32, seed=3)
    assert torch.equal(nets.params[0], net.params)
    y, kept = nets.forward(x, offsets)
    z, kept1 = net.forward(x)
    dy = (y - target) * (2.0 / y.numel())
    nets.backward(dy, kept, offsets)
    net.backward(dy, kept1)
    assert float((y - z).abs().max()) <= 1e-4
    assert float((nets.grads[0] - net.grads).norm() / net.grads.norm()) < 4e-5


def test_command(capsys):
    from paper_2609_09020_gb300 import fit_net
    fit_net.main(["--steps", "40", "--size", "48x64", "--net", "4-16-16-3", "--images", "4"])
    assert "PSNR" in capsys.readouterr().out
