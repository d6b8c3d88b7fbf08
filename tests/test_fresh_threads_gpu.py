"""Calls whose first contact with CUDA, in a thread that has just begun, is their own:
nothing has made the device's context current there."""
import threading

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pic():
    from paper_2609_09020_gb300 import build, pic
    build.build()
    return pic


def in_a_thread(f):
    """f's error, if it has one, in a thread of its own."""
    errors = []

    def run():
        try:
            f()
        except BaseException as e:  # noqa: BLE001
            errors.append(e)

    t = threading.Thread(target=run)
    t.start()
    t.join()
    if errors:
        raise errors[0]


def normal(shape, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").mul_(0.1).to(dtype)


@pytest.mark.parametrize("rows,K,N", [(3000, 512, 1024), (300, 512, 1024), (100, 512, 256), (20000, 64, 64)], ids=str)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=str)
def test_layers(pic, rows, K, N, dtype):
    """Outputs given, and memory for workspaces there already: the first CUDA call of the thread is the layer's."""
    x, w, dy = normal((rows, K), dtype, 0), normal((2, N, K), dtype, 1), normal((rows, N), dtype, 2)
    o = torch.tensor([0, rows // 3, rows], device="cuda")
    out, dx, dw, db = torch.empty_like(dy), torch.empty_like(x), torch.empty_like(w), torch.empty((2, N), dtype=dtype, device="cuda")
    single = torch.empty_like(dy)
    calls = [(lambda: pic.grouped_linear(x, w, o, out=out), [out]),
             (lambda: pic.grouped_linear_backward(dy, x, w, o, dx=dx, dweight=dw, dbias=db), [dx, dw, db]),
             (lambda: pic.linear(x, w[0], out=single), [single]),
             (lambda: pic.linear_backward(dy, x, w[0], dx=dx, dweight=dw[0], dbias=db[0]), [dx, dw[0], db[0]])]
    for call, outputs in calls:
        call()
        torch.cuda.synchronize()
        want = [t.clone() for t in outputs]
        for t in outputs:
            t.zero_()
        torch.cuda.synchronize()
        in_a_thread(call)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outputs, want))
    pic.grouped_linear_check()


@pytest.mark.parametrize("shape", [(64, 64), (300, 400)], ids=str)
def test_updates(pic, shape):
    g, out = normal(shape, torch.float32, 0), torch.zeros(shape, device="cuda")
    h = pic.Orthogonalizer([g], out=[out])
    h.orthogonalize()
    torch.cuda.synchronize()
    want = out.clone()
    out.zero_()
    torch.cuda.synchronize()
    in_a_thread(h.orthogonalize)
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    out.zero_()
    made = []
    in_a_thread(lambda: made.append(pic.Orthogonalizer([g], out=[out])))
    in_a_thread(made[0].orthogonalize)
    in_a_thread(made[0].check)
    assert torch.equal(out, want)
    in_a_thread(made[0].close)
    h.close()


@pytest.mark.parametrize("precision,dims", [("fp32", (4, 16, 16, 3)), ("fp16_tc", (7, 64, 64, 3))])
def test_decoder(pic, precision, dims):
    """A decoder made in one thread, used in another and closed in a third."""
    from paper_2609_09020_gb300 import workloads as wk
    H, W, L = 48, 64, dims[0]
    inputs = wk.make_inputs(wk.custom("threads", H=H, W=W, L=L, C=1, dims=dims, act="relu", seed=0))
    put = lambda a: torch.from_numpy(a).cuda()
    latents, steps, blob = put(inputs.latents), put(inputs.steps), put(inputs.weights_for(precision))
    rgb = torch.zeros((1, 3, H, W), device="cuda")
    want = torch.zeros_like(rgb)
    dec = pic.Decoder(L, 1, dims, "relu", precision, max_H=H, max_W=W)
    dec.decode(latents, steps, blob, H, W, want)
    dec.check()
    torch.cuda.synchronize()
    in_a_thread(lambda: dec.decode(latents, steps, blob, H, W, rgb))
    torch.cuda.synchronize()
    assert torch.equal(rgb, want)
    made = []
    rgb.zero_()
    torch.cuda.synchronize()
    in_a_thread(lambda: made.append(pic.Decoder(L, 1, dims, "relu", precision, max_H=H, max_W=W)))
    in_a_thread(lambda: made[0].decode(latents, steps, blob, H, W, rgb))
    in_a_thread(made[0].check)
    assert torch.equal(rgb, want)
    in_a_thread(made[0].close)
    dec.close()
