"""The bounded waits of the grouped layers' and the orthogonalised updates' kernels,
made to run out on purpose (as test_linear_wait_gpu.py's): said once, and the next
call is right."""
import math

import pytest

torch = pytest.importorskip("torch")

import group_ref  # noqa: E402
import linear_ref as ref  # noqa: E402
import orth_ref  # noqa: E402

pytestmark = pytest.mark.gpu
SHORT_LIMIT = 1 << 10


@pytest.fixture(scope="module")
def pic():
    from paper_2609_09020_gb300 import build, pic
    build.build()
    return pic


def normal(shape, dtype, seed, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").mul_(std).to(dtype)


H, F, B = torch.float16, torch.float32, torch.bfloat16


def timed_out(pic, call, check):
    lib = pic.load_library()
    torch.cuda.synchronize()
    assert lib.pic_linear_test_wait_fault(1, SHORT_LIMIT) == pic.PIC_OK
    try:
        call()
        torch.cuda.synchronize()
    finally:
        lib.pic_linear_test_wait_fault(0, 0)
    with pytest.raises(pic.PicError) as e:
        check()
    assert e.value.status == pic.PIC_ERR_TIMEOUT
    check()  # said once


# several tiles for a CTA: tiles of 64, 128 and 256 columns, few rows turned, fp32 in planes
FORWARD = [(9, 200000, 192, 64, H), (9, 70000, 136, 128, H), (3, 8192, 128, 8192, H), (64, 640, 136, 16384, B),
           (5, 6000, 1024, 2048, F)]


@pytest.mark.parametrize("groups,rows,K,N,dtype", FORWARD, ids=str)
def test_forward(pic, groups, rows, K, N, dtype):
    x, w = normal((rows, K), dtype, 1), normal((groups, N, K), dtype, 2, 1 / math.sqrt(K))
    offsets = [rows * i // groups for i in range(groups + 1)]
    o = torch.tensor(offsets, device="cuda")
    timed_out(pic, lambda: pic.grouped_linear(x, w, o), pic.grouped_linear_check)
    y = pic.grouped_linear(x, w, o)
    pic.grouped_linear_check()
    for g, i, j in group_ref.spans(offsets)[::max(1, groups // 3)]:
        at = torch.arange(i, j, max(1, (j - i) // 97), device="cuda")
        want, _ = ref.forward(x[at], w[g], None, "none", None)
        ref.check(y[at], want)


@pytest.mark.parametrize("groups,rows,K,N,dtype", [(7, 80000, 64, 64, H), (7, 80000, 100, 64, B), (7, 80000, 40, 40, F),
                                                   (2, 2000, 4096, 4096, B)], ids=str)
def test_gradient(pic, groups, rows, K, N, dtype):
    x, w = normal((rows, K), dtype, 1), normal((groups, N, K), dtype, 2, 0.1)
    dy, z = normal((rows, N), dtype, 3, 0.1), normal((rows, N), dtype, 4)
    offsets = [rows * i // groups for i in range(groups + 1)]
    o = torch.tensor(offsets, device="cuda")
    timed_out(pic, lambda: pic.grouped_linear_backward(dy, x, w, o, act="relu", pre=z), pic.grouped_linear_check)
    got = pic.grouped_linear_backward(dy, x, w, o, act="relu", pre=z)
    pic.grouped_linear_check()
    for g, v in zip(got, group_ref.backward(dy, x, w, z, offsets, "relu")):
        ref.check(g, v)


@pytest.mark.parametrize("shape,count,dtype", [((300, 300), 60, B), ((60, 2000), 60, F), ((2048, 2048), 5, B)], ids=str)
def test_orthogonalizer(pic, shape, count, dtype):
    g = [normal(shape, dtype, s) for s in range(count)]
    out = [torch.zeros_like(t) for t in g]
    h = pic.Orthogonalizer(g, out=out)
    timed_out(pic, lambda: h.orthogonalize(), h.check)
    h.orthogonalize()
    h.check()
    for i in (0, count // 2, count - 1):
        orth_ref.check(out[i], g[i])
    h.close()
