"""The linear layer's bounded waits, made to run out on purpose (see
test_wait_abort_gpu.py): one warp of the first tile withholds an mbarrier
arrival, the MMA thread's wait for free accumulators gives up after a few
thousand polls, every role of the CTA (of both CTAs, where a pair shares a tile)
skips what is left, copies and MMAs in flight are drained and tensor memory is
freed.  The status word says so once; the next call is right."""
import math

import pytest

torch = pytest.importorskip("torch")

import linear_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu
SHORT_LIMIT = 1 << 10


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_09020_gb300 import build
    build.build()


def normal(shape, dtype, seed, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").mul_(std).to(dtype)


H, F = torch.float16, torch.float32
# tiles of one CTA, one after another (64 and 128 columns), of a pair; fp32 through
# registers and in planes
FORWARD = [(150000, 192, 64, H), (70000, 136, 128, H), (8192, 128, 8192, H), (30000, 512, 64, F), (6000, 1024, 2048, F)]
# narrow gradients by TMA and through registers, fp32
NARROW = [(80000, 64, 64, H), (80000, 31, 64, H), (80000, 100, 64, H), (80000, 40, 40, F)]


def timed_out(pic, call):
    lib = pic.load_library()
    torch.cuda.synchronize()
    assert lib.pic_linear_test_wait_fault(1, SHORT_LIMIT) == pic.PIC_OK
    try:
        call()
        torch.cuda.synchronize()
    finally:
        lib.pic_linear_test_wait_fault(0, 0)
    with pytest.raises(pic.PicError) as e:
        pic.linear_check()
    assert e.value.status == pic.PIC_ERR_TIMEOUT
    pic.linear_check()  # said once


@pytest.mark.parametrize("M,K,N,dtype", FORWARD)
def test_forward(M, K, N, dtype):
    from paper_2609_09020_gb300 import pic
    x, w = normal((M, K), dtype, 1), normal((N, K), dtype, 2, 1 / math.sqrt(K))
    timed_out(pic, lambda: pic.linear(x, w))
    y = pic.linear(x, w)
    pic.linear_check()
    rows = torch.arange(0, M, max(1, M // 777), device="cuda")
    want, _ = ref.forward(x[rows], w, None, "none", None)
    ref.check(y[rows], want)


@pytest.mark.parametrize("M,K,N,dtype", NARROW)
def test_narrow_gradient(M, K, N, dtype):
    from paper_2609_09020_gb300 import pic
    x, w = normal((M, K), dtype, 1), normal((N, K), dtype, 2, 0.1)
    dy, z = normal((M, N), dtype, 3, 0.1), normal((M, N), dtype, 4)
    timed_out(pic, lambda: pic.linear_backward(dy, x, w, act="relu", pre=z))
    got = pic.linear_backward(dy, x, w, act="relu", pre=z)
    pic.linear_check()
    for g, v in zip(got, ref.backward(dy, x, w, z, "relu")):
        ref.check(g, v)


def test_hook_arguments():
    from paper_2609_09020_gb300 import pic
    assert pic.load_library().pic_linear_test_wait_fault(2, 0) == pic.PIC_ERR_INVALID_ARG
