"""16-bit products over very many rows whose terms all have one sign.

A tensor core truncates when it adds to an accumulator, so a sum that stays in one
shrinks with every 16 terms.  The kernels take sums out of tensor memory after at most
1024 additions (2^14 terms) and add those to nearest: at most 1024 x 2^-23 of the sum is
lost, and 2^-24 for each of the partial sums, of which there are a few hundred here; then
one rounding to fp16, 2^-11.  (Without that, 2^16 additions lose some 2e-3.)"""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
F16 = torch.float16
LOST = 1024 * 2.0 ** -23


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_09020_gb300 import build
    build.build()


def positive(shape, seed, size):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.rand(shape, generator=g, device="cuda", dtype=F16).add_(0.5).mul_(size)


def product64(a, b):
    """a^T b in fp64, a block of rows at a time."""
    out = torch.zeros((a.shape[1], b.shape[1]), dtype=torch.float64, device="cuda")
    step = 1 << 20
    for i in range(0, a.shape[0], step):
        out += a[i:i + step].double().t() @ b[i:i + step].double()
    return out


def check(got, want, sums):
    tolerance = (2.0 ** -11 + LOST + sums * 2.0 ** -24) * want
    worst = float(((got.double() - want).abs() / want).max())
    assert bool(((got.double() - want).abs() <= tolerance).all()), worst


@pytest.mark.parametrize("M,K,N,pad", [(100_000_000, 8, 8, 0), (60_000_001, 5, 3, 0), (40_000_000, 8, 8, 8)])
def test_narrow_gradient(M, K, N, pad):
    """Rows by TMA, as runs of memory, through registers."""
    from paper_2609_09020_gb300 import pic
    x, dy, w = positive((M, K + pad), 1, 1.0)[:, :K], positive((M, N), 2, 1e-5), positive((N, K), 3, 1.0)
    _, dw, db = pic.linear_backward(dy, x, w, need=("weight", "bias"))
    pic.linear_check()
    check(dw, product64(dy, x), 2000)
    # db: threads of 304 x 256 and their sums, all to nearest
    check(db, product64(dy, torch.ones((M, 1), dtype=F16, device="cuda"))[:, 0], 4000)


@pytest.mark.parametrize("K,N,part", [(2304, 2304, False), (300, 200, True)])
def test_tiled_gradient(K, N, part):
    """dw of a million rows: tiles that are not cut along the rows, and tiles that are."""
    from paper_2609_09020_gb300 import pic
    M = 16_000_000 if part else 1_000_001
    x, dy, w = positive((M, K), 1, 1.0), positive((M, N), 2, 1e-3 if not part else 1e-4), positive((N, K), 3, 1.0)
    _, dw, _ = pic.linear_backward(dy, x, w, need=("weight",))
    pic.linear_check()
    n, k = slice(N - 40, N), slice(K - 50, K)
    check(dw[n, k], product64(dy[:, n], x[:, k]), 1000)
    check(dw[:30, :30], product64(dy[:, :30], x[:, :30]), 1000)


def test_forward():
    """A few hundred thousand terms a sum, bias, activation and residual behind them."""
    from paper_2609_09020_gb300 import pic
    M, K, N = 2304, 300_000, 2304
    x, w = positive((M, K), 4, 0.05), positive((N, K), 5, 0.05)
    b, r = positive((N,), 6, 1.0), positive((M, N), 7, 1.0)
    y, z = pic.linear(x, w, b, act="relu", residual=r, save_pre=True)
    pic.linear_check()
    m, n = slice(M - 30, M), slice(N - 30, N)
    want = x[m].double() @ w[n].double().t() + b[n].double()
    check(z[m, n], want, 100)
    check(y[m, n], want + r[m, n].double(), 100)


@pytest.mark.parametrize("M,K,N", [(2304, 40_000, 2304)])
def test_waits_that_run_out(M, K, N):
    """An arrival withheld in the first tile while its sums are carried on: the status says
    so once, and the next call is right."""
    from paper_2609_09020_gb300 import pic
    lib = pic.load_library()
    x, w = positive((M, K), 8, 0.05), positive((N, K), 9, 0.05)
    torch.cuda.synchronize()
    assert lib.pic_linear_test_wait_fault(1, 1 << 10) == pic.PIC_OK
    try:
        pic.linear(x, w)
        torch.cuda.synchronize()
    finally:
        lib.pic_linear_test_wait_fault(0, 0)
    with pytest.raises(pic.PicError) as e:
        pic.linear_check()
    assert e.value.status == pic.PIC_ERR_TIMEOUT
    pic.linear_check()
    y = pic.linear(x, w)
    pic.linear_check()
    check(y[:30, :30], x[:30].double() @ w[:30].double().t(), 100)
