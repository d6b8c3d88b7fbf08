"""Infinite and NaN values in fp32 sums that are far longer than a tile's: they reach
their row and column and nothing else, and no wait of the kernels runs out while the
sums they touch are computed again.

The data are integers from -3 to 3, so that every partial sum is an integer below
2^24 and each finite output has to be the exact sum."""
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_09020_gb300 import build
    build.build()


def whole(shape, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-3, 4, shape, generator=g, device="cuda", dtype=torch.int8).float()


def product64(a, b):
    """a^T b in fp64, a block of rows at a time."""
    out = torch.zeros((a.shape[1], b.shape[1]), dtype=torch.float64, device="cuda")
    for i in range(0, a.shape[0], 32768):
        out += a[i:i + 32768].double().t() @ b[i:i + 32768].double()
    return out


# rows, in, out: planes, with more tiles than there are pairs of SMs, so that the rows are
# not shared out; through registers, in parts of tens of thousands of rows
@pytest.mark.parametrize("M,K,N", [(262144, 640, 4096), (300001, 24, 640)])
def test_weight_gradient(M, K, N):
    from paper_2609_09020_gb300 import pic
    x, dy = whole((M, K), 1), whole((M, N), 2)
    w = whole((N, K), 3)
    want = product64(dy, x)
    at = M - 12345
    x[at, 11], dy[5, 7], dy[M // 2, N - 1] = math.inf, math.nan, -math.inf
    _, dw, _ = pic.linear_backward(dy, x, w, need=("weight",))
    pic.linear_check()
    rows = torch.ones(N, dtype=torch.bool, device="cuda")
    cols = torch.ones(K, dtype=torch.bool, device="cuda")
    rows[7] = rows[N - 1] = cols[11] = False
    assert torch.equal(dw[rows][:, cols].double(), want[rows][:, cols])
    assert bool(dw[7].isnan().all())
    limit = dy[at] * math.inf  # NaN where dy is zero
    assert torch.equal(dw[rows, 11].nan_to_num(nan=5.0), limit[rows].nan_to_num(nan=5.0))
    limit = x[M // 2] * -math.inf
    assert torch.equal(dw[N - 1][cols].nan_to_num(nan=5.0), limit[cols].nan_to_num(nan=5.0))


@pytest.mark.parametrize("M,K,N", [(4096, 70000, 640), (200, 150001, 130)])
def test_forward(M, K, N):
    from paper_2609_09020_gb300 import pic
    x, w = whole((M, K), 4), whole((N, K), 5)
    want = product64(x.t(), w.t())
    x[M - 1, K - 2], w[0, 66000] = math.nan, math.inf
    y = pic.linear(x, w)
    pic.linear_check()
    assert torch.equal(y[:-1, 1:].double(), want[:-1, 1:])
    assert bool(y[-1].isnan().all())
    limit = x[:-1, 66000] * math.inf
    assert torch.equal(y[:-1, 0].nan_to_num(nan=5.0), limit.nan_to_num(nan=5.0))


def test_everything_is_nan():
    """The most that can have to be computed again."""
    from paper_2609_09020_gb300 import pic
    x = torch.full((20000, 300), math.nan, device="cuda")
    dy, w = whole((20000, 400), 6), whole((400, 300), 7)
    dx, dw, db = pic.linear_backward(dy, x, w)
    y = pic.linear(x, w)
    pic.linear_check()
    assert bool(dw.isnan().all()) and bool(y.isnan().all())
    assert torch.equal(dx.double(), dy.double() @ w.double()) and torch.equal(db.double(), dy.double().sum(0))
