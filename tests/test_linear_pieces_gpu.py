"""The accuracy of fp32 products, which the kernels for more than a few rows form from
three bfloat16 pieces of each operand.

One product alone (K = 1): rounding to nearest leaves a middle piece of at most 2^-8 and
a last one of at most 2^-16 of the value, so the three products of pieces that are left
out are below 2^-23 of the product; and the last addition may truncate, another 2^-23:
2^-22 in all.  (Pieces by truncation are up to 2^-7 and 2^-15: 4.7e-7 at 0x3f80ffff
squared, always with the product's sign.)

Long sums, of random and of one sign: the root mean square of the error, relative to the
sums'.  The kernels state 6.0e-7 (2.1e-6 for one sign with pieces by truncation); 1.5e-6
is above twice that, and any product of pieces that is lost is 2.3e-6 or more by itself (test_lost_pieces_are_seen, on the CPU)."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

ONE = 2.0 ** -22
RMS = 1.5e-6


@pytest.fixture(scope="module")
def pic():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_09020_gb300 import build, pic
    build.build()
    return pic


def hard(shape, seed):
    """Values from 1 to 2, signed, whose low halves are all ones, all zeros but one, or random."""
    g = torch.Generator().manual_seed(seed)
    top = torch.randint(0, 128, shape, generator=g, dtype=torch.int32)
    low = torch.randint(0, 65536, shape, generator=g, dtype=torch.int32)
    kind = torch.randint(0, 4, shape, generator=g, dtype=torch.int32)
    low = torch.where(kind == 0, 0xffff, torch.where(kind == 1, 0x8000, torch.where(kind == 2, 0x7fff, low)))
    top = torch.where(kind == 0, top % 3, top)
    v = (0x3f800000 | top << 16 | low).view(torch.float32)
    return torch.where(torch.rand(shape, generator=g) < 0.5, -v, v).cuda()


def relative(got, want):
    return float(((got.double() - want).abs() / want.abs()).max())


@pytest.mark.gpu
@pytest.mark.parametrize("M,N", [(1, 500), (8, 3000), (40, 100), (300, 64), (1000, 128), (300, 300), (50, 9000),
                                 (8192, 8192), (5000, 3000)])
def test_one_product(pic, M, N):
    """y of K = 1: few rows, thin, through registers (w on either side), planes."""
    x, w = hard((M, 1), 1), hard((N, 1), 2)
    x[0], w[0] = (torch.tensor([0x3f80ffff], dtype=torch.int32).view(torch.float32).item(),) * 2
    y = pic.linear(x, w)
    want = x.double() @ w.double().t()
    pic.linear_check()
    assert relative(y, want) <= ONE


@pytest.mark.gpu
@pytest.mark.parametrize("M,K,N", [(2000, 64, 64), (5000, 40, 33), (3000, 100, 80), (1500, 300, 500), (600, 2048, 1000)])
def test_one_product_of_a_gradient(pic, M, K, N):
    """One row of x and one column of dy are not zero: each output is one product."""
    x, w, dy = torch.zeros((M, K), device="cuda"), hard((N, K), 3), torch.zeros((M, N), device="cuda")
    row, col = M - 7, N // 2
    x[row] = hard((K,), 4)
    dy[:, col] = hard((M,), 5)
    dx, dw, _ = pic.linear_backward(dy, x, w)
    pic.linear_check()
    assert relative(dx, dy[:, col:col + 1].double() * w[col].double()) <= ONE
    assert relative(dw[col], dy[row, col].double() * x[row].double()) <= ONE
    dw[col] = 0
    assert not bool(dw.any())


@pytest.mark.gpu
@pytest.mark.parametrize("M,K,N", [(4, 4096, 512), (300, 128, 128), (5000, 100, 64), (300, 1024, 300), (200, 4096, 200),
                                   (20, 1024, 8192), (2048, 1024, 4096), (2048, 4096, 2048), (4000, 200, 3000)])
@pytest.mark.parametrize("positive", [False, True])
def test_root_mean_square(pic, positive, M, K, N):
    g = torch.Generator(device="cuda").manual_seed(6)
    x, w = (torch.randn(s, generator=g, device="cuda") for s in ((M, K), (N, K)))
    if positive:
        x, w = x.abs(), w.abs()
    y = pic.linear(x, w).double()
    dx, dw, _ = pic.linear_backward(y.float(), x, w)
    pic.linear_check()
    dy = y.float().double()
    want = x.double() @ w.double().t()
    for got, v in ((y, want), (dx.double(), dy @ w.double()), (dw.double(), dy.t() @ x.double())):
        assert float((got - v).norm() / v.norm()) < RMS


@pytest.mark.gpu
@pytest.mark.parametrize("M,K,N", [(3000, 24, 40), (300, 90, 300), (4000, 200, 3000)])
def test_largest_values(pic, M, K, N):
    """Values that bfloat16 would round to infinity are finite, and so is what is made of them."""
    top = float(np.finfo(np.float32).max)
    x, w = torch.zeros((M, K), device="cuda"), torch.full((N, K), 0.5, device="cuda")
    x[1, 3], x[M - 1, K - 1], x[5, 0] = top, -top, 3.3963e38
    y = pic.linear(x, w)
    want = x.double() @ w.double().t()
    dx, dw, _ = pic.linear_backward(x[:, :1].expand(M, N).contiguous(), w[:1].expand(M, K).contiguous(), w)
    pic.linear_check()
    assert bool(((y.double() - want).abs() <= ONE * want.abs()).all())
    assert bool(dw.isfinite().all()) and relative(dw, torch.full_like(dw, 0.5).double() * x[5, 0].double()) <= ONE
    assert not bool(dx.isnan().any())


# ---- the arithmetic by itself, on the CPU -----------------------------------
def bf16(v):
    """fp32 rounded to 8 bits, to nearest even."""
    u = np.asarray(v, np.float32).view(np.uint32).astype(np.uint64)
    u = (u + 0x7fff + ((u >> 16) & 1)) & 0xffff0000
    return u.astype(np.uint32).view(np.float32)


def pieces(v):
    hi = bf16(v)
    r = (v - hi).astype(np.float32)
    mid = bf16(r)
    r = (r - mid).astype(np.float32)
    lo = bf16(r)
    return hi, mid, lo, (r - lo).astype(np.float32)


PAIRS = [(2, 0), (0, 2), (1, 1), (1, 0), (0, 1), (0, 0)]  # lo hi, hi lo, mid mid, mid hi, hi mid, hi hi


def values(n, seed=0):
    rng = np.random.default_rng(seed)
    u = rng.integers(0x00800000, 0x7f000000, n, dtype=np.uint32)
    u[::5] |= 0xffff
    u[1::5] = (u[1::5] & 0xffff0000) | 0x8000
    v = (u | (rng.integers(0, 2, n, dtype=np.uint32) << 31)).view(np.float32)
    return v[np.abs(v) > 1e-25]


def test_pieces_are_the_value():
    v = values(200000)
    hi, mid, lo, left = pieces(v)
    assert not left.any()
    assert (np.abs(mid) <= 2.0 ** -8 * np.abs(v)).all() and (np.abs(lo) <= 2.0 ** -16 * np.abs(v)).all()
    assert (hi.astype(np.float64) + mid + lo == v).all()


def test_what_is_left_out():
    a, b = values(100000, 1), values(100000, 2)
    n = min(len(a), len(b))
    a, b = (np.where(np.abs(v[:n]) > 1e18, np.float32(1.5), v[:n]) for v in (a, b))
    pa, pb = ([p.astype(np.float64) for p in pieces(v)] for v in (a, b))
    made = sum(pa[i] * pb[j] for i, j in PAIRS)
    want = a.astype(np.float64) * b
    assert (np.abs(made - want) <= 2.0 ** -23 * np.abs(want)).all()


@pytest.mark.parametrize("lost", range(6))
@pytest.mark.parametrize("K", [128, 1024, 4096])
def test_lost_pieces_are_seen(K, lost):
    """The bar of test_root_mean_square, on sums that lack one product of pieces."""
    rng = np.random.default_rng(7)
    x, w = rng.standard_normal((40, K)).astype(np.float32), rng.standard_normal((50, K)).astype(np.float32)
    px, pw = ([p.astype(np.float64) for p in pieces(v)] for v in (x, w))
    y = sum(px[i] @ pw[j].T for t, (i, j) in enumerate(PAIRS) if t != lost)
    want = x.astype(np.float64) @ w.T.astype(np.float64)
    error = np.linalg.norm(y - want) / np.linalg.norm(want)
    assert error > 1.5 * RMS, (lost, error)


def test_truncated_pieces_are_seen():
    """The bar of test_one_product, on pieces by truncation: what it is there to catch."""
    v = np.array([0x3f80ffff], np.uint32).view(np.float32)
    p, r = [], v
    for _ in range(3):
        c = (r.view(np.uint32) & np.uint32(0xffff0000)).view(np.float32)
        p.append(c.astype(np.float64))
        r = (r - c).astype(np.float32)
    made = sum(p[i] * p[j] for i, j in PAIRS)
    assert abs(made[0] / float(v[0]) ** 2 - 1) > ONE
