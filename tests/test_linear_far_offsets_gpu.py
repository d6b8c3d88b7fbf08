"""Elements whose offsets, in elements and in bytes, pass 32 bits: rows that lie far apart,
and matrices of more than 2^31 elements.  Data are small integers, so sums are exact."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_09020_gb300 import build
    build.build()


@pytest.fixture(autouse=True)
def _give_back():
    yield
    torch.cuda.empty_cache()


def whole(shape, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-2, 3, shape, generator=g, device="cuda", dtype=torch.int8).to(dtype)


class Far:
    """Matrices whose rows lie 5.2e9 elements / rows apart, in one allocation side by side."""

    def __init__(self, rows, dtype, shift):
        self.ld = 5_200_000_000 // rows // 8 * 8 + (3 if shift else 0)
        self.buf = torch.empty(self.ld * rows, dtype=dtype, device="cuda")
        self.rows, self.at = rows, 1 if shift else 0

    def take(self, rows, cols):
        assert rows <= self.rows
        v = self.buf.as_strided((rows, cols), (self.ld, 1), self.at)
        self.at += (cols + 15) // 8 * 8
        assert self.at < self.ld
        return v

    def put(self, m):
        v = self.take(*m.shape)
        v.copy_(m)
        return v


@pytest.mark.parametrize("dtype", [F16, F32], ids=["fp16", "fp32"])
@pytest.mark.parametrize("shift", [False, True])
@pytest.mark.parametrize("M,K,N", [(4, 72, 40), (14, 300, 70), (60, 40, 48), (90, 200, 150), (1200, 64, 64), (1100, 33, 20),
                                   (300, 600, 520)])
def test_rows_far_apart(M, K, N, shift, dtype):
    from paper_2609_09020_gb300 import pic
    far = Far(max(M, N), dtype, shift)
    x, w, r = whole((M, K), dtype, 1), whole((N, K), dtype, 2), whole((M, N), dtype, 3)
    dy, z = whole((M, N), dtype, 4), whole((M, N), dtype, 5)
    z = torch.where(z >= 0, 8, -8).to(dtype)
    fx, fw, fr, fdy, fz = (far.put(m) for m in (x, w, r, dy, z))
    y, dx, dw = far.take(M, N), far.take(M, K), far.take(N, K)
    pic.linear(fx, fw, act="relu", residual=fr, out=y)
    _, _, db = pic.linear_backward(fdy, fx, fw, act="gelu", pre=fz, dx=dx, dweight=dw)
    pic.linear_check()
    want = (x.double() @ w.double().t()).clamp(min=0) + r.double()
    dz = torch.where(z > 0, dy, 0).double()
    assert torch.equal(y.double(), want)
    assert torch.equal(dx.double(), dz @ w.double()) and torch.equal(dw.double(), dz.t() @ x.double())
    assert torch.equal(db.double(), dz.sum(0))
    assert torch.equal(fx, x) and torch.equal(fdy, dy) and torch.equal(fr, r)


@pytest.mark.parametrize("M,K,N,dtype", [(40_000_003, 8, 64, F16), (36_000_001, 60, 13, BF16), (34_000_001, 7, 64, F32),
                                         (9_000_001, 250, 256, F16), (1_100_001, 2000, 9, F32)])
def test_more_than_2_31_elements(M, K, N, dtype):
    from paper_2609_09020_gb300 import pic
    x, w, b = whole((M, K), dtype, 1), whole((N, K), dtype, 2), whole((1, N), dtype, 3)[0]
    y = pic.linear(x, w, b, act="relu")
    at = torch.cat([torch.arange(0, M, M // 500, device="cuda"), torch.arange(M - 300, M, device="cuda")])
    want = (x[at].double() @ w.double().t() + b.double()).clamp(min=0)
    assert torch.equal(y[at], want.to(dtype))
    dx, _, db = pic.linear_backward(y, x, w, act="relu", pre=y, need=("x", "bias") if K > 8 else ("x", "weight"))
    pic.linear_check()
    assert torch.equal(dx[at], (y[at].double() @ w.double()).to(dtype))


@pytest.mark.parametrize("in_place", [False, True])
def test_clip_more_than_2_31_elements(in_place):
    from paper_2609_09020_gb300 import pic
    n = 2_300_000_011
    g = torch.ones(n, dtype=BF16, device="cuda")
    g[-1], g[1 << 31] = 3.0, -2.0
    out = g if in_place else torch.zeros_like(g)
    norm = pic.GradClip([g], out=[out]).clip(0.25 * (n + 11) ** 0.5)
    assert abs(float(norm) / (n + 11) ** 0.5 - 1) < 2.0 ** -18
    assert float(out[-1]) == 0.75 and float(out[1 << 31]) == -0.5
    assert int((out == 0.25).sum()) == n - 2
