"""pic.linear and pic.linear_backward against the definitions in fp64."""
import math

import pytest

torch = pytest.importorskip("torch")

import linear_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.float16, torch.bfloat16]
IDS = ["fp32", "fp16", "bf16"]


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_09020_gb300 import build
    build.build()


def normal(shape, dtype, seed, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").mul_(std).to(dtype)


def wide(rows, cols, dtype, seed, pad, shift, std=1.0):
    """A [rows][cols] view of a wider tensor whose other columns are NaN."""
    t = torch.full((rows, cols + pad), math.nan, dtype=dtype, device="cuda")
    v = t[:, shift:shift + cols]
    v.copy_(normal((rows, cols), dtype, seed, std))
    return v


# rows, in, out: one row, few rows, tile edges and past them, the nets' layers, odd
# sizes, long sums, single columns
SIZES = [(1, 1, 1), (1, 64, 64), (1, 4096, 512), (2, 257, 3), (3, 7, 64), (5, 1000, 130), (8, 512, 256),
         (16, 2048, 128), (17, 640, 72), (31, 96, 1000), (32, 128, 48), (33, 256, 257), (64, 64, 64),
         (100, 40, 40), (127, 65, 129), (128, 128, 128), (129, 1111, 63), (200, 16, 3), (255, 264, 512),
         (256, 1024, 256), (257, 72, 520), (1000, 7, 64), (1021, 64, 3), (4097, 14, 64), (5000, 64, 64),
         (513, 2056, 1), (300, 1, 300)]


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_forward(size, dtype):
    from paper_2609_09020_gb300 import pic
    M, K, N = size
    act = ("none", "relu", "gelu")[(M + K + N) % 3]
    x, w = normal((M, K), dtype, 1), normal((N, K), dtype, 2, 1.4 / math.sqrt(K))
    b, r = normal((N,), dtype, 3, 0.1), normal((M, N), dtype, 4)
    for bias, res in ((b, r), (None, None)):
        y, z = pic.linear(x, w, bias, act=act, residual=res, save_pre=True)
        want_y, want_z = ref.forward(x, w, bias, act, res)
        ref.check(y, want_y, "y")
        ref.check(z, want_z, "pre")
        assert torch.equal(y, pic.linear(x, w, bias, act=act, residual=res))
    pic.linear_check()


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("act", ["none", "relu", "gelu"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_backward(size, act, dtype):
    from paper_2609_09020_gb300 import pic
    M, K, N = size
    x, w = normal((M, K), dtype, 1), normal((N, K), dtype, 2, 1.4 / math.sqrt(K))
    dy, z = normal((M, N), dtype, 5, 0.1), normal((M, N), dtype, 6, 1.4)
    got = pic.linear_backward(dy, x, w, act=act, pre=z)
    want = ref.backward(dy, x, w, z, act)
    for g, v, name in zip(got, want, ("dx", "dw", "db")):
        ref.check(g, v, name)
    for i, name in enumerate(("x", "weight", "bias")):  # each by itself, the same
        one = pic.linear_backward(dy, x, w, act=act, pre=z, need=(name,))
        assert [v is None for v in one] == [j != i for j in range(3)]
        ref.check(one[i], want[i], name)
    pic.linear_check()


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("pad,shift", [(1, 0), (8, 0), (8, 8), (5, 3), (64, 16)])
@pytest.mark.parametrize("size", [(1, 300, 70), (9, 128, 65), (130, 65, 72), (400, 264, 256)], ids=str)
def test_strides(size, pad, shift, dtype):
    """Rows further apart than their width, bases off every boundary; what lies
    between the rows is NaN and stays out of the results."""
    from paper_2609_09020_gb300 import pic
    M, K, N = size
    x, w = wide(M, K, dtype, 1, pad, shift), wide(N, K, dtype, 2, pad, shift, 0.1)
    r = wide(M, N, dtype, 4, pad, shift)
    out = torch.full((M, N + pad), 7.0, dtype=dtype, device="cuda")
    y, z = pic.linear(x, w, None, act="gelu", residual=r, out=out[:, shift:shift + N], save_pre=True)
    want_y, want_z = ref.forward(x, w, None, "gelu", r)
    ref.check(y, want_y, "y")
    ref.check(z, want_z, "pre")
    assert bool((out[:, :shift] == 7).all()) and bool((out[:, shift + N:] == 7).all())
    dy, zz = wide(M, N, dtype, 5, pad, shift), wide(M, N, dtype, 6, pad, shift)
    for act in ("none", "gelu"):
        got = pic.linear_backward(dy, x, w, act=act, pre=zz)
        for g, v, name in zip(got, ref.backward(dy, x, w, zz, act), ("dx", "dw", "db")):
            ref.check(g, v, name)
    pic.linear_check()


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("size", [(40, 65, 61), (300, 1001, 515), (1, 301, 69), (700, 259, 1501), (2000, 61, 35), (1500, 5, 1),
                                  (1100, 70, 121)], ids=str)
def test_rows_that_end_inside_16_bytes(size, dtype):
    """Rows that start on 16-byte boundaries, but whose width is no multiple of 16
    bytes: the NaN behind the last column stays out, and nothing is written there."""
    from paper_2609_09020_gb300 import pic
    M, K, N = size

    def padded(rows, cols, seed, std=1.0):
        return wide(rows, cols, dtype, seed, -cols % 8 + 8, 0, std)

    x, w, r = padded(M, K, 1), padded(N, K, 2, 1.4 / math.sqrt(K)), padded(M, N, 3)
    buf = torch.full((M + 1, (N + 7) // 8 * 8), 7.0, dtype=dtype, device="cuda")
    for act, res in (("none", None), ("gelu", r)):
        y = pic.linear(x, w, act=act, residual=res, out=buf[:M, :N])
        ref.check(y, ref.forward(x, w, None, act, res)[0], "y")
        assert bool((buf[:, N:] == 7).all()) and bool((buf[M] == 7).all())
    dy, z = padded(M, N, 5, 0.1), padded(M, N, 6, 1.4)
    for act in ("none", "gelu"):
        got = pic.linear_backward(dy, x, w, act=act, pre=z)
        for g, v, name in zip(got, ref.backward(dy, x, w, z, act), ("dx", "dw", "db")):
            ref.check(g, v, name)
    pic.linear_check()


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("N", [1, 3, 17, 31, 32, 49, 63])
@pytest.mark.parametrize("rows", [64, 70, 5000])
def test_narrow_outputs(rows, N, dtype):
    """Outputs and residuals whose rows lie end to end, in strides, and one of each;
    several tiles a CTA, and a last one that is not whole."""
    from paper_2609_09020_gb300 import pic
    K = 33
    x, w, b = normal((rows, K), dtype, 1), normal((N, K), dtype, 2, 0.2), normal((N,), dtype, 3)
    flat, gaps = normal((rows, N), dtype, 4), wide(rows, N, dtype, 4, 6, 1)
    want_y, want_z = ref.forward(x, w, b, "relu", flat)
    buf = torch.full((rows, N + 5), 7.0, dtype=dtype, device="cuda")
    for res in (flat, gaps):
        for out in (None, buf[:, 2:2 + N]):
            y, z = pic.linear(x, w, b, act="relu", residual=res, out=out, save_pre=True)
            ref.check(y, want_y, "y")
            ref.check(z, want_z, "pre")
    assert bool((buf[:, :2] == 7).all()) and bool((buf[:, 2 + N:] == 7).all())
    pic.linear_check()


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("size", [(20000, 64, 64), (9000, 40, 3), (70001, 8, 16), (4096, 512, 384),
                                  (600, 4096, 200), (1500, 1536, 1600), (2500, 328, 2600), (520, 2500, 2600),
                                  (2305, 2304, 2311)], ids=str)
def test_larger(size, dtype):
    from paper_2609_09020_gb300 import pic
    M, K, N = size
    x, w = normal((M, K), dtype, 1), normal((N, K), dtype, 2, 1.4 / math.sqrt(K))
    b, dy, z = normal((N,), dtype, 3, 0.1), normal((M, N), dtype, 5, 0.02), normal((M, N), dtype, 6, 1.4)
    y, pre = pic.linear(x, w, b, act="relu", save_pre=True)
    want_y, want_z = ref.forward(x, w, b, "relu", None)
    ref.check(y, want_y, "y")
    ref.check(pre, want_z, "pre")
    got = pic.linear_backward(dy, x, w, act="gelu", pre=z)
    for g, v, name in zip(got, ref.backward(dy, x, w, z, "gelu"), ("dx", "dw", "db")):
        ref.check(g, v, name)
    again = pic.linear_backward(dy, x, w, act="gelu", pre=z)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    pic.linear_check()


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("size", [(1, 4096, 4096), (1, 16384, 16), (3, 4104, 1000), (9, 2048, 4096), (16, 512, 16384),
                                  (24, 4096, 600), (25, 5000, 2000), (32, 2048, 2056), (32, 16384, 96), (32, 1, 5000),
                                  (33, 4096, 512), (2, 8192, 24)], ids=str)
def test_few_rows(size, dtype):
    """Weights read once: K in many turns, over the CTAs of a cluster, ends inside a turn."""
    from paper_2609_09020_gb300 import pic
    M, K, N = size
    x, w = normal((M, K), dtype, 1), normal((N, K), dtype, 2, 1.4 / math.sqrt(K))
    b, r, dy = normal((N,), dtype, 3, 0.1), normal((M, N), dtype, 4), normal((M, N), dtype, 5, 0.1)
    y, z = pic.linear(x, w, b, act="gelu", residual=r, save_pre=True)
    want_y, want_z = ref.forward(x, w, b, "gelu", r)
    ref.check(y, want_y, "y")
    ref.check(z, want_z, "pre")
    got = pic.linear_backward(dy, x, w, act="gelu", pre=z)
    for g, v, name in zip(got, ref.backward(dy, x, w, z, "gelu"), ("dx", "dw", "db")):
        ref.check(g, v, name)
    pic.linear_check()


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("act", ["none", "relu", "gelu"])
@pytest.mark.parametrize("size", [(1024, 3, 3), (1030, 128, 128), (2049, 65, 128), (3000, 100, 65), (1300, 64, 17),
                                  (1024, 1, 64), (30011, 64, 64), (25000, 7, 40), (40000, 128, 96)], ids=str)
def test_narrow_gradient(size, act, dtype):
    """Layers of synthesis nets over many rows: all of the gradient, and each part
    by itself; contiguous, and with NaN between the rows."""
    from paper_2609_09020_gb300 import pic
    M, K, N = size
    for pad, shift in ((0, 0), (3, 1), (8, 8)):
        x, w = wide(M, K, dtype, 1, pad, shift), wide(N, K, dtype, 2, pad, shift, 1.4 / math.sqrt(K))
        dy, z = wide(M, N, dtype, 5, pad, shift, 0.1), wide(M, N, dtype, 6, pad, shift, 1.4)
        want = ref.backward(dy, x, w, z, act)
        got = pic.linear_backward(dy, x, w, act=act, pre=z)
        for g, v, name in zip(got, want, ("dx", "dw", "db")):
            ref.check(g, v, name)
        if pad == 0:
            again = pic.linear_backward(dy, x, w, act=act, pre=z)
            assert all(torch.equal(a, b) for a, b in zip(got, again))
            for need in (("x",), ("weight",), ("x", "bias"), ("weight", "bias")):
                some = pic.linear_backward(dy, x, w, act=act, pre=z, need=need)
                for i, name in enumerate(("x", "weight", "bias")):
                    assert (some[i] is not None) == (name in need)
                    if name in need:
                        ref.check(some[i], want[i], name)
    pic.linear_check()


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_narrow_infinities(dtype):
    """Infinite and NaN values reach what depends on them, as in IEEE arithmetic,
    and nothing else."""
    from paper_2609_09020_gb300 import pic
    M, K, N = 5000, 24, 40
    x, w = normal((M, K), dtype, 1), normal((N, K), dtype, 2, 0.2)
    dy, z = normal((M, N), dtype, 5, 0.1), normal((M, N), dtype, 6, 1.4)
    clean = ref.backward(dy, x, w, z, "gelu")
    dy[1700, 11], dy[1701, 12], x[4000, 5] = math.inf, math.nan, -math.inf
    dx, dw, db = pic.linear_backward(dy, x, w, act="gelu", pre=z)
    keep = torch.ones(M, dtype=torch.bool, device="cuda")
    keep[1700] = keep[1701] = False
    ref.check(dx[keep], (clean[0][0][keep], clean[0][1][keep]), "dx")
    d = ref.act_grad64(z[1700, 11].double(), "gelu")
    assert torch.equal(dx[1700], (torch.sign(d * w[11].double()) * math.inf).to(dtype))
    assert bool(dx[1701].isnan().all())
    rows = [n for n in range(N) if n not in (11, 12)]
    cols = [k for k in range(K) if k != 5]
    ref.check(dw[rows][:, cols], (clean[1][0][rows][:, cols], clean[1][1][rows][:, cols]), "dw")
    assert bool(dw[rows][:, 5].isinf().all()) and bool(dw[12].isnan().all()) and bool(dw[11][cols].isinf().all())
    ref.check(db[rows], (clean[2][0][rows], clean[2][1][rows]), "db")
    assert bool(db[11].isinf()) and bool(db[12].isnan())
    # a weight: every row of dx, nothing of dw
    w[3, 9] = math.inf
    dx, dw, _ = pic.linear_backward(normal((M, N), dtype, 5, 0.1), normal((M, K), dtype, 1), w, act="none")
    assert bool(dx[:, 9].isinf().all()) and int((~dx.isfinite()).any(0).sum()) == 1 and bool(dw.isfinite().all())


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_no_rows(dtype):
    from paper_2609_09020_gb300 import pic
    x, w, b = normal((0, 24), dtype, 1), normal((8, 24), dtype, 2), normal((8,), dtype, 3)
    y, z = pic.linear(x, w, b, act="gelu", save_pre=True)
    assert y.shape == z.shape == (0, 8)
    dx, dw, db = pic.linear_backward(y, x, w, act="gelu", pre=z)
    assert dx.shape == (0, 24)
    assert dw.shape == (8, 24) and not bool(dw.any()) and db.shape == (8,) and not bool(db.any())


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("rows", [1, 6, 40, 300])
def test_residual_forms(rows, dtype):
    """A residual that is the output itself, and one row for all."""
    from paper_2609_09020_gb300 import pic
    x, w = normal((rows, 96), dtype, 1), normal((80, 96), dtype, 2, 0.1)
    r, one = normal((rows, 80), dtype, 4), normal((1, 80), dtype, 5)
    want, _ = ref.forward(x, w, None, "relu", r)
    y = r.clone()
    assert pic.linear(x, w, act="relu", residual=y, out=y) is y
    ref.check(y, want)
    want, _ = ref.forward(x, w, None, "relu", one.expand(rows, 80))
    ref.check(pic.linear(x, w, act="relu", residual=one.expand(rows, 80)), want)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_leading_dimensions(dtype):
    from paper_2609_09020_gb300 import pic
    x, w = normal((3, 5, 48), dtype, 1), normal((24, 48), dtype, 2, 0.1)
    y, z = pic.linear(x, w, act="gelu", save_pre=True)
    assert y.shape == z.shape == (3, 5, 24)
    want, _ = ref.forward(x.view(15, 48), w, None, "gelu", None)
    ref.check(y.view(15, 24), want)
    dx, dw, db = pic.linear_backward(y, x, w, act="gelu", pre=z)
    assert dx.shape == x.shape and dw.shape == w.shape and db.shape == (24,)
    one = pic.linear(x[0, 0], w)
    assert one.shape == (24,)
    ref.check(one.view(1, 24), ref.forward(x[0, :1], w, None, "none", None)[0])


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_infinities_in_large_products(dtype):
    """One infinite or NaN value in a product of many tiles and a long sum: what
    IEEE arithmetic gives, in its row, its column and nowhere else."""
    from paper_2609_09020_gb300 import pic
    M, K, N = 400, 700, 300
    x, w = normal((M, K), dtype, 1), normal((N, K), dtype, 2, 0.1)
    dy, z = normal((M, N), dtype, 3), normal((M, N), dtype, 4)
    (want, tol), _ = ref.forward(x, w, None, "none", None)
    x[301, 650], x[5, 2], w[77, 300] = math.inf, math.nan, -math.inf
    y = pic.linear(x, w)
    assert bool(torch.isnan(y[5]).all())
    assert torch.equal(y[301][:77], torch.sign(w[:77, 650]) * math.inf)
    keep_r = torch.ones(M, dtype=torch.bool, device="cuda")
    keep_r[301] = keep_r[5] = False
    assert torch.equal(y[keep_r, 77], torch.sign(x[keep_r, 300]) * -math.inf)
    cols = torch.ones(N, dtype=torch.bool, device="cuda")
    cols[77] = False
    ref.check(y[keep_r][:, cols], (want[keep_r][:, cols], tol[keep_r][:, cols]))
    dy[17, 33] = math.inf
    dx, dw, db = pic.linear_backward(dy, x.clamp(-4, 4).nan_to_num(), w.clamp(-4, 4), need=("x", "weight", "bias"))
    assert bool(dx[17].isinf().all()) and bool(dw[33].isinf().all()) and float(db[33]) == math.inf
    assert not bool(dx[:17].isinf().any()) and int(dw.isinf().any(1).sum()) == 1 and not bool(dw.isnan().any())


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("rows", [4, 20, 150])
def test_infinities_and_nan(rows, dtype):
    """A NaN or infinite row changes its own row alone; activations take the
    limits of their functions."""
    from paper_2609_09020_gb300 import pic
    K, N = 72, 40
    x, w = normal((rows, K), dtype, 1), normal((N, K), dtype, 2, 0.1)
    want, _ = ref.forward(x, w, None, "gelu", None)
    x[1, 3] = math.nan
    w[:, 5] = 0.5
    w[::2, 5] = -0.5
    want, _ = ref.forward(torch.where(torch.isnan(x), 0.0, x), w, None, "gelu", None)
    x[2, 5] = math.inf
    y = pic.linear(x, w, act="gelu")
    keep = [i for i in range(rows) if i not in (1, 2)]
    ref.check(y[keep], (want[0][keep], want[1][keep]))
    assert bool(torch.isnan(y[1]).all())
    assert bool((y[2, ::2] == 0).all()) and bool((y[2, 1::2] == math.inf).all())
    r = pic.linear(x, w, act="relu")
    assert bool(torch.isnan(r[1]).all()) and bool((r[2, ::2] == 0).all())
    # gradients: act'(inf) = 1, act'(-inf) = 0, and a zero derivative beats any dy
    z = torch.zeros((rows, N), dtype=dtype, device="cuda")
    z[:, 0], z[:, 1], z[:, 2] = math.inf, -math.inf, -3.0
    dy = torch.ones((rows, N), dtype=dtype, device="cuda")
    for act in ("relu", "gelu"):
        _, _, db = pic.linear_backward(dy, x, w, act=act, pre=z, need=("bias",))
        assert float(db[0]) == rows and float(db[1]) == 0
    dy[:, 2] = math.inf
    _, _, db = pic.linear_backward(dy, x, w, act="relu", pre=z, need=("bias",))
    assert float(db[2]) == 0


def test_other_stream():
    """On a stream that is not torch's current one, behind work of that stream."""
    from paper_2609_09020_gb300 import pic
    s = torch.cuda.Stream()
    x, w = normal((700, 264), torch.bfloat16, 1), normal((300, 264), torch.bfloat16, 2, 0.1)
    want, _ = ref.forward(x, w, None, "gelu", None)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        late = torch.zeros_like(x)
        torch.cuda._sleep(20_000_000)
        late.copy_(x)
    for stream in (s, s.cuda_stream):
        y, z = pic.linear(late, w, act="gelu", save_pre=True, stream=stream)
        g = pic.linear_backward(y, late, w, act="gelu", pre=z, stream=stream)
        junk = [torch.full((1 << 20,), 3.0, device="cuda") for _ in range(8)]  # may take freed workspaces
        s.synchronize()
        ref.check(y, want)
        for a, v in zip(g, ref.backward(y, x, w, z, "gelu")):
            ref.check(a, v)
        del junk
    pic.linear_check(s)


@pytest.mark.parametrize("act", ["none", "gelu"])
def test_gradient_against_differences(act):
    """d/dt of sum(c * y) along random directions of x, w and b, by central
    differences of the fp32 forward pass.  f = sum(c y) is summed in fp64; its
    fp32 outputs are off by at most e = (K + 32) 2^-23 S each (random signs: 6
    standard deviations of the sum of c e over them), which a difference over
    2h divides; the third-order term is below h^2 times the sum of |c| |dz|^3
    (|gelu'''| < 1)."""
    from paper_2609_09020_gb300 import pic
    M, K, N, h = 37, 29, 23, 2.0 ** -7
    f32 = torch.float32
    x, w, b = normal((M, K), f32, 1), normal((N, K), f32, 2, 0.3), normal((N,), f32, 3)
    c = normal((M, N), f32, 4)
    _, z = pic.linear(x, w, b, act=act, save_pre=True)
    dx, dw, db = pic.linear_backward(c, x, w, act=act, pre=z)

    def f(t, ux, uw, ub):
        return float((c.double() * pic.linear(x + t * ux, w + t * uw, b + t * ub, act=act).double()).sum())

    zero = [torch.zeros_like(v) for v in (x, w, b)]
    (_, e), _ = ref.forward(x, w, b, act, None)
    for i, g in enumerate((dx, dw, db)):
        u = list(zero)
        u[i] = normal(g.shape, f32, 7 + i).mul_(0.5)
        # steps that fp32 holds exactly: round the direction to 8 bits
        u[i] = u[i].bfloat16().float()
        slope = float((g.double() * u[i].double()).sum())
        diff = (f(h, *u) - f(-h, *u)) / (2 * h)
        dz = u[0].double() @ w.double().t() if i == 0 else (x.double() @ u[1].double().t() if i == 1 else u[2].double())
        third = h * h * float((c.double().abs() * dz.abs() ** 3).sum())
        step = 2.0 ** -24 * 8 / h * float((c.double().abs() * (x.abs().double() @ w.abs().double().t() + 1)).norm())
        noise = 6 * float((c.double() * e).norm()) * math.sqrt(2) / (2 * h)
        assert abs(slope - diff) <= noise + third + step, (i, slope, diff, noise, third, step)


def test_tolerances_catch_mistakes():
    """The bounds are tight enough to see one dropped term, one row's bias and
    a wrong activation derivative (planted in the reference, on small data)."""
    x, w, b = torch.randn(8, 64), torch.randn(16, 64) / 8, torch.randn(16) * 0.1
    (y, tol), _ = ref.forward(x.bfloat16(), w.bfloat16(), b.bfloat16(), "gelu", None)
    x2 = x.bfloat16().clone()
    x2[:, 63] = 0
    (y2, _), _ = ref.forward(x2, w.bfloat16(), b.bfloat16(), "gelu", None)
    (y3, _), _ = ref.forward(x.bfloat16(), w.bfloat16(), None, "gelu", None)
    assert float(((y2 - y).abs() > tol).double().mean()) > 0.5
    assert float(((y3 - y).abs() > tol).double().mean()) > 0.5


def shifted(rows, cols, dtype, seed, ld, shift, std=1.0):
    """A [rows][cols] view with `ld` elements from row to row, `shift` past a boundary; NaN around it."""
    t = torch.full((rows * ld + cols + shift,), math.nan, dtype=dtype, device="cuda")
    v = torch.as_strided(t, (rows, cols), (ld, 1), shift)
    v.copy_(normal((rows, cols), dtype, seed, std))
    return v


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("place", [(0, 0), (0, 1), (3, 2), (8, 8), (16, 0)], ids=str)  # columns between rows, shift
@pytest.mark.parametrize("size", [(16, 16, 16), (17, 64, 64), (333, 40, 44), (250, 33, 24), (1000, 128, 128), (95, 111, 77),
                                  (4111, 3, 96), (2600, 72, 5), (31, 127, 121), (40, 1, 33)], ids=str)
def test_narrow_places(size, place, dtype):
    """Narrow layers whose matrices lie in wider ones, on and off 16-byte boundaries; nothing around is read or written."""
    from paper_2609_09020_gb300 import pic
    M, K, N = size
    pad, shift = place
    x, w = shifted(M, K, dtype, 1, K + pad, shift), shifted(N, K, dtype, 2, K + pad, shift, 1.4 / math.sqrt(K))
    b, r = normal((N,), dtype, 3, 0.1), shifted(M, N, dtype, 4, N + pad, shift)
    out = shifted(M, N, dtype, 5, N + pad, shift)
    whole = torch.as_strided(out, (M * (N + pad) + N + shift,), (1,), 0)
    kept = torch.isnan(whole).clone()
    for act, res in (("none", r), ("relu", None), ("gelu", r)):
        want_y, want_z = ref.forward(x, w, b, act, res)
        y, z = pic.linear(x, w, b, act=act, residual=res, out=out, save_pre=True)
        assert y is out
        ref.check(y, want_y, "y")
        ref.check(z, want_z, "pre")
        assert torch.equal(torch.isnan(whole), kept)
        ref.check(pic.linear(x, w, b, act=act, residual=res), want_y, "y")
    pic.linear_check()


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("pad", [0, 3])
def test_narrow_nonfinite(pad, dtype):
    """Infinite and NaN values in rows and weights of a narrow layer stay in their rows and columns."""
    from paper_2609_09020_gb300 import pic
    M, K, N = 3000, 45, 50
    x, w = shifted(M, K, dtype, 1, K + pad, 0), normal((N, K), dtype, 2, 0.2)
    want, tol = ref.forward(x, w, None, "none", None)[0]
    x[7, 44], x[1234, 0], x[2999, 20] = math.inf, math.nan, -math.inf
    y = pic.linear(x, w)
    keep = torch.ones(M, dtype=torch.bool, device="cuda")
    keep[7] = keep[1234] = keep[2999] = False
    ref.check(y[keep], (want[keep], tol[keep]))
    assert torch.equal(y[7], torch.sign(w[:, 44]) * math.inf) and bool(torch.isnan(y[1234]).all())
    assert torch.equal(y[2999], torch.sign(w[:, 20]) * -math.inf)
    x = normal((M, K), dtype, 1).abs() + 0.5
    want, tol = ref.forward(x, w, None, "none", None)[0]
    w[49, 44] = -math.inf
    y = pic.linear(x, w)
    assert bool((y[:, 49] == -math.inf).all())
    ref.check(y[:, :49], (want[:, :49], tol[:, :49]))


@pytest.mark.parametrize("size", [(9, 700, 9000), (33, 2100, 5003), (64, 4097, 2050), (10, 130, 30000)], ids=str)
def test_fp32_few_rows_many_columns(size):
    """fp32 with fewer rows than a tile over wide outputs, infinities and gradients included."""
    from paper_2609_09020_gb300 import pic
    M, K, N = size
    dtype = torch.float32
    x, w = normal((M, K), dtype, 1), normal((N, K), dtype, 2, 1.4 / math.sqrt(K))
    b, r, dy = normal((N,), dtype, 3, 0.1), normal((M, N), dtype, 4), normal((M, N), dtype, 5, 0.1)
    for act, res in (("gelu", r), ("none", None)):
        y, z = pic.linear(x, w, b, act=act, residual=res, save_pre=True)
        want_y, want_z = ref.forward(x, w, b, act, res)
        ref.check(y, want_y, "y")
        ref.check(z, want_z, "pre")
        assert torch.equal(y, pic.linear(x, w, b, act=act, residual=res))
    got = pic.linear_backward(dy, x, w, act="gelu", pre=z)
    for g, v, name in zip(got, ref.backward(dy, x, w, z, "gelu"), ("dx", "dw", "db")):
        ref.check(g, v, name)
    x[M - 1, 5] = math.inf
    want = torch.sign(w[:, 5]) * math.inf
    y2 = pic.linear(x, w, b)
    assert torch.equal(y2[M - 1], want)
    ref.check(y2[:M - 1], tuple(t[:M - 1] for t in ref.forward(x[:M - 1], w, b, "none", None)[0]), "y")
    pic.linear_check()
