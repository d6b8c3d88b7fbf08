"""Sums that have one right value: the data are small integers, so that every partial
sum is an integer below 2^24 in any order, and each output is the exact sum rounded once
to its type.  A tile of rows that is left out, added twice or taken from another call
shows in most of the outputs, which rounding bounds over this many rows do not see
(test_a_lost_tile_is_seen, on the CPU)."""
import pytest

torch = pytest.importorskip("torch")

TYPES = [torch.float32, torch.float16, torch.bfloat16]
IDS = ["fp32", "fp16", "bf16"]
# several tiles of 128 rows for each of 152 CTAs, the last ones not whole
SIZES = [(25000, 7, 40), (30011, 64, 64), (40000, 128, 96), (70001, 8, 16), (50001, 33, 64), (120007, 40, 40),
         (59000, 64, 3), (41003, 100, 128)]


def whole(shape, dtype, seed, most, device, pad=0):
    """Integers from -most to most, in rows `pad` elements apart."""
    g = torch.Generator(device=device).manual_seed(seed)
    t = torch.randint(-most, most + 1, (shape[0], shape[1] + pad), generator=g, device=device, dtype=torch.int8)
    return t.to(dtype)[:, :shape[1]]


def gate(shape, dtype, seed, device, pad=0):
    """Pre-activations of +-8, where the derivatives of ReLU and of GELU are 1 and 0 in fp32."""
    return whole(shape, dtype, seed, 1, device, pad).ge(0).to(dtype).mul_(16).sub_(8)


def gradients64(dy, x, w, z, act):
    dz = dy.double() if act == "none" else torch.where(z > 0, dy, torch.zeros_like(dy)).double()
    return dz @ w.double(), dz.t() @ x.double(), dz.sum(0)


@pytest.fixture(scope="module")
def pic():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_09020_gb300 import build, pic
    build.build()
    return pic


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("pad", [0, 3, 8])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_narrow_gradient(pic, size, pad, dtype):
    M, K, N = size
    x, dy = whole((M, K), dtype, 1, 2, "cuda", pad), whole((M, N), dtype, 2, 2, "cuda", pad)
    w, z = whole((N, K), dtype, 3, 2, "cuda", pad), gate((M, N), dtype, 4, "cuda", pad)
    for act in ("none", "relu", "gelu"):
        want = gradients64(dy, x, w, z, act)
        got = pic.linear_backward(dy, x, w, act=act, pre=z)
        for g, v, name in zip(got, want, ("dx", "dw", "db")):
            assert torch.equal(g, v.to(dtype)), (act, name)
        one = pic.linear_backward(dy, x, w, act=act, pre=z, need=("weight", "bias"))
        assert torch.equal(one[1], got[1]) and torch.equal(one[2], got[2])
    pic.linear_check()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("size", [(9000, 200, 136), (4000, 520, 700), (600, 2048, 96), (20001, 65, 129), (40, 300, 5000),
                                  (12, 500, 260)], ids=str)
def test_gradient(pic, size, dtype):
    M, K, N = size
    x, dy = whole((M, K), dtype, 1, 2, "cuda"), whole((M, N), dtype, 2, 2, "cuda")
    w, z = whole((N, K), dtype, 3, 2, "cuda"), gate((M, N), dtype, 4, "cuda")
    for act in ("none", "relu", "gelu"):
        got = pic.linear_backward(dy, x, w, act=act, pre=z)
        for g, v, name in zip(got, gradients64(dy, x, w, z, act), ("dx", "dw", "db")):
            assert torch.equal(g, v.to(dtype)), (act, name)
    pic.linear_check()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("size", [(25000, 7, 40), (70001, 64, 64), (40000, 128, 96), (20000, 136, 200), (3000, 4100, 300),
                                  (600, 20000, 500), (24, 5000, 3000), (3, 4000, 700)], ids=str)
def test_forward(pic, size, dtype):
    M, K, N = size
    x, w = whole((M, K), dtype, 1, 2, "cuda"), whole((N, K), dtype, 2, 2, "cuda")
    b, r = whole((1, N), dtype, 3, 4, "cuda")[0], whole((M, N), dtype, 4, 9, "cuda")
    z = x.double() @ w.double().t() + b.double()
    y, pre = pic.linear(x, w, b, act="relu", residual=r, save_pre=True)
    pic.linear_check()
    assert torch.equal(pre, z.to(dtype)) and torch.equal(y, (z.clamp(min=0) + r.double()).to(dtype))


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_a_lost_tile_is_seen(size, dtype):
    """Gradients that lack 128 of the rows, or have them twice, are not those of test_narrow_gradient."""
    M, K, N = size
    x, dy, w = whole((M, K), dtype, 1, 2, "cpu"), whole((M, N), dtype, 2, 2, "cpu"), whole((N, K), dtype, 3, 2, "cpu")
    _, dw, db = gradients64(dy, x, w, None, "none")
    first = 128 * (M // 256)
    tile = slice(first, first + 128)
    part_w, part_b = dy[tile].double().t() @ x[tile].double(), dy[tile].double().sum(0)
    for sign in (-1, 1):
        assert float(((dw + sign * part_w).to(dtype) != dw.to(dtype)).double().mean()) > 0.5
        assert bool(((db + sign * part_b).to(dtype) != db.to(dtype)).any())


@pytest.mark.parametrize("act,other", [("relu", "none"), ("none", "relu")])
def test_a_wrong_derivative_is_seen(act, other):
    """Both in the exact gradients here and in the rounding bounds of linear_ref."""
    import linear_ref as ref
    M, K, N = 300, 20, 30
    g = torch.Generator().manual_seed(5)
    x, dy, w, z = (torch.randn(s, generator=g).bfloat16() for s in ((M, K), (M, N), (N, K), (M, N)))
    for (v, tol), (u, _) in zip(ref.backward(dy, x, w, z, act), ref.backward(dy, x, w, z, other)):
        assert float(((u - v).abs() > tol).double().mean()) > 0.5
    for (v, tol), (u, _) in zip(ref.backward(dy, x, w, z, "gelu"), ref.backward(dy, x, w, z, "relu")):
        assert float(((u - v).abs() > tol).double().mean()) > 0.3
    z = gate((M, N), torch.bfloat16, 4, "cpu")
    xi, dyi, wi = (whole(s, torch.bfloat16, i, 2, "cpu") for i, s in enumerate(((M, K), (M, N), (N, K))))
    for a, b in zip(gradients64(dyi, xi, wi, z, act), gradients64(dyi, xi, wi, z, other)):
        assert float((a != b).double().mean()) > 0.5
