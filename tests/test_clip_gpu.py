"""pic.GradClip against the definition in fp64.  The norm: a thread adds at most
64 squares in fp32 (65 roundings of 2^-24, about 2^-18 of their sum), the rest
is fp64 and one rounding; the square root halves the relative error."""
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
ROUND = {F32: 2.0 ** -24, F16: 2.0 ** -11, BF16: 2.0 ** -8}
TINY = {F32: 2.0 ** -149, F16: 2.0 ** -25, BF16: 2.0 ** -134}
NORM_TOL = 2.0 ** -18  # half of (64 + 1) 2^-24 of the squares' sum, and its rounding


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_09020_gb300 import build
    build.build()


def make(n, dtype, seed, front=0, std=0.3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(front + n, generator=g, device="cuda").mul_(std).to(dtype)[front:]


def norm64(tensors):
    return math.sqrt(sum(float((t.double() ** 2).sum()) for t in tensors))


def check(norm, outs, grads, max_norm):
    want = norm64(grads)
    assert abs(float(norm) - want) <= NORM_TOL * want
    coef = min(1.0, max_norm / (want + 1e-6))
    for o, g in zip(outs, grads):
        v = g.double() * coef
        # coef: the norm's error, the sum and the quotient, the product
        tol = (NORM_TOL + 4 * 2.0 ** -24 + ROUND[o.dtype] * (1 + 2.0 ** -10)) * v.abs() + TINY[o.dtype]
        assert bool(((o.double() - v).abs() <= tol).all())


LISTS = {
    "one": [(1, F32, 0)],
    "one_odd": [(3, F16, 1)],
    "empty_ones": [(0, F32, 0), (5, BF16, 0), (0, F16, 0)],
    "net_7_64_64_3": [(448, F32, 0), (64, F32, 0), (4096, F32, 0), (64, F32, 0), (192, F32, 0), (3, F32, 0)] * 5,
    "offsets": [(n, t, f) for t in (F32, F16, BF16) for f in range(9) for n in (1, 7, 8, 9, 1023)],
    "chunk_edges": [(n, t, f) for t in (F32, F16, BF16) for n in (32767, 32768, 32769, 65537) for f in (0, 1)],
    "large": [(3_000_001, F32, 0), (5_000_000, BF16, 1), (40_000_001, F16, 0)],
    "many": [(17 + i % 50, (F32, F16, BF16)[i % 3], i % 4) for i in range(3000)],
}


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("name", LISTS)
def test_clip(name, in_place):
    from paper_2609_09020_gb300 import pic
    grads = [make(n, t, 10 + i, f) for i, (n, t, f) in enumerate(LISTS[name])]
    kept = [g.clone() for g in grads]
    outs = grads if in_place else [torch.full_like(g, 5.0) for g in grads]
    clip = pic.GradClip(grads, out=None if in_place else outs)
    total = norm64(kept)
    for max_norm in (4 * total, 0.5 * total, math.inf, 0.0):  # in place, the last ones have clipped input
        before = [g.clone() for g in grads]
        norm = clip.clip(max_norm)
        assert norm.shape == () and norm.dtype == F32
        check(norm, outs, before, max_norm)
    if not in_place:
        assert all(torch.equal(a, b) for a, b in zip(grads, kept))
    clip.close()


def test_neighbours_are_untouched():
    """Slices of one buffer with gaps: nothing is written between them."""
    from paper_2609_09020_gb300 import pic
    for dtype in (F32, F16, BF16):
        buf = make(20000, dtype, 3)
        ref = buf.clone()
        cuts = [(0, 3), (5, 100), (101, 4097), (4097, 4200), (4203, 19999)]
        grads = [buf[a:b] for a, b in cuts]
        want = [g.clone() for g in grads]
        norm = pic.GradClip(grads).clip(0.01)
        check(norm, grads, want, 0.01)
        inside = torch.zeros(20000, dtype=torch.bool, device="cuda")
        for a, b in cuts:
            inside[a:b] = True
        assert torch.equal(buf[~inside], ref[~inside])


def test_new_values_each_call():
    """The handle keeps the tensors, not what was in them."""
    from paper_2609_09020_gb300 import pic
    g = [make(5000, F32, 1), make(77, BF16, 2)]
    outs = [torch.empty_like(t) for t in g]
    clip = pic.GradClip(g, out=outs)
    for seed in range(5):
        for i, t in enumerate(g):
            t.copy_(make(t.numel(), t.dtype, 100 * seed + i, std=10.0 ** (seed - 2)))
        check(clip.clip(1.0), outs, g, 1.0)


def test_no_tensors_and_zeros():
    from paper_2609_09020_gb300 import pic
    assert float(pic.GradClip([]).clip(1.0)) == 0.0
    z = [torch.zeros(100000, dtype=t, device="cuda") for t in (F32, F16, BF16)]
    norm = pic.GradClip(z).clip(1.0)
    assert float(norm) == 0.0 and not any(bool(t.any()) for t in z)


@pytest.mark.parametrize("size", [1e30, 1e-30, 3e38, 1e-42])
def test_extreme_sizes(size):
    """Squares outside fp32's range: the norm is right all the same."""
    from paper_2609_09020_gb300 import pic
    g = [torch.full((1000,), size, device="cuda"), torch.zeros(70000, device="cuda")]
    g[1][::2] = size * 0.5 if size < 1e38 else 0.0
    if size == 3e38:
        g[0] = g[0][:1]
    want = norm64(g)
    out = [torch.empty_like(t) for t in g]
    norm = pic.GradClip(g, out=out).clip(1e-3 * want)
    assert abs(float(norm) - want) <= NORM_TOL * want + 2.0 ** -149
    if size > 1:
        check(norm, out, g, 1e-3 * want)


def test_infinite_and_nan():
    from paper_2609_09020_gb300 import pic
    for dtype in (F32, F16, BF16):
        g = make(5000, dtype, 1)
        g[1234] = math.inf
        out = torch.empty_like(g)
        norm = pic.GradClip([g], out=[out]).clip(1.0)
        assert float(norm) == math.inf
        assert math.isnan(float(out[1234])) and int(torch.isnan(out).sum()) == 1  # inf * 0
        assert not bool(out[:1234].any())
        g[7] = math.nan
        norm = pic.GradClip([g], out=[out]).clip(1.0)
        assert math.isnan(float(norm)) and bool(torch.isnan(out).all())


def test_repeatable():
    from paper_2609_09020_gb300 import pic
    g = [make(1_000_003, F32, 1), make(2_000_001, BF16, 2, front=1)]
    out = [torch.empty_like(t) for t in g]
    clip = pic.GradClip(g, out=out)
    first, kept = float(clip.clip(1.0)), None
    kept = [o.clone() for o in out]
    for _ in range(10):
        assert float(clip.clip(1.0)) == first
        assert all(torch.equal(a, b) for a, b in zip(out, kept))


def test_other_stream():
    from paper_2609_09020_gb300 import pic
    s = torch.cuda.Stream()
    src = make(300000, F32, 1)
    g, out = torch.zeros_like(src), torch.empty_like(src)
    clip = pic.GradClip([g], out=[out])
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        g.copy_(src)
    norm = clip.clip(1.0, stream=s)
    s.synchronize()
    check(norm, [out], [src], 1.0)


def test_refusals():
    from paper_2609_09020_gb300 import pic
    g = make(100, F32, 1)
    clip = pic.GradClip([g])
    for bad in (-1.0, math.nan):
        with pytest.raises(pic.PicError):
            clip.clip(bad)
    clip.close()
    with pytest.raises(ValueError):
        clip.clip(1.0)
    with pytest.raises(ValueError):
        pic.GradClip([g], out=[])
    with pytest.raises(ValueError):
        pic.GradClip([g], out=[g.half()])
    with pytest.raises(ValueError):
        pic.GradClip([make(100, F32, 1).view(10, 10).t()])
    with pytest.raises(ValueError):
        pic.GradClip([torch.zeros(4, dtype=torch.float64, device="cuda")])
    with pytest.raises(pic.PicError):
        pic.GradClip([g, g])
    with pytest.raises(pic.PicError):
        pic.GradClip([g[:50]], out=[g[1:51]])


def test_linear_refusals():
    from paper_2609_09020_gb300 import pic
    x, w = make(48, F16, 1).view(3, 16), make(128, F16, 2).view(8, 16)
    dy = make(24, F16, 3).view(3, 8)
    bad = [dict(act="tanh"), dict(bias=make(7, F16, 1)), dict(bias=make(8, F32, 1)),
           dict(residual=make(16, F16, 1).view(2, 8)), dict(out=make(24, F16, 1).view(8, 3).t()),
           dict(out=make(27, F16, 1).view(3, 9))]
    for kw in bad:
        with pytest.raises(ValueError):
            pic.linear(x, w, **kw)
    for xx, ww in ((x.float(), w), (x, w[:, :15]), (x[:1].expand(3, 16), w), (x, w.view(-1)), (x.double(), w.double())):
        with pytest.raises(ValueError):
            pic.linear(xx, ww)
    with pytest.raises(ValueError):
        pic.linear_backward(dy, x, w, act="gelu")
    with pytest.raises(ValueError):
        pic.linear_backward(dy, x, w, need=("y",))
    with pytest.raises(ValueError):
        pic.linear_backward(dy[:2], x, w)
