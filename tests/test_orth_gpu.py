"""pic.Orthogonalizer against the definition in fp64 (orth_ref's bounds)."""
import pytest
import torch

import orth_ref as ref

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
TYPES = [F32, F16, BF16]


@pytest.fixture(scope="module")
def pic():
    from paper_2609_09020_gb300 import build, pic
    build.build()
    return pic


def normal(shape, dtype=F32, seed=0, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def run(pic, tensors, **kw):
    out = [torch.full_like(t, 7.0) for t in tensors]
    h = pic.Orthogonalizer(tensors, out=out)
    h.orthogonalize(**kw)
    h.check()
    h.close()
    return out


SHAPES = [(1, 1), (1, 7), (9, 1), (2, 3), (7, 64), (64, 7), (64, 64), (3, 64), (65, 64), (64, 200), (100, 33), (128, 128),
          (127, 130), (129, 129), (200, 300), (256, 256), (300, 200), (257, 640), (500, 70), (70, 500), (513, 385)]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_shapes(pic, shape, dtype):
    g = normal(shape, dtype, seed=shape[0], scale=0.02)
    ref.check(run(pic, [g])[0], g)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("shape", [(1024, 1024), (768, 2304), (2048, 640), (1000, 1100)], ids=str)
def test_larger(pic, shape, dtype):
    g = normal(shape, dtype, seed=1, scale=0.02)
    ref.check(run(pic, [g])[0], g)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("steps", [0, 1, 2, 3, 4, 5])
def test_steps_of_long_and_small_matrices(pic, dtype, steps):
    """By tiles and by one CTA, and how many halves a product has goes by the step."""
    cases = [normal(s, dtype, seed=3, scale=0.02) for s in ((64, 4096), (6000, 48), (128, 1100), (64, 64), (8, 500), (100, 90))]
    for g in cases:
        ref.check(run(pic, [g], steps=steps)[0], g, steps=steps, name=f"{tuple(g.shape)}")
    for g, o in zip(cases, run(pic, cases, steps=steps)):
        ref.check(o, g, steps=steps, name=f"{tuple(g.shape)} of several")


@pytest.mark.parametrize("steps", [1, 5])
@pytest.mark.parametrize("shape", [(4, 572), (4, 454), (2, 900), (639, 4), (779, 2), (4, 9000), (2000, 16000)], ids=str)
def test_long_sums(pic, shape, steps):
    """Sums far longer than they are many: what each addition loses adds up."""
    for seed in range(1 if shape[0] == 2000 else 4):
        g = normal(shape, F32, seed=seed, scale=0.02)
        ref.check(run(pic, [g], steps=steps)[0], g, steps=steps, name=f"seed {seed}")


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("shape", [(64, 64), (48, 100), (160, 160), (320, 200)], ids=str)
def test_few_directions(pic, shape, dtype):
    """One direction; eight; eight and noise; singular values over six decades; equal rows; one element."""
    r, c = shape
    few = normal((r, 8), seed=1) @ normal((8, c), seed=2)
    u, _ = torch.linalg.qr(normal((r, r), seed=3))
    v, _ = torch.linalg.qr(normal((c, c), seed=4))
    n = min(r, c)
    decay = u[:, :n] * torch.logspace(0, -6, n, device="cuda") @ v[:, :n].t()
    one = torch.zeros(shape, device="cuda")
    one[r // 2, c - 1] = -3.0
    cases = [normal((r, 1), seed=5) @ normal((1, c), seed=6), few, few + normal(shape, seed=7, scale=0.01), decay,
             torch.ones(shape, device="cuda"), one, torch.eye(r, c, device="cuda")]
    cases = [t.to(dtype) for t in cases]
    for i, (g, o) in enumerate(zip(cases, run(pic, cases))):
        ref.check(o, g, name=f"case {i}")


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_sizes_of_values(pic, dtype):
    """Norms at both ends of the type's range, where squares leave fp32's."""
    top = 60000.0 if dtype == F16 else 1e38
    low = 1e-6 if dtype == F16 else 1e-36
    for shape in ((40, 30), (200, 180)):
        g = normal(shape, F32, seed=2).clamp(-3, 3) / 3
        cases = [(g * top).to(dtype), (g * low).to(dtype), torch.zeros(shape, dtype=dtype, device="cuda")]
        for scale, t, o in zip((top, low, 0), cases, run(pic, cases, eps=0.0 if dtype != F16 else 1e-30)[:2]):
            ref.check(o, t, eps=0.0 if dtype != F16 else 1e-30, name=str(scale))
        zero = run(pic, [cases[2], cases[0]])
        assert not zero[0].any()


def test_eps(pic):
    g = normal((90, 70), F32, seed=3, scale=1e-5)
    ref.check(run(pic, [g], eps=1e-3)[0], g, eps=1e-3)
    z = torch.zeros((90, 70), device="cuda")
    assert run(pic, [z], eps=0.0)[0].isnan().all()


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("steps", [0, 1, 2, 3, 6, 10])
def test_steps(pic, steps, dtype):
    for shape in ((64, 40), (150, 260)):
        g = normal(shape, dtype, seed=4)
        ref.check(run(pic, [g], steps=steps)[0], g, steps=steps)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_other_coefficients(pic, dtype):
    """Plain Newton-Schulz (3/2, -1/2) and the quintic that converges (15/8, -10/8, 3/8)."""
    for shape in ((64, 40), (150, 260)):
        g = normal(shape, dtype, seed=5)
        for co in ((1.5, -0.5, 0.0), (1.875, -1.25, 0.375), (1.0, 0.0, 0.0)):
            ref.check(run(pic, [g], coefficients=co, steps=8)[0], g, coefficients=co, steps=8)


def test_a_list(pic):
    """Matrices of all types and shapes at once, slices of one buffer and of wider tensors, 3-D tensors, and empty
    ones."""
    buf = normal((40000,), F32, seed=6)
    stack = normal((5, 48, 33), F16, seed=7)
    tensors = [buf[1:1 + 64 * 7].view(64, 7), buf[449:449 + 64 * 64].view(64, 64), normal((300, 200), BF16, seed=8),
               normal((130, 260), F16, seed=9)[:, 3:250], normal((90, 40), BF16, seed=10)[:, 1:38], stack,
               normal((0, 5), F32), normal((4, 0), F32), normal((3, 1000), F32, seed=11), normal((1025, 40), F32, seed=12),
               normal((6, 70, 90), F32, seed=13)[1:5, 2:, :80], normal((2000, 3), BF16, seed=14)]
    got = run(pic, tensors)
    for i, (t, o) in enumerate(zip(tensors, got)):
        if t.dim() == 3:
            for j in range(t.shape[0]):
                ref.check(o[j], t[j], name=f"{i}.{j}")
        elif t.numel():
            ref.check(o, t, name=str(i))


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_in_place_and_beside(pic, dtype):
    """In place, into columns of a wider tensor whose rest stays, and the same every time."""
    for shape in ((64, 64), (200, 130)):
        g = normal(shape, dtype, seed=15)
        want = run(pic, [g])[0]
        mine = g.clone()
        h = pic.Orthogonalizer([mine])
        h.orthogonalize()
        h.check()
        assert torch.equal(mine, want)
        h.close()
        wide = torch.full((shape[0], shape[1] + 5), 3.0, dtype=dtype, device="cuda")
        h = pic.Orthogonalizer([g], out=[wide[:, 2:2 + shape[1]]])
        for _ in range(2):
            h.orthogonalize()
            assert torch.equal(wide[:, 2:2 + shape[1]], want)
        assert bool((wide[:, :2] == 3).all()) and bool((wide[:, 2 + shape[1]:] == 3).all())
        h.check()


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_not_finite(pic, bad, dtype):
    """All of its own matrix is NaN, and no other's."""
    for shape in ((64, 40), (150, 260), (300, 129)):
        a, b, c = (normal(shape, dtype, seed=s) for s in (16, 17, 18))
        b[shape[0] // 2, 5] = bad
        got = run(pic, [a, b, c])
        assert bool(got[1].isnan().all())
        for t, o in ((a, got[0]), (c, got[2])):
            ref.check(o, t)
        same = run(pic, [a, torch.zeros_like(b), c])
        assert torch.equal(same[0], got[0]) and torch.equal(same[2], got[2])


def test_captured_and_other_streams(pic):
    tensors = [normal((64, 64), F32, seed=19), normal((300, 140), BF16, seed=20), normal((140, 300), F16, seed=21)]
    out = [torch.zeros_like(t) for t in tensors]
    want = run(pic, tensors)
    h = pic.Orthogonalizer(tensors, out=out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    h.orthogonalize(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h.orthogonalize()
    for seed in (30, 40):
        for i, t in enumerate(tensors):
            t.copy_(normal(t.shape, t.dtype, seed + i))
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in out]
        assert all(torch.equal(a, b) for a, b in zip(got, run(pic, tensors)))
    h.check()


def test_many_matrices(pic):
    nets = [normal((64, 7), F32, seed=s) for s in range(200)] + [normal((64, 64), F32, seed=s) for s in range(200)]
    for t, o in list(zip(nets, run(pic, nets)))[::37]:
        ref.check(o, t)


def test_offsets_past_32_bits(pic):
    """A matrix of more than 2^31 elements: zeros but for columns at both ends, which come to
    what the matrix of these columns alone does."""
    rows, cols = 20, 2 ** 27 + 40
    at = torch.cat([torch.arange(0, 77), torch.arange(cols - 300, cols)]).cuda()
    few = normal((rows, len(at)), BF16, seed=22)
    g = torch.zeros((rows, cols), dtype=BF16, device="cuda")
    g[:, at] = few
    h = pic.Orthogonalizer([g])
    h.orthogonalize()
    h.check()
    h.close()
    ref.check(g[:, at], few)
    g[:, at] = 0
    assert not g.any()


def test_refusals(pic):
    z = lambda *s, **o: torch.zeros(s, device="cuda", **o)
    buf = z(100)
    for bad in (dict(tensors=[z(5)]), dict(tensors=[z(2, 2, 2, 2)]), dict(tensors=[z(4, 5).double()]),
                dict(tensors=[torch.zeros(4, 5)]), dict(tensors=[z(5, 4).t()]), dict(tensors=[z(1, 5).expand(4, 5)]),
                dict(tensors=[z(1, 4, 5).expand(3, 4, 5)]), dict(tensors=[z(4, 5)], out=[]),
                dict(tensors=[z(4, 5)], out=[z(5, 4)]), dict(tensors=[z(4, 5)], out=[z(4, 5).half()])):
        with pytest.raises(ValueError):
            pic.Orthogonalizer(**bad)
    for tensors, out in (([buf[:20].view(4, 5), buf[10:30].view(4, 5)], None),
                         ([z(4, 5)] * 2, None), ([z(4, 5), z(4, 5)], [buf[:20].view(4, 5), buf[19:39].view(4, 5)]),
                         ([buf[:20].view(4, 5), z(4, 5)], [z(4, 5), buf[:20].view(4, 5)]),
                         ([buf[:20].view(4, 5)], [buf[5:25].view(4, 5)])):
        with pytest.raises(pic.PicError):
            pic.Orthogonalizer(tensors, out=out)
    wide = z(6, 20)
    pic.Orthogonalizer([wide[:, :7], wide[:, 7:12], wide[1:, 12:]]).close()
    h = pic.Orthogonalizer([z(4, 5)])
    for bad in (dict(steps=-1), dict(steps=65), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
                dict(coefficients=(3.0, 1.0, 1.0)), dict(coefficients=(float("nan"), 0.0, 0.0)),
                dict(coefficients=(2.5, 0.0, 0.0)), dict(coefficients=(1.0, -13.0, 13.0), steps=1)):
        with pytest.raises(pic.PicError):
            h.orthogonalize(**bad)
    h.close()
    with pytest.raises(ValueError):
        h.orthogonalize()
