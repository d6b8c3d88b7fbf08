"""That bfloat16 matrices of up to 64 on the smaller side, and those that one CTA takes,
are held in two halves, as include/pic_orth.h says: out is the rounded value of one that
is near the definition's.

Bound.  out = the nearest bfloat16 to v, and v is off by at most E: four times the largest
that the steps are off by with two halves (emulated, products and sums in fp64) or in fp32,
and 2^-18 (as orth_ref has it).  Then |out - exact| <= half a unit of |exact| + E, plus E.
Held in one half, the steps are off by a good part of such a unit, which the bound has no
room for (the first test).
"""
import pytest

torch = pytest.importorskip("torch")

import orth_ref  # noqa: E402

BF16 = torch.bfloat16
# by a CTA each, some with more than 64 on the smaller side, and by tiles
SHAPES = [(8, 8), (64, 7), (64, 64), (3, 64), (33, 50), (64, 200), (80, 83), (83, 70), (64, 1000), (60, 3000), (5000, 40)]


def matrix(shape, device):
    g = torch.Generator().manual_seed(shape[0])
    return (torch.randn(shape, generator=g) * 0.02).to(BF16).to(device)


def steps_of(g, halves):
    """orth_ref.emulated's steps, with `halves` for everything and every step."""
    a, b, c = orth_ref.USUAL
    x = g.double()
    x = x / (torch.sqrt((x * x).sum()) + 1e-7)
    flip = x.shape[0] > x.shape[1]
    x = x.t() if flip else x
    for _ in range(5):
        u = orth_ref.halves(x, halves)
        p = orth_ref.halves(orth_ref.product(u, (u[0].t(), u[1].t())), halves)
        q = orth_ref.halves(b * (p[0] + p[1]) + c * orth_ref.product(p, p), halves)
        x = a * (u[0] + u[1]) + orth_ref.product(q, u)
    return x.t() if flip else x


def bound(g):
    """(exact, tolerance of out)"""
    want = orth_ref.exact(g)
    most = 4 * max(float((f(g) - want).abs().max()) for f in (lambda t: steps_of(t, 2), orth_ref.single)) + 2.0 ** -18
    # half a unit in the last of 8 places, of the value that was rounded
    _, e = torch.frexp(want.abs() + most)
    return want, torch.ldexp(torch.ones_like(want), e - 9) + most


@pytest.mark.parametrize("shape", [(8, 8), (64, 64), (64, 1000), (80, 83)], ids=str)
def test_one_half_is_outside(shape):
    g = matrix(shape, "cpu")
    want, tol = bound(g)
    assert bool(((steps_of(g, 2).to(BF16).double() - want).abs() <= tol).all())
    for one in (steps_of(g, 1), orth_ref.emulated(g)):  # X in two halves but before the last two steps, and everything in one
        off = (one.to(BF16).double() - want).abs() > tol
        assert int(off.sum()) > 0.05 * off.numel()


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_two_halves(shape):
    from paper_2609_09020_gb300 import build, pic
    build.build()
    g = matrix(shape, "cuda")
    many = [g] + [matrix((s, 60), "cuda") for s in (7, 30, 50)]
    for tensors in ([g], many):
        out = [torch.zeros_like(t) for t in tensors]
        h = pic.Orthogonalizer(tensors, out=out)
        h.orthogonalize()
        h.check()
        h.close()
        for t, o in zip(tensors, out):
            want, tol = bound(t)
            off = (o.double() - want).abs() > tol
            assert not off.any(), f"{tuple(t.shape)}: {int(off.sum())} of {off.numel()}"
