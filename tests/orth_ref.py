"""Newton-Schulz products in fp64, and what the arithmetic that include/pic_orth.h
describes makes of them: shared by the tests of pic.Orthogonalizer.

Bounds.  The steps amplify what is rounded on the way by a factor that depends
on the matrix's singular values, so there is none in closed form that is of use.
The bound is four times the largest of what two evaluations of the same steps
are off by, plus the rounding of out:
  emulated   with the halves that X, A and b A + c A^2 are held in (of bfloat16 one,
             X in two but before the last two steps; small matrices have two),
             products and sums otherwise in fp64
  single     all in fp32 (for what sums in fp32 add; a kernel's are other sums
             of the same kind)
and 2^-18 of the largest singular value beside them, for matrices so small that
both happen to be exact.
"""
import torch

import linear_ref as ref

USUAL = (3.4445, -4.7750, 2.0315)
SCALE = 4096.0


def exact(g, steps=5, coefficients=USUAL, eps=1e-7):
    a, b, c = coefficients
    x = g.double()
    x = x / (torch.sqrt((x * x).sum()) + eps)
    flip = x.shape[0] > x.shape[1]
    x = x.t() if flip else x
    for _ in range(steps):
        p = x @ x.t()
        x = a * x + (b * p + c * (p @ p)) @ x
    return x.t() if flip else x


def halves(x, n):
    hi = (x * SCALE).half().double()
    lo = (x * SCALE - hi).half().double()
    return hi / SCALE, lo / SCALE if n == 2 else torch.zeros_like(lo)


def product(p, q):
    return p[0] @ q[0] + p[0] @ q[1] + p[1] @ q[0]


def emulated(g, steps=5, coefficients=USUAL, eps=1e-7):
    a, b, c = coefficients
    n = 1 if g.dtype == torch.bfloat16 else 2
    x = g.double()
    x = x / (torch.sqrt((x * x).sum()) + eps)
    flip = x.shape[0] > x.shape[1]
    x = x.t() if flip else x
    for k in range(steps):
        held = halves(x, 2 if n == 2 or steps - k >= 3 else 1)
        u = held if n == 2 else halves(x, 1)
        p = halves(product(u, (u[0].t(), u[1].t())), n)
        q = halves(b * (p[0] + p[1]) + c * product(p, p), n)
        x = a * (held[0] + held[1]) + product(q, u)
    return x.t() if flip else x


def single(g, steps=5, coefficients=USUAL, eps=1e-7):
    a, b, c = coefficients
    x = g.float()
    top = x.abs().max().clamp(min=1e-30)
    x = x / top  # (a norm in fp32's range)
    x = x / (torch.sqrt((x * x).sum()) + eps / top)
    flip = x.shape[0] > x.shape[1]
    x = x.t() if flip else x
    for _ in range(steps):
        p = x @ x.t()
        x = a * x + (b * p + c * (p @ p)) @ x
    return (x.t() if flip else x).double()


def check(got, g, steps=5, coefficients=USUAL, eps=1e-7, name=""):
    want = exact(g, steps, coefficients, eps)
    off = [f(g, steps, coefficients, eps) - want for f in (emulated, single)]
    t = g.dtype
    d = got.double() - want
    most = max(float(o.abs().max()) for o in off) * 4 + 2.0 ** -18
    ref.check(got, (want, most + ref.ROUND[t] * (want.abs() + most) + ref.TINY[t]), name)
    # and by their mean square, which a few elements that are off do not hide in
    mean = lambda v: float(v.square().mean().sqrt())
    bound = max(mean(o) for o in off) * 4 + ref.ROUND[t] * mean(want) + ref.TINY[t] + 2.0 ** -18 * mean(want)
    assert mean(d) <= bound, f"{name}: {mean(d)} > {bound}"
