"""Generates the polynomials behind the linear layer's GELU in fp32 and its
derivative (csrc/pic_gelu_grad.cuh; GELU before a rounding to 16 bits is
gen_gelu.py's).

GELU'(z) = Phi(z) + z phi(z).  With a = |z| and t(a) = Phi(-a) - a phi(a),

    GELU'(z) = t(a) for z < 0, 1 - t(a) else,
    t(a) = 2^(-a^2 log2(e) / 2) p(a),   p(a) = phi(0) (M(a) - a),

M(a) = Phi(-a) / phi(a) Mills' ratio, which is smooth: p is fitted by a
polynomial on 0 <= a <= A, A = 6, with the power as its weight (beyond A,
|t| < 4e-8 is taken as 0), of degree 9 for gradients that are rounded to 16
bits and of degree 11 for fp32, where the roundings of the evaluation are what
is left.  Lawson's reweighting turns the least-squares fit on Chebyshev nodes
into a minimax one.  The kernels take one 2^x, nine (eleven) multiply-adds and a
few operations more, against erfc and an exponential with their branches.

GELU itself in fp32 is max(z, 0) - g(a), g(a) = a Phi(-a) = 2^(...) r(a),
r(a) = phi(0) a M(a), fitted in the same way by a polynomial of degree 12
without a constant term.

Run:  python -m paper_2609_09020_gb300.gen_gelu_grad  (prints the header)
"""
from __future__ import annotations

import numpy as np
from numpy.polynomial import chebyshev, polynomial
from scipy.special import erfcx, ndtr

A = 6.0
DEG = 9
DEG_FP32 = 11
DEG_GELU = 12
PASSES = 200
HALF_LOG2E = -0.5 / np.log(2.0)


def _mills(a):
    return np.sqrt(np.pi / 2) * erfcx(a / np.sqrt(2))


def fit(deg=DEG):
    """Coefficients of p, lowest degree first."""
    return _fit(deg, lambda a: (_mills(a) - a) / np.sqrt(2 * np.pi))


def fit_gelu():
    """Coefficients of r, lowest degree first: a times those of phi(0) M(a), fitted with the weight a phi(a)."""
    return np.concatenate([[0.0], _fit(DEG_GELU - 1, lambda a: _mills(a) / np.sqrt(2 * np.pi), lambda a: a)])


def _fit(deg, func, more_weight=lambda a: np.ones_like(a)):
    a = 0.5 * A * (1 - np.cos(np.linspace(0, np.pi, 4001)))
    w = np.exp(-0.5 * a * a) * more_weight(a)
    f = func(a)
    v = chebyshev.chebvander(2 * a / A - 1, deg)
    lw = np.ones_like(a)
    for _ in range(PASSES):
        wt = w * np.sqrt(lw)
        c, *_ = np.linalg.lstsq(v * wt[:, None], f * wt, rcond=None)
        e = np.abs(w * (v @ c - f))
        lw *= e / e.max() + 1e-3
        lw /= lw.mean()
    p, power = np.zeros(1), np.ones(1)
    for k in chebyshev.cheb2poly(c):
        p = polynomial.polyadd(p, k * power)
        power = polynomial.polymul(power, [-1.0, 2 / A])
    return p


def grad_fp32(z, c):
    """fp32 emulation of the kernels' evaluation (the power correctly rounded)."""
    f32 = np.float32
    z = np.asarray(z, f32)
    a = np.minimum(np.abs(z), f32(A))
    p = np.full_like(a, f32(c[-1]))
    for k in c[-2::-1]:
        p = (a.astype(np.float64) * p + float(f32(k))).astype(f32)
    e = np.exp2(((a * a).astype(f32) * f32(HALF_LOG2E)).astype(f32).astype(np.float64)).astype(f32)
    t = (e * p).astype(f32)
    return np.where(z <= f32(-A), f32(0), np.where(z < 0, t, f32(1) - t))


def gelu_fp32(z, c):
    """The same of GELU."""
    f32 = np.float32
    z = np.asarray(z, f32)
    a = np.minimum(np.abs(z), f32(A))
    p = np.full_like(a, f32(c[-1]))
    for k in c[-2::-1]:
        p = (a.astype(np.float64) * p + float(f32(k))).astype(f32)
    e = np.exp2(((a * a).astype(f32) * f32(HALF_LOG2E)).astype(f32).astype(np.float64)).astype(f32)
    g = np.where(a >= f32(A), f32(0), p)
    return (np.maximum(z, f32(0)).astype(np.float64) - e.astype(np.float64) * g).astype(f32)


def max_error_gelu(c) -> float:
    z = np.linspace(-12, 12, 1_200_001)
    return float(np.max(np.abs(gelu_fp32(z, c).astype(np.float64) - z.astype(np.float32) * ndtr(z.astype(np.float32).astype(np.float64)))))


def max_error(c) -> float:
    z = np.linspace(-12, 12, 1_200_001)
    ref = ndtr(z) + z * np.exp(-0.5 * z * z) / np.sqrt(2 * np.pi)
    return float(np.max(np.abs(grad_fp32(z, c).astype(np.float64) - ref)))


def header(c, c32, gelu) -> str:
    lines = ["// Generated by paper_2609_09020_gb300/gen_gelu_grad.py -- do not edit.",
             f"// Phi(-a) - a phi(a) ~= 2^(kGeluGradPower a^2) p(a) on 0 <= a <= {A:g}; max error of GELU' in",
             f"// fp32 ~ {max_error(c):.1e} (degree {DEG}), {max_error(c32):.1e} (degree {DEG_FP32}).",
             f"// a Phi(-a) ~= 2^(kGeluGradPower a^2) r(a); max error of GELU on |z| < 12, the rounding of the",
             f"// result included, ~ {max_error_gelu(gelu):.1e}.",
             "#pragma once", "", "namespace pic {", "",
             f"constexpr float kGeluGradA = {float(np.float32(A))!r}f;",
             f"constexpr float kGeluGradPower = {float(np.float32(HALF_LOG2E))!r}f;",
             f"constexpr int kGeluGradDeg = {DEG};", f"constexpr int kGeluGradDeg32 = {DEG_FP32};",
             f"constexpr int kGeluDeg32 = {DEG_GELU};", "",
             "// Coefficients of p and of r, highest degree first (Horner order)."]
    for name, k in (("gelu_grad_c", c), ("gelu_grad_c32", c32), ("gelu_c32", gelu)):
        lines += [f"__host__ __device__ constexpr float {name}(int i) {{", "  constexpr float c[] = {"]
        lines += [f"      {float(np.float32(v))!r}f," for v in k[::-1]]
        lines += ["  };", "  return c[i];", "}"]
    return "\n".join(lines + ["", "}  // namespace pic", ""])


if __name__ == "__main__":
    print(header(fit(), fit(DEG_FP32), fit_gelu()), end="")
