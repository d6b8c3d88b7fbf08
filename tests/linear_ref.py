"""The linear layer and its gradient in fp64, with bounds of what rounding may
change: shared by the tests of pic.linear and pic.linear_backward.

Bounds (S = |x| |w|^T + |b|, the sum of the terms' sizes):
  product   a sum of K terms in fp32 in any order, with additions that may
            truncate: K + 32 times 2^-23 S (32: operands kept in fp32, or in
            pieces that carry 24 bits of them, and the bias)
  act       ReLU has slope <= 1, GELU <= 1.13; the function itself within 1e-6
  output    one rounding: half an ulp relative, half the smallest step absolute
  dz        rounded to the type; act' within 1e-6 |dy| beside it
"""
import math

import torch

ROUND = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}
SLOPE = 1.13
ACT_ERR = 1e-6


def act64(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "gelu":
        return z * torch.special.ndtr(z)
    return z


def act_grad64(z, act):
    if act == "relu":
        return (z > 0).double()
    if act == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    return torch.ones_like(z)


def forward(x, w, b, act, r):
    """((y, tolerance), (z, tolerance))"""
    t, K = x.dtype, x.shape[-1]
    x, w = x.double(), w.double()
    z, size = x @ w.t(), x.abs() @ w.abs().t()
    if b is not None:
        z, size = z + b.double(), size + b.double().abs()
    e = (K + 32) * 2.0 ** -23 * size
    y = act64(z, act)
    ey = e * SLOPE + (ACT_ERR if act == "gelu" else 0.0)
    if r is not None:
        y = y + r.double()
        ey = ey + 2.0 ** -24 * (y.abs() + ey)
    return ((y, ey + ROUND[t] * (y.abs() + ey) + TINY[t]), (z, e + ROUND[t] * (z.abs() + e) + TINY[t]))


def backward(dy, x, w, z, act):
    """(dx, tolerance), (dw, tolerance), (db, tolerance)"""
    t = dy.dtype
    M, N = dy.shape
    dy64, x, w = dy.double(), x.double(), w.double()
    dz = dy64 if act == "none" else dy64 * act_grad64(z.double(), act)
    e_act = ACT_ERR * dy64.abs() if act == "gelu" else torch.zeros_like(dz)
    e = e_act + (0.0 if act == "none" else ROUND[t] * (dz.abs() + e_act) + TINY[t])

    def out(v, size, terms, err):
        err = err + (terms + 32) * 2.0 ** -23 * size
        return v, err + ROUND[t] * (v.abs() + err) + TINY[t]

    big = dz.abs() + e
    dx = out(dz @ w, big @ w.abs(), N, e @ w.abs())
    dw = out(dz.t() @ x, big.t() @ x.abs(), M, e.t() @ x.abs())
    db = out(dz.sum(0), big.sum(0), M, e_act.sum(0))
    return dx, dw, db


def check(got, want, name=""):
    v, tol = want
    assert got.shape == v.shape, name
    d = (got.double() - v).abs()
    bad = ~(d <= tol)
    if bool(bad.any()):
        at = tuple(int(i) for i in torch.nonzero(bad)[0])
        raise AssertionError(f"{name}: {int(bad.sum())} of {bad.numel()} values off; first at {at}: "
                             f"{float(got[at])} != {float(v[at])} within {float(tol[at])}")
