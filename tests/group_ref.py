"""Grouped linear layers in fp64, group by group, with linear_ref's bounds."""
import torch

import linear_ref as ref


def spans(offsets):
    return [(g, i, j) for g, (i, j) in enumerate(zip(offsets, offsets[1:]))]


def forward(x, w, b, offsets, act):
    """((y, tolerance), (z, tolerance)) with NaN in the rows of no group"""
    M, N = x.shape[0], w.shape[1]
    new = lambda: torch.full((M, N), float("nan"), dtype=torch.float64, device=x.device)
    y, ey, z, ez = new(), new(), new(), new()
    for g, i, j in spans(offsets):
        if j > i:
            (y[i:j], ey[i:j]), (z[i:j], ez[i:j]) = ref.forward(x[i:j], w[g], None if b is None else b[g], act, None)
    return (y, ey), (z, ez)


def backward(dy, x, w, z, offsets, act):
    """(dx, tolerance), (dw, tolerance), (db, tolerance)"""
    G, N, K = w.shape
    new = lambda shape, v: torch.full(shape, v, dtype=torch.float64, device=dy.device)
    nan = float("nan")
    dx, ex = new((dy.shape[0], K), nan), new((dy.shape[0], K), nan)
    dw, ew, db, eb = new((G, N, K), 0.0), new((G, N, K), 0.0), new((G, N), 0.0), new((G, N), 0.0)
    for g, i, j in spans(offsets):
        if j > i:
            (dx[i:j], ex[i:j]), (dw[g], ew[g]), (db[g], eb[g]) = ref.backward(
                dy[i:j], x[i:j], w[g], None if z is None else z[i:j], act)
    return (dx, ex), (dw, ew), (db, eb)


def check_rows(got, want, offsets, kept, name):
    """The rows of groups against (value, tolerance), the others as they were."""
    first, last = offsets[0], offsets[-1]
    ref.check(got[first:last], (want[0][first:last], want[1][first:last]), name)
    assert torch.equal(got[:first], kept[:first]) and torch.equal(got[last:], kept[last:]), name
