"""pic.grouped_linear and pic.grouped_linear_backward against the definition in
fp64, within linear_ref's bounds."""
import random

import pytest
import torch

import group_ref
import linear_ref as ref

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
TYPES = [F32, F16, BF16]


@pytest.fixture(scope="module")
def pic():
    from paper_2609_09020_gb300 import build, pic
    build.build()
    return pic


def normal(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def offsets_tensor(offsets):
    return torch.tensor(offsets, dtype=torch.int64, device="cuda")


def case(rows, groups, inp, outp, dtype, seed, bias=True):
    x = normal((rows, inp), dtype, seed)
    w = normal((groups, outp, inp), dtype, seed + 1, inp ** -0.5)
    b = normal((groups, outp), dtype, seed + 2, 0.3) if bias else None
    return x, w, b


def check_forward(pic, offsets, rows, inp, outp, dtype, act, seed=0, bias=True):
    x, w, b = case(rows, len(offsets) - 1, inp, outp, dtype, seed, bias)
    out = normal((rows, outp), dtype, seed + 3)
    kept = out.clone()
    y, z = pic.grouped_linear(x, w, offsets_tensor(offsets), b, act=act, out=out, save_pre=True)
    assert y is out
    pic.grouped_linear_check()
    wy, wz = group_ref.forward(x, w, b, offsets, act)
    group_ref.check_rows(y, wy, offsets, kept, "y")
    ref.check(z[offsets[0]:offsets[-1]], tuple(t[offsets[0]:offsets[-1]] for t in wz), "z")


def check_backward(pic, offsets, rows, inp, outp, dtype, act, seed=0):
    x, w, _ = case(rows, len(offsets) - 1, inp, outp, dtype, seed)
    dy, z = normal((rows, outp), dtype, seed + 4), normal((rows, outp), dtype, seed + 5, 1.4)
    dx = normal((rows, inp), dtype, seed + 6)
    kept = dx.clone()
    got, dw, db = pic.grouped_linear_backward(dy, x, w, offsets_tensor(offsets), act=act,
                                              pre=None if act == "none" else z, dx=dx)
    assert got is dx
    pic.grouped_linear_check()
    wx, ww, wb = group_ref.backward(dy, x, w, z, offsets, act)
    group_ref.check_rows(dx, wx, offsets, kept, "dx")
    ref.check(dw, ww, "dw")
    ref.check(db, wb, "db")


# rows of the groups, and around them: none, single ones, ends inside and on tiles
SPREADS = [
    (1, [0, 1]),
    (5, [0, 0, 5]),
    (130, [0, 128, 130]),
    (64, [0, 0, 0, 64, 64]),
    (300, [7, 7, 8, 9, 73, 137, 265, 265, 290]),
    (40, [40, 40]),
    (500, [0, 255, 256, 256, 499, 500]),
    (700, [100, 356, 612]),
    (129, [0, 1, 2, 3, 5, 8, 13, 21, 34, 55, 89, 129]),
]
SHAPES = [(1, 1), (3, 5), (64, 64), (40, 24), (7, 64), (128, 3), (200, 136), (72, 300), (513, 129)]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,offsets", SPREADS, ids=str)
def test_forward_spreads(pic, rows, offsets, dtype):
    for i, (inp, outp) in enumerate([(40, 24), (64, 64), (264, 200)]):
        check_forward(pic, offsets, rows, inp, outp, dtype, ["gelu", "relu", "none"][i], seed=i)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,offsets", SPREADS, ids=str)
def test_backward_spreads(pic, rows, offsets, dtype):
    for i, (inp, outp) in enumerate([(40, 24), (64, 64), (264, 200)]):
        check_backward(pic, offsets, rows, inp, outp, dtype, ["gelu", "relu", "none"][i], seed=i)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("act", ["none", "relu", "gelu"])
@pytest.mark.parametrize("inp,outp", SHAPES, ids=str)
def test_shapes(pic, inp, outp, act, dtype):
    check_forward(pic, [0, 70, 70, 199], 199, inp, outp, dtype, act, seed=inp)
    check_forward(pic, [0, 2, 3, 5], 5, inp, outp, dtype, act, seed=outp, bias=False)
    check_backward(pic, [0, 70, 70, 199], 199, inp, outp, dtype, act, seed=inp)
    check_backward(pic, [0, 2, 3, 5], 5, inp, outp, dtype, act, seed=outp)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_many_groups(pic, dtype):
    rng = random.Random(3)
    offsets = [0]
    for _ in range(1024):
        offsets.append(offsets[-1] + rng.choice([0, 0, 1, 2, 7, 40]))
    check_forward(pic, offsets, offsets[-1], 24, 40, dtype, "gelu")
    check_backward(pic, offsets, offsets[-1], 24, 40, dtype, "gelu")
    offsets = offsets[:301]
    check_forward(pic, offsets, offsets[-1], 136, 264, dtype, "relu")
    check_backward(pic, offsets, offsets[-1], 136, 264, dtype, "relu")


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("inp,outp", [(64, 64), (16, 48), (3, 17), (256, 160)], ids=str)
def test_long_groups(pic, inp, outp, dtype):
    """Many tiles of a group, sums over many rows."""
    offsets = [0, 20000, 20001, 41111, 41111, 60000]
    check_forward(pic, offsets, 60000, inp, outp, dtype, "relu")
    check_backward(pic, offsets, 60000, inp, outp, dtype, "relu")


@pytest.mark.parametrize("dtype", [F16, BF16], ids=str)
def test_large(pic, dtype):
    offsets = [0, 700, 700, 1500, 1629, 2600]
    check_forward(pic, offsets, 2600, 1024, 1152, dtype, "gelu")
    check_backward(pic, offsets, 2600, 1024, 1152, dtype, "gelu")


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_few_rows_of_wide_layers(pic, dtype):
    rng = random.Random(5)
    offsets = [0]
    for _ in range(24):
        offsets.append(offsets[-1] + rng.choice([0, 0, 1, 2, 5]))
    check_forward(pic, offsets, offsets[-1], 1000, 1544, dtype, "none")
    check_forward(pic, offsets, offsets[-1], 2048, 520, dtype, "gelu", seed=1)
    check_backward(pic, offsets, offsets[-1], 1000, 1544, dtype, "gelu", seed=2)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("inp,outp,pad", [(64, 64, 3), (40, 24, 8), (200, 136, 1), (264, 520, 8)], ids=str)
def test_strides(pic, inp, outp, pad, dtype):
    """Slices of wider tensors, at all alignments, weights in one buffer with the biases."""
    offsets, rows, G = [3, 90, 90, 210, 400], 410, 4
    at = pad // 2
    wide = lambda cols, seed: normal((rows, cols + pad), dtype, seed)[:, at:at + cols]
    x, dy, z = wide(inp, 0), wide(outp, 1), wide(outp, 2)
    blob = normal((G, outp * (inp + pad) + outp + pad), dtype, 3, inp ** -0.5)
    w = blob[:, pad:pad + outp * (inp + pad)].unflatten(1, (outp, inp + pad))[:, :, :inp]
    b = blob[:, outp * (inp + pad) + pad:]
    o = offsets_tensor(offsets)
    y = torch.zeros((rows, outp + pad), dtype=dtype, device="cuda")
    got, pre = pic.grouped_linear(x, w, o, b, act="gelu", out=y[:, at:at + outp], save_pre=True)
    wy, wz = group_ref.forward(x, w, b, offsets, "gelu")
    group_ref.check_rows(got, wy, offsets, torch.zeros_like(got), "y")
    ref.check(pre[3:400], tuple(t[3:400] for t in wz), "z")
    assert not y[:, :at].any() and not y[:, at + outp:].any()
    dx = torch.zeros((rows, inp + pad), dtype=dtype, device="cuda")
    grad = torch.zeros_like(blob)
    gw = grad[:, pad:pad + outp * (inp + pad)].unflatten(1, (outp, inp + pad))[:, :, :inp]
    gb = grad[:, outp * (inp + pad) + pad:]
    gx, _, _ = pic.grouped_linear_backward(dy, x, w, o, act="gelu", pre=z, dx=dx[:, at:at + inp], dweight=gw, dbias=gb)
    wx, ww, wb = group_ref.backward(dy, x, w, z, offsets, "gelu")
    group_ref.check_rows(gx, wx, offsets, torch.zeros_like(gx), "dx")
    ref.check(gw, ww, "dw")
    ref.check(gb, wb, "db")
    assert not dx[:, :at].any() and not dx[:, at + inp:].any() and not grad[:, :pad].any()
    gaps = grad[:, pad:pad + outp * (inp + pad)].unflatten(1, (outp, inp + pad))[:, :, inp:]
    assert not gaps.any()
    pic.grouped_linear_check()


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("inp,outp", [(64, 64), (24, 40), (264, 200)], ids=str)
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_groups_keep_to_themselves(pic, bad, inp, outp, dtype):
    """Rows, weights and biases that are not finite reach nothing of another group, nor
    do rows of no group."""
    offsets, rows = [2, 37, 100, 100, 235], 240
    x, w, b = case(rows, 4, inp, outp, dtype, 0)
    dy, z = normal((rows, outp), dtype, 4), normal((rows, outp), dtype, 5)
    for t in (x, dy, z):
        t[:2] = bad
        t[37:100] = bad
        t[235:] = bad
    w[1], w[2], b[1], b[2] = bad, bad, bad, bad
    o = offsets_tensor(offsets)
    y, pre = pic.grouped_linear(x, w, o, b, act="relu", save_pre=True)
    dx, dw, db = pic.grouped_linear_backward(dy, x, w, o, act="gelu", pre=z)
    wy, wz = group_ref.forward(x, w, b, offsets, "relu")
    wx, ww, wb = group_ref.backward(dy, x, w, z, offsets, "gelu")
    for i, j in ((2, 37), (100, 235)):
        for got, want, name in ((y, wy, "y"), (pre, wz, "z"), (dx, wx, "dx")):
            ref.check(got[i:j], (want[0][i:j], want[1][i:j]), name)
    for g in (0, 3):
        ref.check(dw[g], (ww[0][g], ww[1][g]), "dw")
        ref.check(db[g], (wb[0][g], wb[1][g]), "db")
    assert not dw[2].any() and not db[2].any()
    assert not torch.isfinite(dw[1]).any() and not torch.isfinite(db[1]).any()
    if bad != bad:
        assert bool(y[37:100].isnan().all()) and bool(dx[37:100].isnan().all())


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("inp,outp", [(64, 64), (264, 200)], ids=str)
def test_infinite_values_as_the_formula_has_them(pic, inp, outp, dtype):
    """One infinity in x: its column of weights decides the sign, and no NaN comes of it."""
    offsets = [0, 60, 150]
    x, w, b = case(150, 2, inp, outp, dtype, 0)
    x[10, 5] = float("inf")
    x[149, inp - 1] = float("-inf")
    y = pic.grouped_linear(x, w, offsets_tensor(offsets), b)
    for row, k, g in ((10, 5, 0), (149, inp - 1, 1)):
        want = torch.sign(w[g][:, k].float()) * x[row, k].float()
        want = torch.where(w[g][:, k] == 0, torch.full_like(want, float("nan")), want)
        assert torch.equal(y[row].float().nan_to_num(7.0), want.nan_to_num(7.0))
    finite = torch.ones(150, dtype=torch.bool, device="cuda")
    finite[10] = finite[149] = False
    wy, _ = group_ref.forward(x, w, b, offsets, "none")
    ref.check(y[finite], (wy[0][finite], wy[1][finite]), "y")


def test_bad_offsets_are_held_and_reported(pic):
    """Offsets that decrease or leave [0, rows] count as the largest so far, at most rows."""
    x, w, b = case(100, 5, 40, 24, F32, 0)
    wide, ww, wb = case(100, 5, 264, 200, F16, 1)
    for offsets, held in (([0, 50, 20, 60, 300, 100], [0, 50, 50, 60, 100, 100]),
                          ([-5, 10, 10, 2 ** 40, 3, 99], [0, 10, 10, 100, 100, 100]),
                          ([100, 0, 0, 0, 0, 50], [100] * 6)):
        o, h = offsets_tensor(offsets), offsets_tensor(held)
        for a in ((x, w, b), (wide, ww, wb)):
            out, same = (torch.zeros((100, a[1].shape[1]), dtype=a[0].dtype, device="cuda") for _ in range(2))
            pic.grouped_linear(a[0], a[1], h, a[2], out=same)
            pic.grouped_linear_check()
            pic.grouped_linear(a[0], a[1], o, a[2], out=out)
            with pytest.raises(pic.PicError):
                pic.grouped_linear_check()
            pic.grouped_linear_check()
            assert torch.equal(out, same)
            dy = normal((100, a[1].shape[1]), a[0].dtype, 9)
            _, gw, gb = pic.grouped_linear_backward(dy, a[0], a[1], o, need=("weight", "bias"))
            with pytest.raises(pic.PicError):
                pic.grouped_linear_check()
            _, hw, hb = pic.grouped_linear_backward(dy, a[0], a[1], h, need=("weight", "bias"))
            assert torch.equal(gw, hw) and torch.equal(gb, hb)
    pic.grouped_linear_check()


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("need", [("x",), ("weight",), ("bias",), ("x", "bias"), ("weight", "bias")], ids=str)
def test_parts_of_the_gradient(pic, need, dtype):
    offsets = offsets_tensor([0, 100, 150])
    for inp, outp in ((40, 64), (264, 200)):
        x, w, _ = case(150, 2, inp, outp, dtype, 0)
        dy, z = normal((150, outp), dtype, 4), normal((150, outp), dtype, 5)
        all_of = dict(zip(("x", "weight", "bias"), pic.grouped_linear_backward(dy, x, w, offsets, act="gelu", pre=z)))
        some = dict(zip(("x", "weight", "bias"),
                        pic.grouped_linear_backward(dy, x, w, offsets, act="gelu", pre=z, need=need)))
        for k in all_of:
            assert (some[k] is None) == (k not in need)
            if k in need:
                assert torch.equal(some[k], all_of[k]), k


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("inp,outp,rows", [(64, 64, 5000), (264, 200, 900), (520, 264, 30)], ids=str)
def test_again_and_captured(pic, inp, outp, rows, dtype):
    """The same from call to call, on another stream, and in a graph that is replayed with other offsets."""
    offsets = [0, rows // 3, rows // 3, rows - 7, rows]
    x, w, b = case(rows, 4, inp, outp, dtype, 0)
    dy = normal((rows, outp), dtype, 4)
    o = offsets_tensor(offsets)

    def step():
        y, z = pic.grouped_linear(x, w, o, b, act="gelu", save_pre=True)
        return (y, z) + pic.grouped_linear_backward(dy, x, w, o, act="gelu", pre=z)

    first, again = step(), step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y = pic.grouped_linear(x, w, o, b, act="gelu", stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for a, c in zip(first, again):
        assert torch.equal(a, c)
    assert torch.equal(y, first[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for new in (offsets, [0, 1, rows // 2, rows // 2, rows]):
        o.copy_(offsets_tensor(new))
        graph.replay()
        torch.cuda.synchronize()
        for a, c in zip(held, step()):
            assert torch.equal(a, c)
    pic.grouped_linear_check()


def test_gradient_against_differences(pic):
    """The gradient of sum(y r) in fp32, against central differences of the call itself."""
    offsets = [0, 9, 9, 30]
    x, w, b = case(30, 3, 12, 10, F32, 0)
    o, r = offsets_tensor(offsets), normal((30, 10), F32, 8)
    value = lambda: float((pic.grouped_linear(x, w, o, b, act="gelu").double() * r.double()).sum())
    _, z = pic.grouped_linear(x, w, o, b, act="gelu", save_pre=True)
    grads = pic.grouped_linear_backward(r, x, w, o, act="gelu", pre=z)
    # h^2 of the third derivative (GELU's is below 1.6, at most 12 of |r| <= 4 terms): 1e-3;
    # roundings of 300 outputs of size <= 10, 300 * 10 * 2^-23 / (2 h): 1.8e-2
    h = 1e-2
    rng = random.Random(1)
    for t, g in zip((x, w, b), grads):
        for _ in range(12):
            at = tuple(rng.randrange(n) for n in t.shape)
            old = float(t[at])
            t[at] = old + h
            up, high = float(t[at]), value()
            t[at] = old - h
            down, low = float(t[at]), value()
            t[at] = old
            assert abs((high - low) / (up - down) - float(g[at])) <= 2e-2


def test_empty_calls(pic):
    x, w, b = case(0, 3, 40, 24, F16, 0)
    o = offsets_tensor([0, 0, 0, 0])
    assert pic.grouped_linear(x, w, o, b).shape == (0, 24)
    dx, dw, db = pic.grouped_linear_backward(torch.empty((0, 24), dtype=F16, device="cuda"), x, w, o)
    assert dx.shape == (0, 40) and not dw.any() and not db.any()
    pic.grouped_linear_check()


def test_rows_past_32_bits(pic):
    """Row offsets in bytes and elements past 2^32: the last group of a tall x."""
    rows = 2 ** 25 + 77
    x = torch.zeros((rows, 136), dtype=BF16, device="cuda")
    offsets = [2 ** 25 - 3, 2 ** 25 + 5, rows]
    tail = normal((80, 136), BF16, 0)
    x[2 ** 25 - 3:] = tail
    w, dy = normal((2, 24, 136), BF16, 1, 0.1), torch.zeros((rows, 24), dtype=BF16, device="cuda")
    dy[2 ** 25 - 3:] = normal((80, 24), BF16, 2)
    o, small = offsets_tensor(offsets), [0, 8, 80]
    y = pic.grouped_linear(x, w, o)
    wy, _ = group_ref.forward(tail, w, None, small, "none")
    ref.check(y[2 ** 25 - 3:], wy, "y")
    dx, dw, db = pic.grouped_linear_backward(dy, x, w, o)
    wx, ww, wb = group_ref.backward(dy[2 ** 25 - 3:], tail, w, None, small, "none")
    ref.check(dx[2 ** 25 - 3:], wx, "dx")
    ref.check(dw, ww, "dw")
    ref.check(db, wb, "db")
    pic.grouped_linear_check()


@pytest.mark.parametrize("inp,outp", [(512, 384), (1000, 130), (136, 640)], ids=str)
def test_large_fp32(pic, inp, outp):
    """fp32 layers large enough for the tensor cores: against the definition, and sums of 512
    and more about as good as fp32 FMAs in order (6.2e-7 of 1024), not worse than 1.5e-6."""
    offsets = [3, 700, 700, 1500, 1629, 2600, 2601]
    check_forward(pic, offsets, 2610, inp, outp, F32, "gelu")
    check_backward(pic, offsets, 2610, inp, outp, F32, "gelu")
    x, w, b = case(2610, 6, inp, outp, F32, 7, bias=False)
    y = pic.grouped_linear(x, w, offsets_tensor(offsets))
    dx, dw, _ = pic.grouped_linear_backward(y, x, w, offsets_tensor(offsets))
    for g, i, j in group_ref.spans(offsets):
        if j - i > 128:
            for got, want in ((y[i:j], x[i:j].double() @ w[g].double().t()), (dx[i:j], y[i:j].double() @ w[g].double()),
                              (dw[g], y[i:j].double().t() @ x[i:j].double())):
                d = (got.double() - want).square().mean().sqrt() / want.square().mean().sqrt()
                assert float(d) <= 1.5e-6


def test_large_fp32_not_finite(pic):
    """In large fp32 layers too, rows that are not finite stay in their group, and an infinity
    or a value that its first piece would round to one is as the formula has it."""
    offsets, rows = [0, 300, 301, 701, 1100], 1100
    x, w, _ = case(rows, 4, 520, 392, F32, 0, bias=False)
    x[300:301], x[701:705], w[3, 17, 5] = float("nan"), float("inf"), float("nan")
    x[10, 100], x[450, 7] = 3.4e38, float("-inf")
    o = offsets_tensor(offsets)
    y = pic.grouped_linear(x, w, o)
    dy = normal((rows, 392), F32, 4)
    dx, dw, db = pic.grouped_linear_backward(dy, x, w, o)
    pic.grouped_linear_check()
    finite = torch.isfinite(x).all(1)
    wy, _ = group_ref.forward(x, w, None, offsets, "none")
    ok = finite.clone()
    ok[701:] = False
    ok[10] = False  # beside fp32's range in places
    ref.check(y[ok], (wy[0][ok], wy[1][ok]), "y")
    assert bool(y[300].isnan().all()) and bool(y[701:, 17].isnan().all())
    others = [c for c in range(392) if c != 17]
    assert torch.isfinite(y[705:][:, others]).all()
    assert torch.equal(y[450].sign(), -w[2, :, 7].sign()) and torch.isinf(y[450]).all()
    near = wy[0][10].abs() < 3e38
    ref.check(y[10][near], (wy[0][10][near], wy[1][10][near]), "y")
    wx, ww, wb = group_ref.backward(dy, x, w, None, offsets, "none")
    ref.check(dx[:701], (wx[0][:701], wx[1][:701]), "dx")
    bad = [c for c in range(520) if c != 5]
    ref.check(dx[701:][:, bad], (wx[0][701:][:, bad], wx[1][701:][:, bad]), "dx")
    assert bool(dx[701:, 5].isnan().all())
    most = [c for c in range(520) if c != 100]
    ref.check(dw[0][:, most], (ww[0][0][:, most], ww[1][0][:, most]), "dw")
    ref.check(db, wb, "db")
    assert bool(dw[1].isnan().all()) and not torch.isfinite(dw[3]).any()
    most = [c for c in range(520) if c != 7]
    ref.check(dw[2][:, most], (ww[0][2][:, most], ww[1][2][:, most]), "dw")
    assert torch.isinf(dw[2][:, 7]).all()


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("inp,outp", [(64, 64), (40, 24), (7, 64), (128, 96), (64, 3)], ids=str)
def test_narrow_gradients(pic, inp, outp, dtype):
    """Narrow layers over many rows: groups of one row, of none, that end on and off tiles, more groups than
    CTAs, fewer tiles than CTAs, and one group of all."""
    rng = random.Random(inp)
    many = [5]
    for _ in range(700):
        many.append(many[-1] + rng.choice([0, 1, 2, 3, 40, 127, 128, 129]))
    for offsets in ([0, 1, 1, 2, 130, 1153, 2000, 2001], [0, 0, 1024, 1024], [0, 30000], many, [3, 900, 1500]):
        rows = offsets[-1] + 4
        check_backward(pic, offsets, rows, inp, outp, dtype, "gelu", seed=outp)
    check_backward(pic, [0, 700, 1800], 1900, inp, outp, dtype, "none")


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_narrow_groups_keep_to_themselves(pic, bad, dtype):
    """As test_groups_keep_to_themselves, over enough rows for the one-pass gradient."""
    offsets, rows = [2, 537, 1100, 1100, 2235], 2240
    for inp, outp in ((64, 64), (24, 40), (128, 72)):
        x, w, b = case(rows, 4, inp, outp, dtype, 0)
        dy, z = normal((rows, outp), dtype, 4), normal((rows, outp), dtype, 5)
        for t in (x, dy, z):
            t[:2] = bad
            t[537:1100] = bad
            t[2235:] = bad
        w[1], w[2] = bad, bad
        for act in ("gelu", "none"):
            dx, dw, db = pic.grouped_linear_backward(dy, x, w, offsets_tensor(offsets), act=act, pre=z)
            wx, ww, wb = group_ref.backward(dy, x, w, z, offsets, act)
            for i, j in ((2, 537), (1100, 2235)):
                ref.check(dx[i:j], (wx[0][i:j], wx[1][i:j]), "dx")
            for g in (0, 3):
                ref.check(dw[g], (ww[0][g], ww[1][g]), "dw")
                ref.check(db[g], (wb[0][g], wb[1][g]), "db")
            assert not dw[2].any() and not db[2].any()
            assert not torch.isfinite(dw[1]).any() and not torch.isfinite(db[1]).any()
        pic.grouped_linear_check()


@pytest.mark.parametrize("dtype", [F16, BF16], ids=str)
@pytest.mark.parametrize("last", [1, 28, 70])
def test_rows_at_the_end_of_an_allocation(pic, dtype, last):
    """x and dy end where the allocator's segments of memory do, with a small group's rows."""
    rows, inp, outp = 500, 232, 376
    offsets = [0, 200, rows - last, rows]

    def at_end(cols, seed):
        held = torch.empty(6 << 20, dtype=dtype, device="cuda")  # 12 MB: a segment of its own
        t = held[held.numel() - rows * cols:].view(rows, cols)
        return t.copy_(normal((rows, cols), dtype, seed))

    x, dy, w = at_end(inp, 1), at_end(outp, 2), normal((3, outp, inp), dtype, 3, inp ** -0.5)
    _, dw, db = pic.grouped_linear_backward(dy, x, w, offsets_tensor(offsets), need=("weight", "bias"))
    pic.grouped_linear_check()
    _, ww, wb = group_ref.backward(dy, x, w, None, offsets, "none")
    ref.check(dw, ww, "dw")
    ref.check(db, wb, "db")
