"""Grouped layers whose sums are longer than one accumulator of the tensor cores takes
(16384): inputs in the forward, outputs in dx.  Bounds as in linear_ref."""
import pytest

torch = pytest.importorskip("torch")

import group_ref  # noqa: E402
import linear_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def pic():
    from paper_2609_09020_gb300 import build, pic
    build.build()
    return pic


def normal(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


# rows and groups: tiles, turned tiles, single rows
SPREADS = [[1, 1, 100, 290], [0, 30, 61, 61, 70], [0, 1, 1, 3]]


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=str)
@pytest.mark.parametrize("deep", [16384, 16385, 16392, 20000, 40001])
@pytest.mark.parametrize("offsets", SPREADS, ids=str)
def test_deep_sums(pic, offsets, deep, dtype):
    rows, groups, wide = offsets[-1] + 2, len(offsets) - 1, 72
    o = torch.tensor(offsets, device="cuda")
    x, b = normal((rows, deep), dtype, 1), normal((groups, wide), dtype, 2)
    w = normal((groups, wide, deep), dtype, 3, deep ** -0.5)
    out = normal((rows, wide), dtype, 4)
    kept = out.clone()
    y, z = pic.grouped_linear(x, w, o, b, act="gelu", out=out, save_pre=True)
    wy, wz = group_ref.forward(x, w, b, offsets, "gelu")
    group_ref.check_rows(y, wy, offsets, kept, "y")
    at = slice(offsets[0], offsets[-1])
    ref.check(z[at], (wz[0][at], wz[1][at]), "z")
    del x, w
    # the same length over the outputs
    dy, pre, x = normal((rows, deep), dtype, 5), normal((rows, deep), dtype, 6), normal((rows, wide), dtype, 7)
    w = normal((groups, deep, wide), dtype, 8, deep ** -0.5)
    dx = normal((rows, wide), dtype, 9)
    kept = dx.clone()
    _, dw, db = pic.grouped_linear_backward(dy, x, w, o, act="relu", pre=pre, dx=dx)
    wx, ww, wb = group_ref.backward(dy, x, w, pre, offsets, "relu")
    group_ref.check_rows(dx, wx, offsets, kept, "dx")
    ref.check(dw, ww, "dw")
    ref.check(db, wb, "db")
    pic.grouped_linear_check()


@pytest.mark.parametrize("dtype", [F16, BF16], ids=str)
def test_deep_rows_keep_to_their_groups(pic, dtype):
    offsets, deep, wide = [0, 40, 90, 130], 16400, 40
    o = torch.tensor(offsets, device="cuda")
    x, w = normal((130, deep), dtype, 1), normal((3, wide, deep), dtype, 2, deep ** -0.5)
    want = pic.grouped_linear(x, w, o)
    x[40:90], w[1] = float("nan"), float("inf")
    got = pic.grouped_linear(x, w, o)
    assert torch.equal(got[:40], want[:40]) and torch.equal(got[90:], want[90:])
    assert bool(got[40:90].isnan().all())
    pic.grouped_linear_check()
