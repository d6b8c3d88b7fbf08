"""Grouped layers whose weights, and gradients of them, have more than 2^31 elements."""
import pytest

torch = pytest.importorskip("torch")

import linear_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def pic():
    from paper_2609_09020_gb300 import build, pic
    build.build()
    return pic


# single rows, some, many (of the last group the elements beyond 2^31), on boundaries and off
@pytest.mark.parametrize("dtype,groups,side,offsets", [
    (BF16, 9, 16384, [0, 1, 1, 1, 2, 2, 3, 3, 3, 5]),
    (BF16, 9, 16384, [0, 100, 100, 100, 160, 160, 161, 161, 161, 290]),
    (BF16, 9, 16001, [0, 30, 30, 30, 60, 60, 61, 61, 61, 90]),
    (BF16, 600, 2048, [0] * 300 + [3] * 300 + [200]),
    (F32, 9, 16384, [0, 1, 1, 1, 2, 2, 3, 3, 3, 5]),
    (F32, 9, 16001, [0, 100, 100, 100, 160, 160, 161, 161, 161, 290]),
], ids=["bf16_single", "bf16_some", "bf16_odd", "bf16_many_groups", "fp32_single", "fp32_odd"])
def test_large_weights(pic, dtype, groups, side, offsets):
    assert groups * side * side > 2 ** 31 and len(offsets) == groups + 1
    gen = torch.Generator(device="cuda").manual_seed(0)
    normal = lambda s, std=1.0: torch.randn(s, generator=gen, device="cuda").mul_(std).to(dtype)
    rows, used = offsets[-1], [g for g in range(groups) if offsets[g + 1] > offsets[g]]
    w = torch.empty((groups, side, side), dtype=dtype, device="cuda")
    for g in used:
        w[g] = normal((side, side), side ** -0.5)
    for g in set(range(groups)) - set(used):
        w[g] = float("nan")  # of groups without rows
    x, dy, o = normal((rows, side)), normal((rows, side)), torch.tensor(offsets, device="cuda")
    y = pic.grouped_linear(x, w, o)
    dw = torch.full_like(w, 7.0)
    dx, _, db = pic.grouped_linear_backward(dy, x, w, o, dweight=dw)
    pic.grouped_linear_check()
    for g in used:
        at = slice(offsets[g], offsets[g + 1])
        for j in range(0, side, 4096):  # fp64 a part of the outputs at a time
            cols = slice(j, min(side, j + 4096))
            ref.check(y[at, cols], ref.forward(x[at], w[g, cols], None, "none", None)[0], f"y {g}")
            want = ref.backward(dy[at, cols], x[at], w[g, cols], None, "none")
            ref.check(dw[g, cols], want[1], f"dw {g}")
            ref.check(db[g, cols], want[2], f"db {g}")
            ref.check(dx[at, cols], ref.backward(dy[at], x[at, cols], w[g][:, cols], None, "none")[0], f"dx {g}")
    empty = torch.ones(groups, dtype=torch.bool, device="cuda")
    empty[used] = False
    assert not db[empty].any()
    for g in range(groups):
        if g not in used:
            assert not dw[g].any()
