"""Gradients whose norm is above fp32's largest value, though each of them is finite:
the norm that is returned is infinite, the clipped gradients are what the formula gives;
and max_norm = infinity, with which nothing is clipped whatever the norm is."""
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_09020_gb300 import build
    build.build()


@pytest.mark.parametrize("max_norm", [1e30, 2.5, 1e-3])
@pytest.mark.parametrize("n", [4, 3000, 70001])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
def test_norm_above_fp32(dtype, n, max_norm):
    """coef is below 2^-98 here, from 2^-126 on in fewer bits: steps of 2^-149, half of
    one of which is 2^-149 |g| in an output; else three roundings and the norm's."""
    from paper_2609_09020_gb300 import pic
    g = torch.linspace(2.0e38, 3.3e38, n, device="cuda").to(dtype)
    g[1::2] *= -1
    small = torch.full((100,), 1.0, device="cuda")
    out, out_small = torch.empty_like(g), torch.empty_like(small)
    clip = pic.GradClip([g, small], out=[out, out_small])
    norm = clip.clip(max_norm)
    clip.check()
    assert float(norm) == math.inf
    want = g.double() * (max_norm / math.sqrt(float((g.double() ** 2).sum())))
    rounding = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    tolerance = want.abs() * (rounding + 2.0 ** -18) + g.double().abs() * 2.0 ** -149
    assert bool(((out.double() - want).abs() <= tolerance).all())
    assert bool((out != 0).all()) and not bool(out_small.isnan().any())


@pytest.mark.parametrize("bad", [math.inf, math.nan, None])
def test_infinite_max_norm(bad):
    from paper_2609_09020_gb300 import pic
    g = torch.linspace(-3.0, 3.0, 5000, device="cuda")
    if bad is not None:
        g[1234] = bad
    out = torch.empty_like(g)
    norm = pic.GradClip([g], out=[out]).clip(math.inf)
    assert torch.equal(out.nan_to_num(nan=7.0), g.nan_to_num(nan=7.0))
    assert float(norm) == math.inf if bad == math.inf else bad is None or math.isnan(float(norm))
