"""A pre-activation that is NaN in the gradient: the derivative of ReLU is 1 where z > 0
and 0 elsewhere, at NaN too, so nothing of it is passed on (dy may be anything there);
that of GELU is NaN and reaches its row of dx, its rows of dw and db, and nothing else."""
import math

import pytest

torch = pytest.importorskip("torch")

import linear_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_09020_gb300 import build
    build.build()


def normal(shape, dtype, seed, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").mul_(std).to(dtype)


# few rows, an elementwise pass and products (of few columns and many), the narrow kernel's ways of loading
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16], ids=["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("M,K,N", [(1, 64, 64), (4, 300, 200), (12, 40, 70), (300, 40, 40), (200, 1000, 333),
                                   (3000, 64, 64), (2000, 33, 21), (1500, 100, 120), (4000, 300, 136)])
def test_gradient(M, K, N, dtype):
    from paper_2609_09020_gb300 import pic
    x, w = normal((M, K), dtype, 1), normal((N, K), dtype, 2, 1.4 / math.sqrt(K))
    dy, z = normal((M, N), dtype, 3, 0.1), normal((M, N), dtype, 4, 1.4)
    m, n = M // 2, N - 3
    clean = z.clone()
    clean[m, n] = -8.0  # a derivative of zero
    z[m, n] = math.nan
    want = ref.backward(dy, x, w, clean, "relu")
    dy_inf = dy.clone()
    dy_inf[m, n] = math.inf
    for d in (dy, dy_inf):
        for g, v, name in zip(pic.linear_backward(d, x, w, act="relu", pre=z), want, ("dx", "dw", "db")):
            ref.check(g, v, name)
    dx, dw, db = pic.linear_backward(dy, x, w, act="gelu", pre=z)
    pic.linear_check()
    (vx, tx), (vw, tw), (vb, tb) = ref.backward(dy, x, w, clean, "gelu")
    rows, outs = torch.arange(M, device="cuda") != m, torch.arange(N, device="cuda") != n
    assert bool(dx[m].isnan().all()) and bool(dw[n].isnan().all()) and bool(db[n].isnan())
    ref.check(dx[rows], (vx[rows], tx[rows]), "dx")
    ref.check(dw[outs], (vw[outs], tw[outs]), "dw")
    ref.check(db[outs], (vb[outs], tb[outs]), "db")
