"""fp32 updates of long and large matrices: out's error beside that of the same steps in
elementary fp32 operations.  Operands have 22 bits, and sums lose up to 2^-24 of themselves
with each 16 of K until they are taken over; the steps multiply both as they multiply what
fp32 operations lose, so that a few times their error is the measure: four, as in orth_ref,
and no allowance beside it but 2^-20.  Whatever else is in the list."""
import pytest

torch = pytest.importorskip("torch")

import orth_ref  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pic():
    from paper_2609_09020_gb300 import build, pic
    build.build()
    return pic


def normal(shape, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").mul_(0.02).to(dtype)


@pytest.mark.parametrize("shape,count", [((130, 20000), 1), ((130, 20000), 40), ((200, 20000), 1), ((512, 20000), 1),
                                         ((20000, 512), 1), ((130, 100000), 1), ((60, 20000), 40), ((700, 20000), 2),
                                         ((1500, 1500), 1), ((1000, 4000), 3), ((2048, 2048), 4), ((2048, 6000), 1)],
                         ids=str)
def test_long(pic, shape, count):
    g = [normal(shape, torch.float32, s) for s in range(count)]
    beside = [normal((300, 200), torch.bfloat16, 5), normal((40, 30), torch.float16, 6)]
    out = [torch.zeros_like(t) for t in g + beside]
    h = pic.Orthogonalizer(g + beside, out=out)
    h.orthogonalize()
    h.check()
    h.close()
    mean = lambda v: float(v.square().mean().sqrt())
    for i in sorted({0, count - 1}):
        want = orth_ref.exact(g[i])
        plain = mean(orth_ref.single(g[i]) - want)
        assert mean(out[i].double() - want) <= 4 * plain + 2.0 ** -20 * mean(want)
    for t, o in zip(beside, out[count:]):
        orth_ref.check(o, t)


@pytest.mark.parametrize("shape", [(1, 2 ** 24 + 5), (3, 5000001), (2 ** 22, 2), (64, 300000)], ids=str)
def test_few_rows(pic, shape):
    """Within orth_ref's bounds where A is a handful of very long sums of squares."""
    g = normal(shape, torch.float32, 2)
    out = torch.zeros_like(g)
    h = pic.Orthogonalizer([g], out=[out])
    h.orthogonalize()
    h.check()
    h.close()
    orth_ref.check(out, g)
