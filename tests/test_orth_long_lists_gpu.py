"""pic.Orthogonalizer of lists whose tensor maps are too many to be acquired at the start
of every CTA (more than 64 matrices), of all tile shapes and types."""
import pytest

torch = pytest.importorskip("torch")

import orth_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def pic():
    from paper_2609_09020_gb300 import build, pic
    build.build()
    return pic


def normal(shape, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").mul_(0.02).to(dtype)


# tiles of 64 columns (up to 64 on the smaller side), of 128, of 256 (above 512, with as many),
# and matrices that one CTA takes between them
LISTS = {
    "all shapes": [(64, 700), (150, 140), (530, 800), (40, 30), (1200, 50), (300, 131)] * 14,
    "64 columns": [(64, 700), (900, 33)] * 40,
    "128 columns": [(129, 200), (260, 135), (300, 300)] * 26,
    "256 columns": [(600, 530), (530, 1100)] * 35,
}


@pytest.mark.parametrize("which", LISTS)
@pytest.mark.parametrize("types", [[F32], [BF16], [F32, BF16, F16, BF16, BF16]], ids=str)
def test_long_lists(pic, which, types):
    shapes = LISTS[which]
    assert len(shapes) > 64
    g = [normal(s, types[i % len(types)], i) for i, s in enumerate(shapes)]
    out = [torch.full_like(t, 7.0) for t in g]
    h = pic.Orthogonalizer(g, out=out)
    h.orthogonalize()
    h.check()
    first = [o.clone() for o in out]
    for i in list(range(0, len(g), 9)) + list(range(len(g) - 6, len(g))):
        ref.check(out[i], g[i], name=f"{i}: {shapes[i]} {g[i].dtype}")
    # again, with the matrices in other places of the list: the same arithmetic but for how sums are cut
    turned = g[1:] + g[:1]
    other = [torch.full_like(t, 7.0) for t in turned]
    h2 = pic.Orthogonalizer(turned, out=other)
    h2.orthogonalize()
    h.orthogonalize()
    h2.check()
    h.check()
    assert all(torch.equal(a, b) for a, b in zip(first, out))
    for i in range(0, len(g), 23):
        ref.check(other[i - 1], g[i], name=f"turned {i}: {shapes[i]} {g[i].dtype}")
    h.close()
    h2.close()


def test_a_long_list_captured(pic):
    g = [normal(s, (F32, BF16)[i % 2], i) for i, s in enumerate(LISTS["all shapes"])]
    out = [torch.zeros_like(t) for t in g]
    h = pic.Orthogonalizer(g, out=out)
    h.orthogonalize()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h.orthogonalize()
    for i, t in enumerate(g):
        t.copy_(normal(t.shape, t.dtype, 100 + i))
    graph.replay()
    torch.cuda.synchronize()
    got = [o.clone() for o in out]
    h.orthogonalize()
    h.check()
    assert all(torch.equal(a, b) for a, b in zip(got, out))
    for i in range(0, len(g), 11):
        ref.check(got[i], g[i], name=str(i))
    h.close()
