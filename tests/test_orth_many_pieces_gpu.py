"""Norms of matrices whose squares are added up by a kernel of their own (more than 4096
pieces of 32 x 512), alone and beside others."""
import pytest

torch = pytest.importorskip("torch")

import orth_ref  # noqa: E402

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


# 4096 pieces, one more, many
@pytest.mark.parametrize("shape,dtype", [((4, 2 ** 21), BF16), ((4, 2 ** 21 + 1), BF16), ((1, 2 ** 24 + 5), F32), ((40, 10 ** 7), F16),
                                         ((2 ** 22, 3), F32)], ids=str)
def test_many_pieces(pic, shape, dtype):
    g = [normal((300, 200), F32, 1), normal(shape, dtype, 2), normal((64, 64), BF16, 3), normal((200, 900), BF16, 4)]
    want = [orth_ref.exact(t, steps=0) for t in g]
    for tensors, exact in ((g[1:2], want[1:2]), (g, want)):
        out = [torch.zeros_like(t) for t in tensors]
        h = pic.Orthogonalizer(tensors, out=out)
        h.orthogonalize(steps=0)
        h.check()
        for o, w in zip(out, exact):
            # a norm and a product in fp32 (four roundings at most), and out's own
            t = o.dtype
            assert bool(((o.double() - w).abs() <= (2.0 ** -22 + orth_ref.ref.ROUND[t]) * w.abs() + orth_ref.ref.TINY[t]).all())
        h.orthogonalize()
        h.check()
        first = [o.clone() for o in out]
        h.orthogonalize()
        h.check()
        assert all(torch.equal(a, b) for a, b in zip(first, out))
        for i, (o, t) in enumerate(zip(out, tensors)):
            if t.numel() < 10 ** 8:
                orth_ref.check(o, t, name=str(i))
        h.close()


def test_a_piece_that_is_not_finite(pic):
    g = [normal((3, 2 ** 22), BF16, 1), normal((300, 200), F32, 2)]
    g[0][2, 2 ** 22 - 1] = float("inf")
    out = [torch.zeros_like(t) for t in g]
    h = pic.Orthogonalizer(g, out=out)
    h.orthogonalize()
    h.check()
    assert bool(out[0].isnan().all())
    orth_ref.check(out[1], g[1])
    h.close()
