"""A call of pic.Orthogonalizer whose waits ran out (test_group_wait_gpu.py) and the calls
behind it, before anything is checked: theirs are right."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
SHORT_LIMIT = 1 << 10
F32, F16 = torch.float32, torch.float16


@pytest.fixture(scope="module")
def pic():
    from paper_2609_09020_gb300 import build, pic
    build.build()
    return pic


def fill(g, seed):
    g.normal_(0.0, 0.02, generator=torch.Generator(device="cuda").manual_seed(seed))


# sums so long that their parts are several rounds of CTAs: some of a tile's never come, and
# an early one would be taken for the last
@pytest.mark.parametrize("shape,dtype", [((8, 2 ** 20), F32), ((70, 2 ** 20), F16)], ids=str)
def test_the_next_call_is_right(pic, shape, dtype):
    g = torch.empty(shape, dtype=dtype, device="cuda")
    out, want = torch.zeros_like(g), torch.zeros_like(g)
    h, other = pic.Orthogonalizer([g], out=[out]), pic.Orthogonalizer([g], out=[want])
    lib = pic.load_library()
    fill(g, 0)
    torch.cuda.synchronize()
    assert lib.pic_linear_test_wait_fault(1, SHORT_LIMIT) == pic.PIC_OK
    try:
        h.orthogonalize(steps=1)
        torch.cuda.synchronize()
    finally:
        lib.pic_linear_test_wait_fault(0, 0)
    for seed in (1, 2):
        fill(g, seed)
        for steps in (1, 5):
            h.orthogonalize(steps=steps)
            other.orthogonalize(steps=steps)
            torch.cuda.synchronize()
            assert torch.equal(out, want)
    with pytest.raises(pic.PicError) as e:
        h.check()
    assert e.value.status == pic.PIC_ERR_TIMEOUT
    h.check()  # said once
    other.check()
    h.orthogonalize()
    h.check()
    assert torch.equal(out, want)
    h.close()
    other.close()


# tiles whose sums are taken over, by pairs of CTAs and by one, in lists of one type and of two
@pytest.mark.parametrize("shape,count,types", [((1024, 1100), 14, [F32]), ((1024, 1100), 14, [F32, torch.bfloat16]),
                                               ((300, 5000), 40, [F32]), ((60, 20000), 60, [F32, F16])], ids=str)
def test_sums_that_are_taken_over(pic, shape, count, types):
    g = [torch.empty(shape, dtype=types[i % len(types)], device="cuda") for i in range(count)]
    for i, t in enumerate(g):
        fill(t, i)
    out, want = [torch.zeros_like(t) for t in g], [torch.zeros_like(t) for t in g]
    h, other = pic.Orthogonalizer(g, out=out), pic.Orthogonalizer(g, out=want)
    lib = pic.load_library()
    other.orthogonalize()
    other.check()
    assert lib.pic_linear_test_wait_fault(1, SHORT_LIMIT) == pic.PIC_OK
    try:
        h.orthogonalize()
        torch.cuda.synchronize()
    finally:
        lib.pic_linear_test_wait_fault(0, 0)
    for _ in range(2):
        h.orthogonalize()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
    with pytest.raises(pic.PicError) as e:
        h.check()
    assert e.value.status == pic.PIC_ERR_TIMEOUT
    h.check()
    h.close()
    other.close()
