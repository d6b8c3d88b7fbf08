"""pic.grouped_linear_check where a wait ran out and offsets were wrong: it says both, one
after the other."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
SHORT_LIMIT = 1 << 10


def test_both_are_said():
    from paper_2609_09020_gb300 import build, pic
    build.build()
    lib = pic.load_library()
    x, w = torch.ones((8192, 128), device="cuda").half(), torch.ones((3, 8192, 128), device="cuda").half()
    o = torch.tensor([0, 4000, 3000, 9000], device="cuda")
    torch.cuda.synchronize()
    assert lib.pic_linear_test_wait_fault(1, SHORT_LIMIT) == pic.PIC_OK
    try:
        pic.grouped_linear(x, w, o)
        torch.cuda.synchronize()
    finally:
        lib.pic_linear_test_wait_fault(0, 0)
    for status in (pic.PIC_ERR_TIMEOUT, pic.PIC_ERR_INVALID_ARG):
        with pytest.raises(pic.PicError) as e:
            pic.grouped_linear_check()
        assert e.value.status == status
    pic.grouped_linear_check()
