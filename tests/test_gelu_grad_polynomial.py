"""The generated polynomial of GELU': its header is the generator's, its error
is the one stated, and it ends where it should."""
import os
import re

import numpy as np

from paper_2609_09020_gb300 import gen_gelu_grad as gen

HEADER = os.path.join(os.path.dirname(os.path.abspath(gen.__file__)), "csrc", "pic_gelu_grad.cuh")


def coefficients(name="gelu_grad_c"):
    text = open(HEADER).read()
    text = text[text.index(name + "(int"):]
    body = text[text.index("c[] = {"):text.index("return c[i]")]
    return np.array([float(v) for v in re.findall(r"(-?[\d.]+(?:e-?\d+)?)f", body)][::-1])


def test_header_is_generated():
    # the fit may differ in the last digits from one linear algebra library to another
    assert np.allclose(coefficients(), gen.fit(), rtol=1e-3, atol=1e-6)


def test_error():
    c = coefficients()
    assert gen.max_error(c) < 5e-7
    assert np.all(gen.grad_fp32(np.array([6.0, 10.0, 1e30, np.inf]), c) == 1)
    assert np.all(gen.grad_fp32(np.array([-6.0, -10.0, -1e30, -np.inf]), c) == 0)
    assert abs(float(gen.grad_fp32(np.array([0.0]), c)[0]) - 0.5) < 5e-7


def test_fp32_polynomial():
    c = coefficients("gelu_grad_c32")
    assert len(c) == gen.DEG_FP32 + 1 and len(coefficients()) == gen.DEG + 1
    assert gen.max_error(c) < 1.5e-7
    assert np.all(gen.grad_fp32(np.array([6.0, np.inf]), c) == 1) and np.all(gen.grad_fp32(np.array([-6.0, -np.inf]), c) == 0)


def test_gelu_polynomial():
    c = coefficients("gelu_c32")
    assert len(c) == gen.DEG_GELU + 1 and c[0] == 0
    z = np.linspace(-12, 12, 300_001).astype(np.float32)
    from scipy.special import ndtr
    want = z.astype(np.float64) * ndtr(z.astype(np.float64))
    # half an ulp of the result, and 1e-7 of the polynomial and its evaluation
    assert np.all(np.abs(gen.gelu_fp32(z, c) - want) <= 1e-7 + 2.0 ** -24 * np.abs(want))
    assert np.all(gen.gelu_fp32(np.array([-6.0, -30.0, -np.inf]), c) == 0)
    assert gen.gelu_fp32(np.array([np.inf]), c)[0] == np.inf and gen.gelu_fp32(np.array([0.0]), c)[0] == 0
