"""How far gelu's polynomial is off: the normal distribution below -a as 2 to a polynomial, evaluated from the kernels' own coefficients in fp32
here, and through a product's activation on the GPU."""
import math
import os
import re

import numpy as np
import pytest
import torch

POINTWISE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_23227_amd", "csrc", "pointwise.h")
ABSOLUTE, TIMES_A, RELATIVE = 1.1e-7, 5e-8, 3.5e-5     # as the comment at normal_tail states them, the last one below 6


def tail(a):
    return np.array([0.5 * math.erfc(float(v) / math.sqrt(2)) for v in a])


def test_the_tail_of_the_normal_distribution():
    with open(POINTWISE) as f:
        body = f.read().split("float normal_tail(float a)")[1].split("}")[0]
    coefficients = [np.float32(v) for v in re.findall(r"(-?\d+\.\d+(?:e-\d+)?)f", body)]
    assert len(coefficients) == 11
    a = np.linspace(0, 8, 200_001, dtype=np.float32)
    p = np.full_like(a, coefficients[0])
    for c in coefficients[1:]:                         # (a product of two fp32 numbers is exact in 64 bits, so this is fma)
        p = (p.astype(np.float64) * a + np.float64(c)).astype(np.float32)
    ref = tail(a)
    off = np.abs(np.exp2(p.astype(np.float64)) - ref)
    assert off.max() <= ABSOLUTE and (a * off).max() <= TIMES_A
    assert (off / ref)[a <= 6].max() <= RELATIVE


@pytest.mark.gpu
def test_gelu_of_negative_numbers():
    """gelu(-a) = -a tail(a), with a rounding in the exponential and one in the product, 2^-23 of it each."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2511_23227_amd as pcpp
    a = torch.linspace(0, 6, 60_001)
    zeros = pcpp.pcpp_mx_pack(torch.zeros(a.numel(), 32, device="cuda")).rows
    y = pcpp.pcpp_mx_product(pcpp.pcpp_mx_pack(torch.zeros(1, 32, device="cuda")).rows, zeros, -a.cuda(), act=pcpp.ACT_GELU, dtype=torch.float32)[0]
    a = a.double().numpy()
    ref = -a * tail(a)
    off = np.abs(y.double().cpu().numpy() - ref)
    assert (off <= TIMES_A + 2.0 ** -22 * np.abs(ref)).all()
    assert (off <= (RELATIVE + 2.0 ** -22) * np.abs(ref)).all()
