"""One large product of a group beside many small ones of the same sign: what the 8-bit matrix instruction drops, for a bf16 output of more than 64
rows, and that nothing is dropped elsewhere.

448 * 448 has the exponent 17: what lies below 2^(17 - 13) = 16 may be lost of each of the 127 other products, which is all of 3 * 3.5 = 10.5, but
not more than that.  So the sum comes out between the exact one and that less 127 * 10.5 = 1333.5 (0.66 % of it, within the 2^-6 of the largest product
that is stated), and is rounded to bf16 then (2^-8); exact products of fp32 sums are off by 128 * 2^-24 and their output's rounding.
"""
import pytest
import torch

import paper_2510_08525_amd as rl

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn
BIG, LOST = 448.0 * 448.0, 127 * 10.5


def _product(m, dtype, place):
    a, b = torch.full((m, 256), 3.0, device="cuda"), torch.full((80, 256), 3.5, device="cuda")
    for x in (a, b):
        x[:, place] = 448.0
        x[:, 128:] = 0.0
    out = torch.empty(m, 80, dtype=dtype, device="cuda")
    rl.scaled_matmul(a.to(E4M3), torch.ones(2, m, device="cuda"), b.to(E4M3), torch.ones(1, 2, device="cuda"), out)
    return out.double()


@pytest.mark.parametrize("place", [0, 37, 127])
@pytest.mark.parametrize("m", [1, 64, 65, 300, 2000])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_one_large_product(m, dtype, place):
    y = BIG + LOST
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    lost = LOST if dtype == torch.bfloat16 and m > 64 else 0.0
    out = _product(m, dtype, place)
    assert (out <= y * (1 + half + 128 * 2.0 ** -24)).all()
    assert (out >= (y - lost) * (1 - half - 128 * 2.0 ** -24)).all(), float(out.min())
    assert (out >= y - 2.0 ** -6 * BIG - half * y).all()


@pytest.mark.parametrize("m", [65, 2000])
def test_nothing_is_lost_within_two_to_the_seventh(m):
    """Values within 2^7 of the group's largest product come out exactly: 16 * 16 beside 127 of 3 * 3.5, whose sum bf16 does not hold but whose
    rounding is that of the exact sum."""
    a, b = torch.full((m, 128), 3.0, device="cuda"), torch.full((80, 128), 3.5, device="cuda")
    a[:, 5] = b[:, 5] = 16.0
    out = torch.empty(m, 80, dtype=torch.bfloat16, device="cuda")
    rl.scaled_matmul(a.to(E4M3), torch.ones(1, m, device="cuda"), b.to(E4M3), torch.ones(1, 1, device="cuda"), out)
    assert (out == torch.tensor(256.0 + LOST).bfloat16().cuda()).all()
