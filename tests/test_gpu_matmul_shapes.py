"""Every shape of workgroups of the 8-bit product, at ragged sizes, against the formula in 64 bits.

Tolerance: as for the other products.  Products of two 8-bit values are exact in fp32; a sum of n fp32 terms in any order is off by n * 2^-24 of the
sum of their absolute values: 128 of a group, the groups, two roundings for the scales, eight partial sums.  A bf16 output of more than 64 rows
is summed inside a group by the 8-bit matrix instruction: each of 128 products may lose 2^-13 of the largest one.  Then the output's rounding.
"""
import pytest
import torch

import paper_2510_08525_amd as rl
from matmul_shapes import SHAPES

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn
U = 2.0 ** -24


def _g(n):
    return -(-n // 128)


def _matrix(rows, k, g):
    """Normal values with a few columns far larger than the rest, as activations have them; NaN between the rows."""
    raw = torch.full((rows, k + 16), 0x7f, dtype=torch.uint8, device="cuda")
    big = 1.0 + 19.0 * (torch.rand(k, generator=g) < 0.01)
    raw[:, :k] = (torch.randn(rows, k, generator=g) * 20 * big).clamp(-448, 448).to(E4M3).view(torch.uint8).cuda()
    return raw.view(E4M3)[:, :k]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_products(m, n, k, dtype):
    g = torch.Generator().manual_seed(m + n + k)
    a, b = _matrix(m, k, g), _matrix(n, k, g)
    sa, sb = (torch.rand(_g(k), m, generator=g) * 2 - 0.5).cuda(), (torch.rand(_g(n), _g(k), generator=g) * 2 - 0.5).cuda()
    out = torch.full((m, n + 5), 7.0, dtype=dtype, device="cuda")
    rl.scaled_matmul(a, sa, b, sb, out[:, :n])
    assert (out[:, n:] == 7.0).all()
    left = a.float().double() * sa.t().double().repeat_interleave(128, 1)[:, :k]
    right = b.float().double() * sb.double().repeat_interleave(128, 0)[:n].repeat_interleave(128, 1)[:, :k]
    y = left @ right.t()
    tol = (128 + _g(k) + 10) * U * (left.abs() @ right.abs().t())
    tol += (2.0 ** -8 if dtype == torch.bfloat16 else U) * y.abs()
    if dtype == torch.bfloat16 and m > 64:
        most = lambda x: torch.nn.functional.pad(x.abs(), (0, _g(k) * 128 - k)).view(x.shape[0], -1, 128).amax(-1)      # noqa: E731
        tol += 2.0 ** -6 * most(left) @ most(right).t()
    err = (out[:, :n].double() - y).abs()
    assert (err <= tol).all(), (int((~(err <= tol)).sum()), (~(err <= tol)).nonzero()[:3].tolist())
    # most of them are much nearer: a group left out or counted twice would not be
    assert err.norm() <= 1.1 * 2.0 ** -8 * y.norm()
