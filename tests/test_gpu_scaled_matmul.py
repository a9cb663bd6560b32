"""Product of 8-bit matrices with a scale for each group of 128, against the formula in 64 bits.

Tolerance: products of two 8-bit values are exact in fp32; a sum of n fp32 terms in any order is off by at most n * 2^-24 of the sum of
their absolute values: 128 terms inside a group, the groups, two roundings for the scales, and eight partial sums; then the output's rounding.
A bf16 output of more than 64 rows is summed inside a group by the 8-bit matrix instruction: each of up to 128 products may lose 2^-13 of the
largest one more (by the exponent of that, at most the product of the group's largest values of both sides).
"""
import pytest
import torch

import paper_2510_08525_amd as rl

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn
U = 2.0 ** -24


def _g(n):
    return -(-n // 128)


def _bytes(rows, cols, g, stride):
    """Any finite value of the type, rows `stride` bytes apart with NaN between them."""
    raw = torch.full((rows, stride), 0x7f, dtype=torch.uint8, device="cuda")
    v = torch.randint(0, 256, (rows, cols), generator=g, dtype=torch.uint8)
    v[(v & 0x7f) == 0x7f] = 0
    raw[:, :cols] = v.cuda()
    return raw.view(E4M3)[:, :cols]


def _inputs(m, n, k, seed=0, pad=0):
    g = torch.Generator().manual_seed(seed + m + 3 * n + 7 * k)
    a, b = _bytes(m, k, g, k + pad), _bytes(n, k, g, k + 2 * pad)
    sa = (torch.rand(_g(k), m, generator=g) * 2 - 0.5).cuda()
    sb = (torch.rand(_g(n), _g(k), generator=g) * 2 - 0.5).cuda()
    return a, sa, b, sb


def _wide(a, sa, b, sb):
    k, n = a.shape[1], b.shape[0]
    left = a.float().double() * sa.t().double().repeat_interleave(128, 1)[:, :k]
    right = b.float().double() * sb.double().repeat_interleave(128, 0)[:n].repeat_interleave(128, 1)[:, :k]
    return left @ right.t(), left.abs() @ right.abs().t()


def _most(x, scales):
    """The largest absolute value of each group, scaled: [groups, rows]."""
    pad = torch.nn.functional.pad(x.float().double(), (0, _g(x.shape[1]) * 128 - x.shape[1]))
    return pad.view(x.shape[0], -1, 128).abs().amax(-1).t() * scales.double().abs()


def _check(out, a, sa, b, sb):
    k, n = a.shape[1], b.shape[0]
    y, size = _wide(a, sa, b, sb)
    half = 2.0 ** -8 if out.dtype == torch.bfloat16 else U
    tol = (128 + _g(k) + 10) * U * size + half * y.abs() + 1e-30
    if out.dtype == torch.bfloat16 and out.shape[0] > 64:
        tol += 2.0 ** -6 * _most(a, sa).t() @ _most(b, sb.t().repeat_interleave(128, 1)[:, :n])
    got = out.double()
    assert torch.isfinite(got).all()
    bad = (got - y).abs() > tol
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist(), float(((got - y).abs() / tol).max()))


SHAPES = [(m, n, k) for m in (1, 3, 16, 17, 33, 64, 65, 129, 300) for n, k in ((1, 16), (5, 128), (128, 144), (300, 1040), (1000, 384))]
SHAPES += [(1, 4608, 3584), (7, 6144, 4096), (16, 128, 9216), (48, 640, 2064), (128, 128, 128), (128, 256, 8192), (130, 4000, 528),
           (333, 4608, 3584), (1000, 1000, 1008), (4096, 4096, 272), (4097, 4100, 144), (2048, 8200, 640), (260, 16640, 16)]


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_products(m, n, k, dtype):
    a, sa, b, sb = _inputs(m, n, k)
    out = torch.full((m, n), float("nan"), dtype=dtype, device="cuda")
    assert rl.scaled_matmul(a, sa, b, sb, out) is out
    _check(out, a, sa, b, sb)


def test_normal_values_are_off_by_the_outputs_rounding():
    """2-norms: a bf16 output's rounding is at most 2^-8 of each value, and the fast sums of such values do not show beside it."""
    g = torch.Generator().manual_seed(1)
    a, b = ((torch.randn(n, 1024, generator=g) * 100).clamp(-448, 448).to(E4M3).cuda() for n in (300, 500))
    sa, sb = torch.rand(8, 300, generator=g).cuda() + 0.5, torch.rand(4, 8, generator=g).cuda() + 0.5
    out = torch.empty(300, 500, dtype=torch.bfloat16, device="cuda")
    rl.scaled_matmul(a, sa, b, sb, out)
    y, _ = _wide(a, sa, b, sb)
    assert (out.double() - y).norm() <= 2.0 ** -8 * y.norm()


@pytest.mark.parametrize("m,n,k", [(1, 130, 272), (20, 77, 400), (64, 515, 128), (200, 300, 656), (4096, 4099, 48)])
def test_strides(m, n, k):
    """Rows apart, with NaN between them; an output whose rows start anywhere and keep what lies between them."""
    a, sa, b, sb = _inputs(m, n, k, pad=48)
    wide_sa = torch.full((_g(k), m + 3), float("nan"), device="cuda")
    wide_sa[:, :m] = sa
    wide_sb = torch.full((_g(n), _g(k) + 2), float("nan"), device="cuda")
    wide_sb[:, :_g(k)] = sb
    for dtype in (torch.bfloat16, torch.float32):
        for shift, gap in ((0, 8), (1, 3)):
            buf = torch.full((shift + m * (n + gap),), 7.0, dtype=dtype, device="cuda")
            out = buf[shift:].view(m, n + gap)[:, :n]
            rl.scaled_matmul(a, wide_sa[:, :m], b, wide_sb[:, :_g(k)], out)
            _check(out, a, sa, b, sb)
            assert (buf[shift:].view(m, n + gap)[:, n:] == 7.0).all() and (buf[:shift] == 7.0).all()


def test_rows_may_repeat():
    a, sa, b, sb = _inputs(1, 200, 256)
    out = torch.empty(70, 200, device="cuda")
    rl.scaled_matmul(a.view(torch.uint8).expand(70, 256).view(E4M3), sa.expand(2, 70).contiguous(), b, sb, out)
    _check(out, a.float().expand(70, 256), sa.expand(2, 70), b, sb)


@pytest.mark.parametrize("m", [4, 200])
def test_nan_and_infinite_scales_stay_in_their_rows(m):
    a, sa, b, sb = _inputs(m, 256, 384)
    raw = a.view(torch.uint8)
    raw[1, 130] = 0x7f                             # a NaN in one row of a
    b.view(torch.uint8)[5, 200] = 0xff             # and one of b
    sa[2, 3] = float("inf")
    out = torch.empty(m, 256, device="cuda")
    rl.scaled_matmul(a, sa, b, sb, out)
    assert out[1].isnan().all() and out[:, 5].isnan().all() and not torch.isfinite(out[3]).any()
    keep_m = [i for i in range(m) if i not in (1, 3)]
    keep_n = [i for i in range(256) if i != 5]
    part = out[keep_m][:, keep_n]
    assert torch.isfinite(part).all()
    raw[1, 130] = 0
    b.view(torch.uint8)[5, 200] = 0
    sa[2, 3] = 1.0
    y, size = _wide(a, sa, b, sb)
    assert ((part.double() - y[keep_m][:, keep_n]).abs() <= 142 * U * size[keep_m][:, keep_n] + U * y[keep_m][:, keep_n].abs()).all()


@pytest.mark.parametrize("m", [2, 300])
def test_equal_calls_give_equal_bits_and_graphs_replay(m):
    a, sa, b, sb = _inputs(m, 1000, 1024)
    out, again = torch.empty(m, 1000, device="cuda"), torch.empty(m, 1000, device="cuda")
    rl.scaled_matmul(a, sa, b, sb, out)
    rl.scaled_matmul(a, sa, b, sb, again)
    assert torch.equal(out, again)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rl.scaled_matmul(a, sa, b, sb, again)
    for seed in range(3):
        x = _inputs(m, 1000, 1024, seed=100 + seed)
        a.view(torch.uint8).copy_(x[0].view(torch.uint8)), sa.copy_(x[1])
        graph.replay()
        torch.cuda.synchronize()
        rl.scaled_matmul(a, sa, b, sb, out)
        assert torch.equal(out, again)
        _check(out, a, sa, b, sb)


def test_tensor_checks():
    a, sa, b, sb = _inputs(4, 256, 256)
    out = torch.empty(4, 256, device="cuda")
    for bad in (lambda: rl.scaled_matmul(a.float(), sa, b, sb, out), lambda: rl.scaled_matmul(a, sa.t(), b, sb, out),
                lambda: rl.scaled_matmul(a, sa, b[:, :128], sb, out), lambda: rl.scaled_matmul(a, sa, b, sb[:1], out),
                lambda: rl.scaled_matmul(a, sa, b, sb, out.half()), lambda: rl.scaled_matmul(a, sa, b, sb, out.t()),
                lambda: rl.scaled_matmul(a, sa.double(), b, sb, out), lambda: rl.scaled_matmul(a, sa, b.cpu(), sb, out)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(rl.RlkvError):                                       # 250 columns: not a multiple of 16
        rl.scaled_matmul(a[:, :250], sa, b[:, :250], sb, out)
