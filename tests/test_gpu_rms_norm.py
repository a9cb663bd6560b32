"""Norm with residual, and quantising, against the formulas in 64 bits.

Tolerances.  fp32: a sum of squares of n positive terms, at most 64 of a thread one after the other and 8 steps over lanes and
wavefronts (more beyond 16384 columns), is off by at most 2^-24 of itself a step, and its root by half of that; the remaining products and
the root add a few: 48 + n / 256 roundings of 2^-24 in all.  bf16: 2^-8 more, the output's rounding.  Scales: those of the values.
8 bits: half a step, 2^-4 of the value or 2^-10, and what the value itself is off.
"""
import numpy as np
import pytest
import torch

import paper_2510_08525_amd as rl

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn
EPS = 1e-5
U = 2.0 ** -24


def _inputs(rows, cols, dtype, seed, pad=0, shift=0):
    g = torch.Generator().manual_seed(seed)
    def matrix(scale):
        m = torch.full((rows * (cols + pad) + shift + 8,), float("nan"), dtype=dtype, device="cuda")
        m = m[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
        m.copy_((torch.randn(rows, cols, generator=g) * scale).to(dtype))
        return m
    return matrix(1.0), matrix(3.0), (1 + 0.2 * torch.randn(cols, generator=g)).to(dtype).cuda()


def _expected(x, res, w):
    h = x.double() + (res.double() if res is not None else 0)
    return h, h / torch.sqrt((h * h).mean(-1, keepdim=True) + EPS) * (w.double() if w is not None else 1)


def _rel(cols):
    return (48 + cols / 256) * U


def _check_values(out, y, rel, dtype):
    half = 2.0 ** -8 if dtype == torch.bfloat16 else U
    assert torch.isfinite(out.float()).all()
    assert ((out.double() - y).abs() <= (rel + half) * y.abs() + 1e-37).all(), float((out.double() - y).abs().max())


def _check_quantized(q, scales, y, rel):
    rows, cols = y.shape
    G = -(-cols // 128)
    pad = torch.nn.functional.pad(y, (0, G * 128 - cols)).view(rows, G, 128)
    s = (pad.abs().amax(-1) / 448).clamp(min=2.0 ** -126)
    assert scales.shape == (G, rows)
    assert ((scales.t().double() - s).abs() <= (rel + 4 * U) * s).all()
    v = (pad / s[..., None]).view(rows, -1)[:, :cols]
    got = q.float().double()
    assert torch.isfinite(got).all()
    near = v.abs() * (rel + 8 * U)
    assert ((got - v).abs() <= torch.clamp(v.abs() * 2.0 ** -4, min=2.0 ** -10) + near * 1.07).all()


# one thread's columns, pieces that end inside a row, every form of the kernel (wavefront or workgroup a row, pieces in registers or
# read twice), many rows per workgroup
SIZES = [(1, 1), (3, 7), (2, 8), (5, 100), (1, 127), (4, 128), (3, 129), (1, 4096), (7, 4097), (2, 5001), (3, 8192), (2, 8200),
         (2, 16384), (3, 20011), (1031, 136), (1024, 4096), (1500, 515), (8195, 40), (9000, 256)]


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("residual", [True, False])
def test_norm(rows, cols, dtype, residual):
    x, res, w = _inputs(rows, cols, dtype, rows + cols)
    res = res if residual else None
    h, y = _expected(x, res, w)
    out = torch.full((rows, cols), float("nan"), dtype=dtype, device="cuda")
    total = torch.full_like(out, float("nan")) if residual else None
    assert rl.rms_norm(x, w, EPS, out, residual=res, sum_out=total) is out
    _check_values(out, y, _rel(cols), dtype)
    if residual:
        _check_values(total, h, 0.0, dtype)
    q = torch.zeros(rows, cols, dtype=torch.uint8, device="cuda").view(E4M3)
    scales = torch.full((-(-cols // 128), rows), float("nan"), device="cuda")
    rl.rms_norm(x, w, EPS, q, scales=scales, residual=res)
    _check_quantized(q, scales, y, _rel(cols))
    rl.quantize(x, q, scales)
    _check_quantized(q, scales, x.double(), 0.0)


@pytest.mark.parametrize("cols,pad,shift", [(300, 4, 0), (256, 8, 0), (256, 1, 0), (512, 0, 1), (129, 7, 3), (9000, 3, 1), (17000, 9, 1)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strides_and_alignment(cols, pad, shift, dtype):
    """Rows apart, rows at any element: what lies between them is neither read into a result nor written."""
    rows = 6
    x, res, w = _inputs(rows, cols, dtype, 5, pad, shift)
    h, y = _expected(x, res, w)
    buf = torch.full((rows * (cols + pad) + shift,), 7.0, dtype=dtype, device="cuda")
    out = buf[shift:].view(rows, cols + pad)[:, :cols]
    raw = torch.zeros(rows * (cols + pad) + shift, dtype=torch.uint8, device="cuda")
    q = raw[shift:].view(rows, cols + pad)[:, :cols].view(E4M3)
    big = torch.full((-(-cols // 128), rows + pad), -1.0, device="cuda")
    rl.rms_norm(x, w, EPS, out, residual=res)
    _check_values(out, y, _rel(cols), dtype)
    rl.rms_norm(x, w, EPS, q, scales=big[:, :rows], residual=res)
    _check_quantized(q, big[:, :rows], y, _rel(cols))
    if pad:
        assert (buf[shift:].view(rows, cols + pad)[:, cols:] == 7.0).all()
        assert (raw[shift:].view(rows, cols + pad)[:, cols:] == 0).all()
        assert (big[:, rows:] == -1.0).all()


@pytest.mark.parametrize("cols", [1000, 4096, 20000])
def test_in_place(cols):
    """The sum over the residual and the output over x: every form reads what it needs before it writes it."""
    x, res, w = _inputs(5, cols, torch.bfloat16, 8)
    h, y = _expected(x, res, w)
    rl.rms_norm(x, w, EPS, x, residual=res, sum_out=res)
    _check_values(x, y, _rel(cols), torch.bfloat16)
    _check_values(res, h, 0.0, torch.bfloat16)


def test_rows_may_repeat():
    x, res, w = _inputs(1, 640, torch.bfloat16, 9)
    h, y = _expected(x, res, w)
    out = torch.empty(4, 640, dtype=torch.bfloat16, device="cuda")
    rl.rms_norm(x.expand(4, 640), None, EPS, out, residual=res.expand(4, 640))
    _check_values(out, _expected(x, res, None)[1].expand(4, 640), _rel(640), torch.bfloat16)


def test_zeros_infinities_nan():
    """A group of zeros, of values whose scale is the least one, with a NaN, with an infinity."""
    x = torch.randn(1, 5 * 128, device="cuda")
    x[0, :128] = 0
    x[0, 128:256] = 1e-40
    x[0, 256] = float("nan")
    x[0, 384] = float("inf")
    q = torch.empty(1, 640, dtype=torch.uint8, device="cuda").view(E4M3)
    s = torch.empty(5, 1, device="cuda")
    rl.quantize(x, q, s)
    v = q.float()
    assert (v[0, :128] == 0).all() and (s[:2] == 2.0 ** -126).all()
    _check_quantized(q[:, 128:256].contiguous(), s[1:2], x[:, 128:256].double(), 0.0)
    assert v[0, 256].isnan() and torch.isfinite(v[0, 257:384]).all()
    _check_quantized(q[:, 257:384].contiguous(), s[2:3], x[:, 257:384].double(), 0.0)
    assert s[3].isinf() and (v[0, 384:512] * s[3]).isnan().all()
    _check_quantized(q[:, 512:].contiguous(), s[4:], x[:, 512:].double(), 0.0)
    out = torch.empty(2, 256, device="cuda")
    rl.rms_norm(torch.zeros(2, 256, device="cuda"), None, EPS, out)
    assert (out == 0).all()


def test_no_rows():
    out = torch.empty(0, 64, device="cuda")
    assert rl.rms_norm(torch.empty(0, 64, device="cuda"), None, EPS, out) is out


def test_stream_and_graph():
    """On a stream of its own, recorded and replayed on other inputs."""
    x, res, w = _inputs(33, 3584, torch.bfloat16, 11)
    q = torch.zeros(33, 3584, dtype=torch.uint8, device="cuda").view(E4M3)
    s = torch.zeros(28, 33, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        rl.rms_norm(x, w, EPS, q, scales=s, residual=res)
    side.synchronize()
    _check_quantized(q, s, _expected(x, res, w)[1], _rel(3584))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rl.rms_norm(x, w, EPS, q, scales=s, residual=res)
    for seed in range(3):
        a, b, _ = _inputs(33, 3584, torch.bfloat16, 20 + seed)
        x.copy_(a), res.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        _check_quantized(q, s, _expected(x, res, w)[1], _rel(3584))


def test_tensor_checks():
    x, res, w = _inputs(4, 256, torch.bfloat16, 3)
    out, s = torch.empty_like(x), torch.empty(2, 4, device="cuda")
    q = torch.empty(4, 256, dtype=torch.uint8, device="cuda").view(E4M3)
    for bad in (lambda: rl.rms_norm(x[0], w, EPS, out), lambda: rl.rms_norm(x.t(), w, EPS, out),
                lambda: rl.rms_norm(x, w[:255], EPS, out), lambda: rl.rms_norm(x, w.float(), EPS, out),
                lambda: rl.rms_norm(x, w, EPS, out.float()), lambda: rl.rms_norm(x, w, EPS, out[:3]),
                lambda: rl.rms_norm(x.cpu(), w, EPS, out), lambda: rl.rms_norm(x, w, EPS, out.cpu()),
                lambda: rl.rms_norm(x, w, EPS, q, scales=s.t()), lambda: rl.rms_norm(x.half(), w, EPS, out),
                lambda: rl.quantize(x, out, s), lambda: rl.quantize(x, q, s.double())):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: rl.rms_norm(x, w, -1.0, out), lambda: rl.rms_norm(x, w, EPS, q), lambda: rl.rms_norm(x, w, EPS, out, scales=s),
                lambda: rl.rms_norm(x, w, EPS, out, sum_out=res)):
        with pytest.raises(rl.RlkvError):
            bad()
