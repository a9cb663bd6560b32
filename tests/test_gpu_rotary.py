"""Rotation of packed projections and their append to the cache.

What is handed out is held to the formula in 64 bits; what goes into a cache has to be, byte for byte of the whole arena, what the plain append
of the handed-out rows leaves there.

Tolerance of (x cos t - y sin t): the angle is off by 2^-24 of up to an eighth of a turn and less than 2^-27 besides, the series and its
evaluation by 3 * 2^-24, the two products and their sum by 2^-24 of |x| + |y| each: 6 * 2^-24 (|x| + |y|) in all, and the output's rounding.
"""
import math

import numpy as np
import pytest
import torch

import paper_2510_08525_amd as rl

pytestmark = pytest.mark.gpu
D = 128
U = 2.0 ** -24


def _freq(pairs, base=500000.0):
    return [base ** (-i / pairs) for i in range(pairs)]


def _cache(Hq, H, B, S, R, dtype, mask, cap, kernel=rl.RLKV_KERNEL_AUTO, fill=0, **kw):
    return rl.Cache(1, Hq, H, D, B, S, R, rl.RLKV_F32 if dtype == torch.float32 else rl.RLKV_BF16, mask, [cap] * B, kernel=kernel,
                    arena_fill=fill, **kw)


def _packed(B, T, heads, dtype, seed, gap=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.full((B, T, heads * D + gap), float("nan"), dtype=dtype)
    x[:, :, :heads * D] = torch.randn(B, T, heads * D, generator=g).to(dtype)
    return x.cuda()[:, :, :heads * D]


def _turned(x, pos, freq, interleaved):
    """x [B, T, heads, D] and the sum of absolute values that its pairs have, in 64 bits."""
    half = len(freq)
    t = pos.double()[..., None, None] * torch.tensor(freq, dtype=torch.float64, device=x.device)
    cos, sin = torch.cos(t), torch.sin(t)
    y, size = x.double(), torch.zeros_like(x, dtype=torch.float64)
    i = (torch.arange(0, 2 * half, 2), torch.arange(1, 2 * half, 2)) if interleaved else (torch.arange(half), torch.arange(half, 2 * half))
    a, b = y[..., i[0]].clone(), y[..., i[1]].clone()
    y[..., i[0]], y[..., i[1]] = a * cos - b * sin, b * cos + a * sin
    size[..., i[0]] = size[..., i[1]] = a.abs() + b.abs()
    return y, size


def _check_split(cache, Hq, H, qkv, start, counts, freq, interleaved, outs):
    """q, k, v as handed out against the formula; rows past the counts untouched (7)."""
    B, T, _ = qkv.shape
    x = qkv.reshape(B, T, Hq + 2 * H, D)
    pos = torch.tensor(start, device="cuda")[:, None] + torch.arange(T, device="cuda")
    y, size = _turned(x[:, :, :Hq + H], pos, freq, interleaved)
    half = 2.0 ** -8 if qkv.dtype == torch.bfloat16 else U
    for b in range(B):
        n = counts[b]
        for got, want, s in ((outs[0], y[:, :, :Hq], size[:, :, :Hq]), (outs[1], y[:, :, Hq:], size[:, :, Hq:]),
                             (outs[2], x[:, :, Hq + H:].double(), None)):
            g, w = got[b, :, :n].double(), want[b, :n].transpose(0, 1)
            assert (got[b, :, n:] == 7.0).all()
            if s is None:
                assert torch.equal(g, w)
            else:
                bad = (g - w).abs() > 6 * U * s[b, :n].transpose(0, 1) + half * w.abs()
                assert not bad.any(), (b, bad.nonzero()[:3].tolist(), float((g - w).abs().max()))


def _outs(B, Hq, H, T, dtype):
    return [torch.full((B, h, T, D), 7.0, dtype=dtype, device="cuda") for h in (Hq, H, H)]


def _same(a, b):
    """Two caches alike: every byte of their arenas but the work lists, which no append writes, and lengths and slots as reported."""
    torch.cuda.synchronize()
    assert torch.equal(a.arena, b.arena)
    assert (a.lengths(0) == b.lengths(0)).all()


FORMS = [dict(dtype=torch.bfloat16), dict(dtype=torch.bfloat16, page_tokens=32, pool_pages=200), dict(dtype=torch.bfloat16, kernel=rl.RLKV_KERNEL_VALU),
         dict(dtype=torch.float32)]
IDS = ["tiled", "paged", "rows", "f32"]


@pytest.mark.parametrize("form", FORMS, ids=IDS)
@pytest.mark.parametrize("Hq,H,pairs,interleaved", [(8, 2, 64, False), (4, 4, 64, True), (7, 1, 8, False), (12, 4, 48, True), (28, 4, 40, False),
                                                    (32, 8, 64, False)])
def test_ragged_chunks(form, Hq, H, pairs, interleaved):
    """Chunks of every kind onto full and compressed heads: nothing, one token, past the ring, over it more than once."""
    form = dict(form)
    dtype = form["dtype"]
    B, S, R, cap = 3, 5, 40, 600
    mask = [1, 0, 0, 1, 1, 0, 1, 0][:H]
    a, b = (_cache(Hq, H, B, S, R, mask=mask, cap=cap, **form) for _ in range(2))
    freq = _freq(pairs)
    rot = rl.Rotary(freq, interleaved=interleaved)
    start = [0] * B
    for i, counts in enumerate([(1, 0, 3), (33, 64, 2), (0, 1, 1), (50, 131, 7), (1, 1, 1), (200, 20, 310)]):
        T = max(counts) + (i % 2)
        qkv = _packed(B, T, Hq + 2 * H, dtype, 10 + i, gap=8 * (i % 3))
        outs = _outs(B, Hq, H, T, dtype)
        b.rotary(0, qkv, counts, rot, *outs)
        _check_split(b, Hq, H, qkv, start, counts, freq, interleaved, outs)
        b.append_ragged(0, outs[1], outs[2], counts)
        q = torch.full_like(outs[0], 7.0)
        a.append_rotary(0, qkv, counts, rot, q)
        assert torch.equal(q, outs[0])
        _same(a, b)
        start = [n + c for n, c in zip(start, counts)]
    for h in range(H):
        if not mask[h]:
            for s in range(B):
                assert (a.slot_positions(0, h, s) == b.slot_positions(0, h, s)).all()
    a.close(), b.close()


@pytest.mark.parametrize("form", FORMS, ids=IDS)
@pytest.mark.parametrize("T", [1, 5, 70])
def test_uniform_with_inactive_slots_and_decode(form, T):
    """Every active sequence by T tokens; steps of one token with the attention behind them, equal to the step in one call bit for bit."""
    form = dict(form)
    dtype = form["dtype"]
    Hq, H, B, S, R = 8, 2, 4, 4, 30
    a, b = (_cache(Hq, H, B, S, R, mask=[1, 0], cap=400, **form) for _ in range(2))
    rot = rl.Rotary(_freq(64))
    first = _packed(B, 9, Hq + 2 * H, dtype, 1)
    outs = _outs(B, Hq, H, 9, dtype)
    for c in (a, b):
        c.rotary(0, first, [9, 4, 1, 7], rot, *outs)
        c.append_rotary(0, first, [9, 4, 1, 7], rot)           # (queries not wanted)
        c.set_active([1, 0, 1, 1])
    qkv = _packed(B, T, Hq + 2 * H, dtype, 2)
    outs = _outs(B, Hq, H, T, dtype)
    b.rotary(0, qkv, None, rot, *outs)
    assert all((o[1] == 7.0).all() for o in outs)
    b.append(0, outs[1], outs[2])
    q = torch.full_like(outs[0], 7.0)
    a.append_rotary(0, qkv, None, rot, q)
    assert torch.equal(q, outs[0])
    _same(a, b)
    assert list(a.lengths(0)) == [9 + T, 4, 1 + T, 7 + T]
    for i in range(40):
        qkv = _packed(B, 1, Hq + 2 * H, dtype, 50 + i)
        outs = _outs(B, Hq, H, 1, dtype)
        b.rotary(0, qkv, None, rot, *outs)
        x, y = (torch.full((B, Hq, D), 3.0, dtype=dtype, device="cuda") for _ in range(2))
        b.append(0, outs[1], outs[2])
        b.decode_attention(0, outs[0][:, :, 0].contiguous(), x, D ** -0.5)
        q = torch.full((B, Hq, D), 7.0, dtype=dtype, device="cuda")
        a.append_rotary(0, qkv, None, rot, q)
        a.decode_attention(0, q, y, D ** -0.5)
        torch.cuda.synchronize()
        assert torch.equal(q, outs[0][:, :, 0]) and torch.equal(x, y) and (y[1] == 3.0).all()
    a.close(), b.close()


def test_against_the_oracle():
    """Attention over rotated keys against the CPU oracle on keys rotated in 64 bits."""
    import oracle
    from harness import to_np, tolerance

    Hq, H, B, S, R = 8, 2, 2, 4, 60
    c = _cache(Hq, H, B, S, R, torch.bfloat16, [1, 0], 200)
    freq, counts = _freq(64), [150, 90]
    rot = rl.Rotary(freq)
    qkv = _packed(B, 150, Hq + 2 * H, torch.bfloat16, 4)
    c.append_rotary(0, qkv, counts, rot)
    one = _packed(B, 1, Hq + 2 * H, torch.bfloat16, 5)
    q, out = (torch.empty(B, Hq, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    c.append_rotary(0, one, None, rot, q)
    c.decode_attention(0, q, out, D ** -0.5)
    pos = torch.arange(150, device="cuda").expand(B, 150)
    k = torch.zeros(B, H, 151, D, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    x, x1 = qkv.reshape(B, 150, -1, D), one.reshape(B, 1, -1, D)
    k[:, :, :150] = _turned(x[:, :, Hq:Hq + H], pos, freq, False)[0].bfloat16().transpose(1, 2)
    v[:, :, :150] = x[:, :, Hq + H:].transpose(1, 2)
    n = torch.tensor(counts, device="cuda")
    turned = _turned(x1[:, :, :Hq + H], n[:, None], freq, False)[0].bfloat16()
    for b in range(B):
        k[b, :, counts[b]], v[b, :, counts[b]] = turned[b, 0, Hq:], x1[b, 0, Hq + H:]
    ref = oracle.decode_attention(to_np(k), to_np(v), np.array(counts) + 1, [1, 0], to_np(turned[:, 0, :Hq].contiguous()), S, R, D ** -0.5)
    err = np.abs(out.float().cpu().numpy() - ref)
    assert (err <= tolerance(ref, rl.RLKV_BF16)).all(), err.max()
    c.close()


def test_far_positions():
    """12.6 million positions on, in single precision: angles are fractions of a turn at any position."""
    Hq, H, R, n = 2, 1, 16, 1 << 20
    c = _cache(Hq, H, 1, 4, R, torch.float32, [0], 1 << 24)
    k = torch.zeros(1, 1, n, D, device="cuda")
    for _ in range(12):
        c.append(0, k, k)
    del k
    at = [12 * n]
    for freq, interleaved in ((_freq(64), False), (_freq(64, 10000.0), True), ([1.0 + 0.37 * i for i in range(64)], False),
                              ([-0.5, 2 * math.pi, 7.0, 0.0, 1e-9, 1e6, -3e3, 0.1], False)):
        qkv = _packed(1, 3, Hq + 2 * H, torch.float32, 3)
        outs = _outs(1, Hq, H, 3, torch.float32)
        c.rotary(0, qkv, None, rl.Rotary(freq, interleaved=interleaved), *outs)
        # (the formula's own argument in 64 bits is off by 2^-53 of itself; 1e6 radians a position leave 2^-10 of it: not held to the tolerance)
        if max(abs(f) for f in freq) < 100:
            _check_split(c, Hq, H, qkv, at, [3], freq, interleaved, outs)
        assert all(torch.isfinite(o).all() for o in outs)
    c.close()


def test_many_sequences():
    """More sequences than counts that travel in a kernel's arguments."""
    Hq, H, B = 2, 2, 150
    a, b = (_cache(Hq, H, B, 2, 20, torch.bfloat16, [1, 0], 64) for _ in range(2))
    freq = _freq(64)
    rot = rl.Rotary(freq)
    counts = [i % 5 for i in range(B)]
    qkv = _packed(B, 4, Hq + 2 * H, torch.bfloat16, 6)
    outs = _outs(B, Hq, H, 4, torch.bfloat16)
    b.rotary(0, qkv, counts, rot, *outs)
    _check_split(b, Hq, H, qkv, [0] * B, counts, freq, False, outs)
    b.append_ragged(0, outs[1], outs[2], counts)
    q = torch.full_like(outs[0], 7.0)
    a.append_rotary(0, qkv, counts, rot, q)
    assert torch.equal(q, outs[0])
    _same(a, b)
    a.close(), b.close()


def test_unaligned_rows_and_wide_values():
    """Rows at any element; a V value beyond the fp16 range raises the layer's flag as the plain append does (the arenas agree)."""
    Hq, H, B, T = 4, 2, 2, 40
    a, b = (_cache(Hq, H, B, 4, 16, torch.bfloat16, [1, 0], 64, prefill_tokens=64) for _ in range(2))
    rot = rl.Rotary(_freq(32))
    width = (Hq + 2 * H) * D
    buf = torch.randn(B * T * (width + 3) + 1, device="cuda").bfloat16()
    qkv = buf[1:].view(B, T, width + 3)[:, :, :width]
    qkv[1, 5, -3] = 1e30
    qbuf = torch.full((B * Hq * T * D + 1,), 7.0, dtype=torch.bfloat16, device="cuda")
    outs = _outs(B, Hq, H, T, torch.bfloat16)
    b.rotary(0, qkv, [T, T], rot, *outs)
    _check_split(b, Hq, H, qkv, [0, 0], [T, T], _freq(32), False, outs)
    b.append_ragged(0, outs[1], outs[2], [T, 8])
    q = qbuf[1:].view(B, Hq, T, D)
    a.append_rotary(0, qkv, [T, 8], rot, q)
    assert torch.equal(q[0], outs[0][0]) and torch.equal(q[1, :, :8], outs[0][1, :, :8]) and (q[1, :, 8:] == 7.0).all()
    _same(a, b)
    a.close(), b.close()


def test_prompt_through_the_prefill():
    """Packed projections of a prompt through rotary and the prefill attention, then steps: the same cache as the append leaves."""
    Hq, H, B, T = 8, 2, 2, 96
    a, b = (_cache(Hq, H, B, 4, 30, torch.bfloat16, [1, 0], 200, prefill_tokens=T) for _ in range(2))
    rot = rl.Rotary(_freq(64))
    for i, counts in enumerate([(96, 50), (10, 96)]):
        qkv = _packed(B, T, Hq + 2 * H, torch.bfloat16, 20 + i)
        outs = _outs(B, Hq, H, T, torch.bfloat16)
        out = torch.empty_like(outs[0])
        a.rotary(0, qkv, counts, rot, *outs)
        a.prefill_attention(0, *outs, counts, out, D ** -0.5)
        b.append_rotary(0, qkv, counts, rot)
    x, y = (torch.empty(B, Hq, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    one = _packed(B, 1, Hq + 2 * H, torch.bfloat16, 30)
    q = torch.empty_like(x)
    for c, o in ((a, x), (b, y)):
        c.append_rotary(0, one, None, rot, q)
        c.decode_attention(0, q, o, D ** -0.5)
    torch.cuda.synchronize()
    assert torch.equal(x, y)
    a.close(), b.close()


def test_refusals():
    lib = rl.load_library()
    Hq, H, B = 4, 2, 2
    c = _cache(Hq, H, B, 4, 16, torch.bfloat16, [1, 0], 10)
    rot = rl.Rotary(_freq(64))
    T, width = 3, (Hq + 2 * H) * D
    qkv = torch.zeros(B, T, width, dtype=torch.bfloat16, device="cuda")
    q, k, v = _outs(B, Hq, H, T, torch.bfloat16)
    cnt = np.array([3, 1], dtype=np.int32)
    bad = rl.binding.RLKV_ERR_INVALID_ARG

    def append(layer=0, x=qkv.data_ptr(), stride=width, n=cnt.ctypes.data, t=T, r=rot.address, out=q.data_ptr()):
        return lib.rlkv_append_rotary(c.handle, layer, x, stride, n, t, r, out, None)

    def split(layer=0, x=qkv.data_ptr(), stride=width, n=cnt.ctypes.data, t=T, r=rot.address, out=q.data_ptr(), k=k.data_ptr(), v=v.data_ptr()):
        return lib.rlkv_rotary(c.handle, layer, x, stride, n, t, r, out, k, v, None)

    for call in (append, split):
        for over in (dict(layer=1), dict(layer=-1), dict(x=None), dict(stride=width - 1), dict(t=0), dict(t=-1), dict(r=None),
                     dict(x=qkv.data_ptr() + 1), dict(out=q.data_ptr() + 1), dict(t=2)):
            assert call(**over) == bad, over
        for freq, pairs in (([1.0] * 7, 7), ([1.0] * 12, 12), ([], 0), ([1.0] * 72, 72), ([float("nan")] * 8, 8), ([float("inf")] * 8, 8)):
            r = rl.Rotary(freq)
            assert call(r=r.address) == bad, freq
    for over in (dict(k=None), dict(v=None), dict(out=None), dict(k=k.data_ptr() + 1)):
        assert split(**over) == bad
    assert append(n=np.array([-1, 0], dtype=np.int32).ctypes.data) == bad
    assert list(c.lengths(0)) == [0, 0]
    many = torch.zeros(B, 11, width, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(rl.RlkvError) as e:
        c.append_rotary(0, many, None, rot)
    assert e.value.status == rl.binding.RLKV_ERR_CAPACITY and list(c.lengths(0)) == [0, 0]
    for call in (lambda: c.append_rotary(0, qkv.float(), None, rot), lambda: c.append_rotary(0, qkv[:, :, :-1], None, rot),
                 lambda: c.append_rotary(0, qkv[:1], None, rot), lambda: c.append_rotary(0, qkv.transpose(0, 1), None, rot),
                 lambda: c.append_rotary(0, qkv, [1], rot), lambda: c.append_rotary(0, qkv, None, rot, q[:, :, :1]),
                 lambda: c.rotary(0, qkv, None, rot, q, k, q)):
        with pytest.raises(ValueError):
            call()
    c.append_rotary(0, qkv, [0, 0], rot, q)
    assert (q == 7.0).all() and list(c.lengths(0)) == [0, 0]
    c.close()
