"""Norm of heads with rotation, and its gradient, against 64 bits.

Tolerances: a value passes through some 20 fp32 operations (the sum of 128 squares among them as a tree of 16 and 8), each off by 2^-24 of what
it works on: 2^-19 of (|a| + |b|) for a pair (a, b) that turns together, as with the rotation alone, and the output's rounding (2^-8 of it in bf16, 2^-24 in fp32).
The gradient subtracts u mean(g w u) from g w: 2^-19 of the sum of both sizes.  A weight's gradient adds up at most 512 rows one behind the other in
fp32 before it goes on in trees and 64 bits: 2^-15 of the sum of sizes."""
import pytest
import torch

import paper_2510_08525_amd as rl

pytestmark = pytest.mark.gpu
D = 128
F32, BF16 = torch.float32, torch.bfloat16
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}
IN, SUM = 2.0 ** -19, 2.0 ** -15


def freq(pairs):
    return [500000.0 ** (-i / pairs) for i in range(pairs)]


def columns(pairs, interleaved):
    half = torch.arange(pairs)
    return (2 * half, 2 * half + 1) if interleaved else (half, half + pairs)


def turned(x, pos, pairs, interleaved, back=False):
    """x [T, heads, D] in 64 bits."""
    if not pairs:
        return x
    t = pos.double()[:, None, None] * torch.tensor(freq(pairs), dtype=torch.float64)
    i, j = columns(pairs, interleaved)
    y, s = x.clone(), torch.sin(-t if back else t)
    y[..., i], y[..., j] = x[..., i] * torch.cos(t) - x[..., j] * s, x[..., j] * torch.cos(t) + x[..., i] * s
    return y


def sizes(x, pairs, interleaved):
    """|a| + |b| in both columns of a pair, |x| in the others."""
    y = x.abs().clone()
    if pairs:
        i, j = columns(pairs, interleaved)
        y[..., i] = y[..., j] = x[..., i].abs() + x[..., j].abs()
    return y


def make(T, Hq, H, dtype, norm, seed=0, positions=None):
    g = torch.Generator().manual_seed(seed)
    qkv = (torch.randn(T, (Hq + 2 * H) * D, generator=g) * 2).to(dtype)
    pos = torch.randint(0, 100000, (T,), generator=g, dtype=torch.int32) if positions is None else torch.tensor(positions, dtype=torch.int32)
    w = [(1 + 0.3 * torch.randn(D, generator=g)).to(dtype) if norm == "weights" else None for _ in range(2)]
    grads = [torch.randn(T, h, D, generator=g).to(dtype) for h in (Hq, H, H)]
    return qkv, pos, w, grads


def rotary(pairs, interleaved):
    return rl.Rotary(freq(pairs), interleaved=interleaved) if pairs else None


def cuda(t):
    return None if t is None else t.cuda()


CASES = [(1, 1, 1), (1, 32, 8), (5, 3, 1), (33, 28, 4), (301, 7, 7), (2100, 28, 4)]
HOW = [("weights", 64, False), ("ones", 32, True), (None, 64, True), ("weights", 8, False), ("weights", 0, False), (None, 0, False), ("weights", 48, True)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T, Hq, H", CASES)
@pytest.mark.parametrize("norm, pairs, interleaved", HOW)
def test_forward(T, Hq, H, norm, pairs, interleaved, dtype):
    qkv, pos, w, _ = make(T, Hq, H, dtype, norm)
    eps = None if norm is None else 1e-3
    outs = [torch.full((T, h, D), 7.0, dtype=dtype, device="cuda") for h in (Hq, H, H)]
    rl.head_norm_rotary(qkv.cuda(), pos.cuda() if pairs else None, rotary(pairs, interleaved), outs[0], outs[1], v_out=outs[2], q_weight=cuda(w[0]),
                        k_weight=cuda(w[1]), eps=eps)
    x = qkv.double().view(T, -1, D)
    for out, part, weight in zip(outs, (x[:, :Hq], x[:, Hq:Hq + H]), w):
        if norm:
            part = part / torch.sqrt(part.square().mean(-1, keepdim=True) + eps) * (1 if weight is None else weight.double())
        want = turned(part, pos, pairs, interleaved)
        assert ((out.double().cpu() - want).abs() <= IN * sizes(part, pairs, interleaved) + HALF[dtype] * want.abs()).all()
    assert torch.equal(outs[2].cpu().double(), x[:, Hq + H:])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T, Hq, H", CASES)
@pytest.mark.parametrize("norm, pairs, interleaved", HOW)
def test_gradient(T, Hq, H, norm, pairs, interleaved, dtype):
    qkv, pos, w, grads = make(T, Hq, H, dtype, norm, 1)
    eps = None if norm is None else 1e-3
    values = T % 2 == 1
    out = torch.full((T, (Hq + 2 * H) * D), 7.0, dtype=dtype, device="cuda")
    gw = [torch.full((D,), 7.0, device="cuda") if norm else None for _ in range(2)]
    rl.head_norm_rotary_grad(qkv.cuda(), pos.cuda() if pairs else None, rotary(pairs, interleaved), grads[0].cuda(), grads[1].cuda(), out,
                             grad_v=grads[2].cuda() if values else None, q_weight=cuda(w[0]), k_weight=cuda(w[1]), eps=eps,
                             grad_q_weight=gw[0], grad_k_weight=gw[1])
    x, got = qkv.double().view(T, -1, D), out.double().cpu().view(T, -1, D)
    for part, grad, weight, grad_w, have in zip((x[:, :Hq], x[:, Hq:Hq + H]), grads, w, gw, (got[:, :Hq], got[:, Hq:Hq + H])):
        g = turned(grad.double(), pos, pairs, interleaved, back=True)
        size = sizes(grad.double(), pairs, interleaved)
        if norm:
            r = 1 / torch.sqrt(part.square().mean(-1, keepdim=True) + eps)
            u, ww = part * r, torch.ones(D, dtype=torch.float64) if weight is None else weight.double()
            want_w = (g * u).sum((0, 1))
            assert ((grad_w.double().cpu() - want_w).abs() <= SUM * (size * u.abs()).sum((0, 1))).all()
            g, size = r * (g * ww - u * (g * ww * u).mean(-1, keepdim=True)), \
                r * (size * ww.abs() + 2 * u.abs() * (size * ww.abs() * u.abs()).mean(-1, keepdim=True))
        assert ((have - g).abs() <= IN * size + HALF[dtype] * g.abs()).all()
    assert torch.equal(got[:, Hq + H:], grads[2].double()) if values else (got[:, Hq + H:] == 7).all()


def test_gradient_against_differences():
    T, Hq, H = 6, 3, 2
    qkv, pos, w, grads = make(T, Hq, H, F32, "weights", 2)
    out, gw = torch.zeros(T, (Hq + 2 * H) * D, device="cuda"), [torch.zeros(D, device="cuda") for _ in range(2)]
    rl.head_norm_rotary_grad(qkv.cuda(), pos.cuda(), rotary(64, False), grads[0].cuda(), grads[1].cuda(), out, q_weight=cuda(w[0]),
                             k_weight=cuda(w[1]), eps=1e-3, grad_q_weight=gw[0], grad_k_weight=gw[1])

    def f(x, wq, wk):
        x = x.view(T, -1, D)
        total = 0
        for part, weight, g in zip((x[:, :Hq], x[:, Hq:Hq + H]), (wq, wk), grads):
            total = total + (turned(part / torch.sqrt(part.square().mean(-1, keepdim=True) + 1e-3) * weight, pos, 64, False) * g.double()).sum()
        return total

    g = torch.Generator().manual_seed(3)
    at = [qkv.double(), w[0].double(), w[1].double()]
    for i, got in enumerate((out, *gw)):
        way = torch.randn(at[i].shape, generator=g).double()
        step = lambda s: f(*(t + s * way if k == i else t for k, t in enumerate(at)))            # noqa: E731
        slope = (step(1e-4) - step(-1e-4)) / 2e-4
        have = (got.double().cpu() * way).sum()
        # differences: their own square is 1e-8 of third derivatives of size 1; the gradient: 2^-15 of the sum of sizes
        assert abs(have - slope) <= 2.0 ** -15 * (got.double().cpu() * way).abs().sum() + 1e-5 * abs(slope)


@pytest.mark.parametrize("positions", [[0, -1, -100000, 2 ** 31 - 1, -(2 ** 31)]])
def test_positions_of_any_sign(positions):
    qkv, pos, _, grads = make(5, 2, 1, F32, None, 4, positions)
    q, k = torch.zeros(5, 2, D, device="cuda"), torch.zeros(5, 1, D, device="cuda")
    rl.head_norm_rotary(qkv.cuda(), pos.cuda(), rotary(64, False), q, k)
    x = qkv.double().view(5, -1, D)
    # (at 2^31 the reference's own angle, a product of 64-bit floats, is off by 2^31 * 2^-53 = 2^-22; so is the library's fraction of a turn)
    want = turned(x[:, :2], pos, 64, False)
    assert ((q.double().cpu() - want).abs() <= (IN + 2.0 ** -20) * sizes(x[:, :2], 64, False)).all()
    back = torch.zeros(5, 4 * D, device="cuda")
    rl.head_norm_rotary_grad(qkv.cuda(), pos.cuda(), rotary(64, False), q, k, back)
    assert torch.allclose(back[:, :3 * D].cpu(), qkv[:, :3 * D], atol=1e-5)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strides_and_in_place(dtype):
    T, Hq, H = 37, 4, 2
    qkv, pos, w, grads = make(T, Hq, H, dtype, "weights", 5)
    wide = torch.full((T, 8 * D + 24), 7.0, dtype=dtype, device="cuda")
    wide[:, 3:3 + 8 * D] = qkv.cuda()
    x = wide[:, 3:3 + 8 * D]                                                     # rows at any element
    r, how = rotary(64, False), dict(q_weight=w[0].cuda(), k_weight=w[1].cuda(), eps=1e-6)
    q, k, v = (torch.zeros(T, h, D, dtype=dtype, device="cuda") for h in (Hq, H, H))
    rl.head_norm_rotary(qkv.cuda(), pos.cuda(), r, q, k, v_out=v, **how)
    front = [torch.zeros(h, T, D, dtype=dtype, device="cuda").transpose(0, 1) for h in (Hq, H, H)]
    rl.head_norm_rotary(x, pos.cuda(), r, front[0], front[1], v_out=front[2], **how)
    assert all(torch.equal(a, b) for a, b in zip(front, (q, k, v)))
    place = qkv.cuda().clone()
    rl.head_norm_rotary(place, pos.cuda(), r, place[:, :4 * D].view(T, 4, D), place[:, 4 * D:6 * D].view(T, 2, D), **how)
    assert torch.equal(place, torch.cat([q.view(T, -1), k.view(T, -1), qkv[:, 6 * D:].cuda()], 1))
    want = torch.full((T, 8 * D), 7.0, dtype=dtype, device="cuda")
    gw = torch.zeros(D, device="cuda")
    rl.head_norm_rotary_grad(x, pos.cuda(), r, grads[0].cuda(), grads[1].cuda(), want, grad_k_weight=gw, **how)
    same = torch.cat([t.reshape(T, -1) for t in grads], 1).cuda()
    same[:, 6 * D:] = 7
    rl.head_norm_rotary_grad(x, pos.cuda(), r, same[:, :4 * D].view(T, 4, D), same[:, 4 * D:6 * D].view(T, 2, D), same, **how)
    assert torch.equal(same, want)


def test_weights_gradients_of_no_tokens_are_zero():
    e = torch.zeros(0, 4 * D, device="cuda")
    gw = [torch.full((D,), 7.0, device="cuda") for _ in range(2)]
    rl.head_norm_rotary_grad(e, None, None, e.view(0, 4, D)[:, :2], e.view(0, 4, D)[:, 2:3], e, eps=1e-6, grad_q_weight=gw[0], grad_k_weight=gw[1])
    assert all((t == 0).all() for t in gw)


def test_not_finite_rows_stay_rows():
    """A NaN or an infinity of one head changes that head alone."""
    qkv, pos, w, _ = make(9, 3, 1, BF16, "weights", 6)
    outs = [[torch.zeros(9, h, D, dtype=BF16, device="cuda") for h in (3, 1)] for _ in range(2)]
    for out, x in zip(outs, (qkv, qkv.clone())):
        if out is outs[1]:
            x[4, D + 5], x[7, 3 * D + 1] = float("nan"), float("inf")
        rl.head_norm_rotary(x.cuda(), pos.cuda(), rotary(64, False), *out, q_weight=w[0].cuda(), k_weight=w[1].cuda(), eps=1e-6)
    same_q, same_k = torch.ones(9, 3, dtype=torch.bool), torch.ones(9, 1, dtype=torch.bool)
    same_q[4, 1], same_k[7, 0] = False, False
    for i, same in enumerate((same_q, same_k)):
        assert torch.equal(outs[0][i].cpu()[same], outs[1][i].cpu()[same])
        assert outs[1][i].cpu()[~same].isnan().any()


def test_recorded_calls():
    T, Hq, H = 70, 4, 2
    qkv, pos, w, grads = make(T, Hq, H, BF16, "weights", 7)
    qkv, pos, r = qkv.cuda(), pos.cuda(), rotary(64, False)
    how = dict(q_weight=w[0].cuda(), k_weight=w[1].cuda(), eps=1e-6)
    q, k = (torch.zeros(T, h, D, dtype=BF16, device="cuda") for h in (Hq, H))
    back, gw = torch.zeros(T, 8 * D, dtype=BF16, device="cuda"), [torch.zeros(D, device="cuda") for _ in range(2)]
    work = torch.zeros(rl.rlkv_head_norm_rotary_grad_workspace(T, Hq, H), dtype=torch.uint8, device="cuda")

    def call():
        rl.head_norm_rotary(qkv, pos, r, q, k, **how)
        rl.head_norm_rotary_grad(qkv, pos, r, q, k, back, grad_q_weight=gw[0], grad_k_weight=gw[1], workspace=work, **how)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(3):
        pos += 11
        work.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (q, k, back, *gw)]
        call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (q, k, back, *gw)))


def test_one_token_goes_into_the_fused_step():
    """Decode steps of a layer with normed heads: head_norm_rotary hands out what append_decode takes; the same through the packed attention."""
    B, Hq, H, steps = 2, 4, 2, 5
    cache = rl.Cache(1, Hq, H, D, B, 4, 60, rl.RLKV_BF16, [[1, 0]], [64] * B)
    r, how = rotary(64, False), dict(eps=1e-6)
    x = torch.randn(steps, B, 8 * D, generator=torch.Generator().manual_seed(8)).to(BF16).cuda()
    outs = []
    for t in range(steps):
        q, k, v = (torch.zeros(B, h, D, dtype=BF16, device="cuda") for h in (Hq, H, H))
        rl.head_norm_rotary(x[t], torch.full((B,), t, dtype=torch.int32, device="cuda"), r, q, k, v_out=v, **how)
        out = torch.zeros(B, Hq, D, dtype=BF16, device="cuda")
        cache.append_decode(0, k.view(B, H, 1, D), v.view(B, H, 1, D), q, out, D ** -0.5)
        outs.append(out)
    packed = x.transpose(0, 1).reshape(B * steps, -1)
    pos = torch.arange(steps, dtype=torch.int32, device="cuda").repeat(B)
    q, k = (torch.zeros(B * steps, h, D, dtype=BF16, device="cuda") for h in (Hq, H))
    rl.head_norm_rotary(packed, pos, r, q, k, **how)
    out = torch.zeros_like(q)
    offsets = torch.arange(B + 1, dtype=torch.int32, device="cuda") * steps
    rl.packed_attention(q, k, packed[:, 6 * D:].view(B * steps, H, D), offsets, out, D ** -0.5, mask=[1, 0], sink=4, recent=60)
    # both round their output (2^-8), and this one its weights besides: 2^-8 of sum w |v| / l <= max |v| < 5
    assert torch.allclose(torch.stack(outs, 1).view(B * steps, Hq, D).float(), out.float(), rtol=2.0 ** -7, atol=5 * 2.0 ** -8)
