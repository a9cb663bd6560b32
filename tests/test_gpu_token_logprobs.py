"""Log probabilities, entropy, most likely tokens and their gradient against the formulas in 64 bits.

Tolerances, with X the largest |scale * logit| that is finite.  An exponent is off by the roundings of scale * log2(e), of the product
and of the maximum: 3 * 2^-24 X * 1.45, less than 6 * 2^-24 X.  A sum of n terms one after the other in a thread (64 of a chunk of 16384, then as many
again), and 20 joins, is off by (n + 40) * 2^-24 of itself with the exponentials' own rounding.  So lse by that and 6 * 2^-24 X; an
entropy, the difference of two such sums' functions neither of which is beyond H + 1, by twice as much of 1 + H.  A gradient's p is off by its
exponent's error: 12 * 2^-24 (X + 4) of itself, and so are the terms it multiplies.  bf16 gradients are rounded once more.
"""
import math

import pytest
import torch

import paper_2510_08525_amd as rl

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
CHUNK = 16384


def _logits(rows, vocab, dtype, seed, spread=3.0, pad=0, shift=0):
    g = torch.Generator().manual_seed(seed)
    buf = torch.full((rows * (vocab + pad) + shift,), float("nan"), dtype=dtype, device="cuda")
    x = buf[shift:].view(rows, vocab + pad)[:, :vocab]
    x.copy_((torch.randn(rows, vocab, generator=g) * spread).to(dtype))
    tokens = torch.randint(0, vocab, (rows,), generator=g, dtype=torch.int32).cuda()
    return x, tokens


def _wide(x, scale):
    z = x.double() * float(torch.tensor(scale, dtype=torch.float32))
    lp = torch.log_softmax(z, -1)
    p = lp.exp()
    entropy = torch.special.entr(p).sum(-1)
    empty = (z == -math.inf).all(-1)
    lp = torch.where(empty[:, None], -math.inf, lp)
    return z, lp, torch.where(empty, 0.0, entropy), torch.logsumexp(z, -1)


def _size(z):
    return torch.where(torch.isfinite(z), z.abs(), 0.0).amax(-1)


def _steps(vocab):
    return 64 * -(-vocab // CHUNK) + 40


def _near(got, want, tol):
    same = (got.double() - want).abs() <= tol
    same |= (got.double() == want) | (got.isnan() & want.isnan())
    assert same.all(), (int((~same).sum()), got[~same][:3].tolist(), want[~same][:3].tolist(), tol[~same][:3].tolist() if tol.dim() else tol)


def _run(x, tokens, scale=1.0, k=0, **kw):
    R = x.shape[0]
    nan = lambda *s: torch.full(s, float("nan"), device="cuda")               # noqa: E731
    lp, h, lse = nan(R), nan(R), nan(R)
    top = (nan(R, k), torch.full((R, k), -9, dtype=torch.int32, device="cuda")) if k else None
    assert rl.token_logprobs(x, tokens, lp, scale=scale, entropy=h, lse=lse, top=top, **kw) is lp
    return lp, h, lse, top


def _check(x, tokens, scale, got):
    z, lp, entropy, lse = _wide(x, scale)
    X, n, V = _size(z), _steps(x.shape[1]), x.shape[1]
    asked = (tokens >= 0) & (tokens < V)
    want = torch.where(asked, lp.gather(1, tokens.long().clamp(0, V - 1)[:, None])[:, 0], 0.0)
    tol = n * U + 6 * U * X
    _near(got[0], want, tol + U * want.abs())
    _near(got[1], entropy, 2 * (1 + entropy) * n * U + 12 * U * X)
    _near(got[2], lse, tol + U * lse.abs())
    if got[3] is not None:
        k = got[3][0].shape[1]
        v, i = torch.sort(z, dim=-1, descending=True, stable=True)
        assert torch.equal(got[3][1].long(), i[:, :k])
        best = lp.gather(1, i[:, :k])
        _near(got[3][0], best, (tol[:, None] + U * best.abs()))


# one token, a piece, the ends of a chunk and of the rows, few rows (split and joined) and many (not)
@pytest.mark.parametrize("rows,vocab,k", [(1, 1, 1), (2, 7, 7), (3, 8, 0), (1, 100, 5), (5, 1000, 20), (2, 16384, 1), (3, 16385, 32), (1, 32768, 4),
                                          (4, 50257, 32), (1, 131072, 20), (2, 300001, 7), (1030, 33, 3), (1500, 515, 0), (1100, 20000, 8),
                                          (7, 128011, 0), (300, 40000, 32), (1024, 16390, 2)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("scale", [1.0, 0.7])
def test_rows(rows, vocab, k, dtype, scale):
    """bf16 logits of large vocabularies are full of equal values: the lists hold the lowest tokens of those."""
    x, tokens = _logits(rows, vocab, dtype, rows + vocab)
    if rows > 2:
        tokens[1], tokens[2] = -1, vocab
    _check(x, tokens, scale, _run(x, tokens, scale, k))


@pytest.mark.parametrize("vocab,pad,shift", [(1000, 8, 0), (1000, 3, 0), (16384, 0, 1), (40001, 7, 5)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strides(vocab, pad, shift, dtype):
    """Rows apart and at any element, with NaN between them."""
    x, tokens = _logits(5, vocab, dtype, 3, pad=pad, shift=shift)
    _check(x, tokens, 1.0, _run(x, tokens, 1.0, 6))


@pytest.mark.parametrize("order", ["up", "down", "equal", "two"])
@pytest.mark.parametrize("rows", [2, 1025])
def test_hard_lists(order, rows):
    """Rows that let every logit, or none after the first chunk, through to the list: ascending, descending, all equal, two values."""
    V, k = 33000, 32
    ramp = torch.arange(V, dtype=torch.float32, device="cuda") / 4096
    row = {"up": ramp, "down": -ramp, "equal": torch.full_like(ramp, 2.5), "two": (torch.arange(V, device="cuda") % 20 == 7).float()}[order]
    x = row.expand(rows, V).contiguous()
    tokens = torch.zeros(rows, dtype=torch.int32, device="cuda")
    _check(x, tokens, 1.0, _run(x, tokens, 1.0, k))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [50, 40000])
@pytest.mark.parametrize("low", [-math.inf, "lowest"])
def test_masks(dtype, vocab, low):
    """Masked logits, by -inf and by the type's lowest value: most of a row, all but one, all; fewer allowed tokens than the list is long."""
    low = torch.finfo(dtype).min if low == "lowest" else low
    x, tokens = _logits(6, vocab, dtype, 8)
    x[0, torch.rand(vocab, device="cuda") < 0.9] = low
    x[1, :] = low
    x[1, 17] = 4.0
    x[2, :] = low
    x[3, 3:] = low
    x[4, : vocab - 1] = low
    tokens[1], tokens[2] = 17, 5
    got = _run(x, tokens, 1.0, 8)
    if low == -math.inf:
        _check(x, tokens, 1.0, got)
        assert got[0][2] == -math.inf and got[1][2] == 0 and got[2][2] == -math.inf and got[3][1][2].tolist() == list(range(8))
    else:
        # (X is the lowest value of the type where it is allowed to count: the tolerance is taken from the others)
        z, lp, entropy, lse = _wide(x, 1.0)
        keep = [0, 1, 3, 4, 5]
        X = torch.where(z > -1e30, z.abs(), 0.0).amax(-1)[keep]
        n = _steps(vocab)
        _near(got[1][keep], entropy[keep], 2 * (1 + entropy[keep]) * n * U + 12 * U * X)
        _near(got[2][keep], lse[keep], n * U + 6 * U * X + U * lse[keep].abs())
        i = torch.sort(x.double(), dim=-1, descending=True, stable=True).indices[:, :8]
        assert torch.equal(got[3][1].long(), i)
        assert abs(float(got[1][2]) - math.log(vocab)) <= 2 * (1 + math.log(vocab)) * n * U     # all equal: the uniform distribution


def test_infinities_and_nan():
    x, tokens = _logits(4, 20000, torch.float32, 9)
    x[0, 777] = math.inf
    x[1, 19999] = math.nan
    x[2, :] = math.nan
    lp, h, lse, (v, i) = _run(x, tokens, 1.0, 3)
    for r in range(3):
        assert lp[r].isnan() and h[r].isnan() and lse[r].isnan() and v[r].isnan().all()
    assert i[0, 0] == 777 and i[1, 0] == 19999 and i[2].tolist() == [0, 1, 2]
    _check(x[3:], tokens[3:], 1.0, (lp[3:], h[3:], lse[3:], (v[3:], i[3:])))


def test_large_logits():
    """Differences of logits near 10^4: exponents are taken from the maximum."""
    x, tokens = _logits(3, 5000, torch.float32, 10, spread=1e4)
    _check(x, tokens, 1.0, _run(x, tokens, 1.0, 4))


def test_only_what_is_asked_for():
    x, tokens = _logits(3, 40000, torch.bfloat16, 12)
    lse = torch.empty(3, device="cuda")
    assert rl.token_logprobs(x, None, None, lse=lse) is None
    _near(lse, _wide(x, 1.0)[3], _steps(40000) * U + 6 * U * _size(x.double()) + 1e-6)
    assert rl.token_logprobs(x[:0], tokens[:0], lse[:0]).numel() == 0


def _grad_wide(x, tokens, scale, g, gh):
    z, lp, entropy, lse = _wide(x, scale)
    p = lp.exp()
    V = x.shape[1]
    asked = (tokens >= 0) & (tokens < V) & torch.isfinite(lse)
    g = torch.where(asked, g.double(), 0.0)
    part = torch.where(p > 0, lp, 0.0) + entropy[:, None]
    d = -p * (g[:, None] + gh.double()[:, None] * part)
    d[torch.arange(len(g)), tokens.long().clamp(0, V - 1)] += g
    size = p * (g.abs()[:, None] + gh.double().abs()[:, None] * (1 + part.abs() + entropy[:, None]))
    hot = torch.zeros_like(p)
    hot[torch.arange(len(g)), tokens.long().clamp(0, V - 1)] = g.abs()
    return scale * d, scale * (12 * U * (_size(z)[:, None] + 4) * size + 2 * U * hot), entropy, lse


def _check_grad(out, want, tol, dtype):
    half = 2.0 ** -8 if dtype == torch.bfloat16 else U
    _near(out, want, tol + half * want.abs() + 1e-37)


@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 7), (2, 8), (4, 1000), (1, 131072), (70, 16385), (2, 300001), (1500, 515)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("pad,shift", [(0, 0), (5, 1)])
def test_gradient(rows, vocab, dtype, pad, shift):
    scale = 0.7
    x, tokens = _logits(rows, vocab, dtype, 40 + vocab, pad=pad, shift=shift)
    if rows > 2:
        tokens[0], tokens[2] = -1, vocab + 5
        x[1, : vocab // 2] = -math.inf
    g, gh = torch.randn(rows, device="cuda"), torch.randn(rows, device="cuda")
    want, tol, entropy, lse = _grad_wide(x, tokens, float(torch.tensor(scale)), g, gh)
    h32, l32 = entropy.float(), lse.float()
    buf = torch.full((rows * (vocab + pad) + shift,), 7.0, dtype=dtype, device="cuda")
    out = buf[shift:].view(rows, vocab + pad)[:, :vocab]
    assert rl.token_logprobs_grad(x, tokens, l32, g, out, scale=scale, entropy=h32, grad_entropy=gh) is out
    _check_grad(out, want, tol, dtype)
    if pad:
        assert (buf[shift:].view(rows, vocab + pad)[:, vocab:] == 7.0).all()
    # each kind alone, and over the logits themselves
    zero = torch.zeros_like(g)
    w, t, _, _ = _grad_wide(x, tokens, float(torch.tensor(scale)), g, zero)
    rl.token_logprobs_grad(x, tokens, l32, g, out, scale=scale)
    _check_grad(out, w, t, dtype)
    w, t, _, _ = _grad_wide(x, tokens, float(torch.tensor(scale)), zero, gh)
    rl.token_logprobs_grad(x, None, l32, None, x, scale=scale, entropy=h32, grad_entropy=gh)
    _check_grad(x, w, t, dtype)


def test_gradient_of_empty_rows_is_zero():
    x = torch.full((2, 300), -math.inf, device="cuda")
    x[1, 4] = 1.0
    tokens = torch.tensor([3, 4], dtype=torch.int32, device="cuda")
    lp, h, lse, _ = _run(x, tokens)
    out = torch.empty_like(x)
    one = torch.ones(2, device="cuda")
    rl.token_logprobs_grad(x, tokens, lse, one, out, entropy=h, grad_entropy=one)
    assert (out == 0).all()


def test_gradient_against_differences():
    """Central differences of the formulas in 64 bits; the step's own error is below 1e-8."""
    x, tokens = _logits(3, 40, torch.float32, 77)
    g, gh = torch.randn(3, device="cuda"), torch.randn(3, device="cuda")
    lp, h, lse, _ = _run(x, tokens, 0.7)
    out = torch.empty_like(x)
    rl.token_logprobs_grad(x, tokens, lse, g, out, scale=0.7, entropy=h, grad_entropy=gh)

    def value(z):
        l = torch.log_softmax(z * float(torch.tensor(0.7)), -1)
        return (g.double() * l.gather(1, tokens.long()[:, None])[:, 0] - gh.double() * (l.exp() * l).sum(-1)).sum()

    step, z = 1e-5, x.double()
    for r in range(3):
        for i in range(0, 40, 3):
            e = torch.zeros_like(z)
            e[r, i] = step
            d = (value(z + e) - value(z - e)) / (2 * step)
            assert abs(float(d - out[r, i])) < 1e-5 * (1 + abs(float(d)))


def test_equal_bits_stream_and_graph():
    """Splits are joined in a fixed order; on a stream of its own; recorded and replayed on other logits."""
    x, tokens = _logits(5, 100000, torch.bfloat16, 30)
    ws = torch.full((rl.rlkv_token_logprobs_workspace(5, 100000, 9),), 255, dtype=torch.uint8, device="cuda")
    assert ws.numel() > 0
    a = _run(x, tokens, 1.0, 9, workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b = _run(x, tokens, 1.0, 9)
    side.synchronize()
    for u, v in zip(a[:3] + a[3], b[:3] + b[3]):
        assert torch.equal(u, v)
    out = torch.empty_like(x)
    g = torch.ones(5, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rl.token_logprobs(x, tokens, a[0], entropy=a[1], lse=a[2], top=a[3], workspace=ws)
        rl.token_logprobs_grad(x, tokens, a[2], g, out, entropy=a[1], grad_entropy=g)
    for seed in range(3):
        x.copy_(_logits(5, 100000, torch.bfloat16, 31 + seed)[0])
        graph.replay()
        torch.cuda.synchronize()
        _check(x, tokens, 1.0, a)
        want, tol, _, _ = _grad_wide(x, tokens, 1.0, g, g)
        _check_grad(out, want, tol + 4 * _steps(100000) * U * want.abs() + 60 * U * torch.softmax(x.double(), -1) * _steps(100000), torch.bfloat16)


def test_tensor_checks():
    x, tokens = _logits(4, 100, torch.bfloat16, 1)
    f = torch.empty(4, device="cuda")
    top = (torch.empty(4, 3, device="cuda"), torch.empty(4, 3, dtype=torch.int32, device="cuda"))
    for bad in (lambda: rl.token_logprobs(x.half(), tokens, f), lambda: rl.token_logprobs(x, tokens.long(), f),
                lambda: rl.token_logprobs(x, tokens[:3], f), lambda: rl.token_logprobs(x, tokens, f.double()),
                lambda: rl.token_logprobs(x.t(), tokens, f), lambda: rl.token_logprobs(x, tokens, f, top=(top[0], top[1].long())),
                lambda: rl.token_logprobs(x, tokens, f, top=(top[0][:2], top[1])), lambda: rl.token_logprobs(x, tokens, f.cpu()),
                lambda: rl.token_logprobs(x, tokens, f, top=tuple(t.t().contiguous().t() for t in top)),
                lambda: rl.token_logprobs_grad(x, tokens, f, f, x.float()), lambda: rl.token_logprobs_grad(x, tokens, f[:2], f, x.clone())):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: rl.token_logprobs(x, tokens, None), lambda: rl.token_logprobs(x, tokens, f, scale=0.0),
                lambda: rl.token_logprobs(x, tokens, f, scale=-1.0), lambda: rl.token_logprobs(x[:, :2], tokens, f, top=top),
                lambda: rl.token_logprobs_grad(x, tokens, f, None, x.clone()), lambda: rl.token_logprobs_grad(x, tokens, f, f, x.clone(), entropy=f),
                lambda: rl.token_logprobs(_logits(4, 100000, torch.bfloat16, 1)[0], tokens, f, workspace=torch.empty(1, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(rl.RlkvError):
            bad()
