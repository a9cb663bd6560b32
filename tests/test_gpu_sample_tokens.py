"""Tokens drawn by given random numbers, against the definition in 64 bits.

Weights are off by 2^-38 of themselves (the exponential) and, as whole numbers of 2^-b, b = min(50, 62 - log2(vocab)), by 2^-(b + 1): a border between two
tokens lies within 2^-37 + vocab * 2^-b of the sum of weights (at least 1) of where 64 bits have it.  The reference names the token, and its neighbour
where u lies that close to a border (and the cut by top_p its own neighbours)."""
import math

import pytest
import torch

import paper_2510_08525_amd as rl

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def weights(x, T):
    z = (x.double() - x.double().max()) / T
    return torch.where(x == -math.inf, 0.0, torch.exp(z))


def kept(x, T, k, p, m):
    """Truth values [vocab], T > 0."""
    n = x.numel()
    order = torch.sort(x, descending=True, stable=True).indices
    w = weights(x, T)[order]
    keep = torch.arange(n) < (k if k > 0 else n)
    if p < 1:
        cum = torch.cumsum(torch.where(keep, w, 0.0), 0)
        keep &= (cum - torch.where(keep, w, 0.0) < p * cum[-1]) | (torch.arange(n) == 0)
    keep &= (w >= m) | (torch.arange(n) == 0)
    return torch.zeros(n, dtype=torch.bool).scatter(0, order, keep)


def draw(x, u, T, k, p, m):
    """(token, log probability, whether u is farther than the bound from a border)"""
    if T <= 0:
        return int((x == x.max()).nonzero()[0]), 0.0, True
    w = torch.where(kept(x, T, k, p, m), weights(x, T), 0.0)
    cum = torch.cumsum(w, 0)
    i = int((cum <= u * cum[-1]).sum())
    i = min(i, int(w.nonzero()[-1]))
    bits = min(50, 62 - math.ceil(math.log2(x.numel()))) if x.numel() > 1 else 50
    near = (cum / cum[-1] - u).abs().min() < 2.0 ** -37 + x.numel() * 2.0 ** -bits
    exact = (w[w > 0] == 1).all()                  # (equal logits: weights of 1 and their sums are whole numbers on both sides, borders the same)
    return i, math.log(w[i] / cum[-1]), bool(exact or not near)


def call(x, u, **how):
    rows = x.shape[0]
    tokens = torch.full((rows,), -7, dtype=torch.int32, device="cuda")
    logprobs = torch.full((rows,), 7.0, device="cuda")
    rl.sample_tokens(x, u, tokens, logprobs=logprobs, **how)
    torch.cuda.synchronize()
    return tokens.cpu(), logprobs.cpu()


def check(x, u, T=1.0, k=0, p=1.0, m=0.0):
    rows = x.shape[0]
    row = lambda v, r: v[r].item() if torch.is_tensor(v) else v                # noqa: E731
    cuda = lambda v: v.cuda() if torch.is_tensor(v) else v                     # noqa: E731
    tokens, logprobs = call(x.cuda(), u.cuda(), temperature=cuda(T), top_k=cuda(k), top_p=cuda(p), min_p=cuda(m))
    sure = 0
    for r in range(rows):
        token, logprob, far = draw(x[r], u[r].item(), row(T, r), row(k, r), row(p, r), row(m, r))
        if far:
            sure += 1
            assert tokens[r] == token, r
            # 64-bit logarithms of sums that are off by vocab * 2^-b, rounded to fp32
            assert abs(logprobs[r].double() - logprob) <= 2.0 ** -24 * abs(logprob) + 1e-9, r
    assert sure >= rows - 1 - rows // 50


def logits(rows, vocab, dtype, seed=0, spread=3.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(rows, vocab, generator=g) * spread).to(dtype), torch.rand(rows, generator=g)


FILTERS = [dict(), dict(T=0.7), dict(k=1), dict(k=50), dict(p=0.9), dict(p=0.5, T=1.5), dict(m=0.1), dict(k=40, p=0.8, m=0.02, T=0.6), dict(T=0.0, k=5),
           dict(p=0.0), dict(m=1.0), dict(k=10 ** 6), dict(T=100.0), dict(T=1e-3), dict(T=100.0, p=0.37, k=700)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("how", FILTERS)
@pytest.mark.parametrize("vocab", [1, 7, 1000, 8193, 50257])
def test_filters(vocab, how, dtype):
    x, u = logits(20, vocab, dtype, vocab)
    check(x, u, **how)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab, spread", [(131072, 3.0), (131072, 0.01), (200001, 30.0)])
def test_large_vocabularies(vocab, spread, dtype):
    x, u = logits(6, vocab, dtype, 1, spread)
    for how in (dict(), dict(p=0.95), dict(k=1000, p=0.5), dict(m=0.5), dict(k=vocab - 1)):
        check(x, u, **how)


def test_a_setting_for_each_row():
    x, u = logits(64, 3001, F32, 2)
    g = torch.Generator().manual_seed(3)
    check(x, u, T=torch.rand(64, generator=g) * 2, k=torch.randint(0, 100, (64,), generator=g, dtype=torch.int32),
          p=torch.rand(64, generator=g) * 1.2, m=torch.rand(64, generator=g) * 0.1)
    off = torch.tensor([float("nan"), -1.0, 0.0, float("inf")])
    tokens, logprobs = call(x[:4].cuda(), u[:4].cuda(), temperature=off.cuda())
    assert (tokens[:3].long() == x[:3].argmax(1)).all() and (logprobs[:3] == 0).all()
    assert tokens[3] == int(u[3].item() * 3001) and abs(logprobs[3] + math.log(3001)) < 1e-6           # (at no end of temperature all are alike)
    same = call(x[:4].cuda(), u[:4].cuda())
    for name in ("top_p", "min_p"):
        bad = torch.tensor([float("nan")] * 4 if name == "top_p" else [float("nan"), -1.0, 0.0, -math.inf]).cuda()
        got = call(x[:4].cuda(), u[:4].cuda(), **{name: bad})
        assert torch.equal(got[0], same[0]) and torch.equal(got[1], same[1])
    got = call(x[:4].cuda(), u[:4].cuda(), top_k=torch.tensor([-5, 0, 3001, 2 ** 31 - 1], dtype=torch.int32).cuda())
    assert torch.equal(got[0], same[0])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_equal_logits_go_by_the_lower_token(dtype):
    vocab = 9000
    x = torch.zeros(8, vocab, dtype=dtype)
    x[:, 1::2] = -0.0
    x[4:, ::3] = 1.0
    u = torch.arange(8) / 8
    for how in (dict(k=10), dict(k=4000), dict(p=0.25), dict(k=5000, p=0.5), dict(k=3001), dict(p=0.7, T=0.5)):
        check(x, u, **how)
    tokens, _ = call(x.cuda(), u.cuda(), top_k=8)
    assert tokens.tolist() == [0, 1, 2, 3, 12, 15, 18, 21]


def test_exact_shares():
    """Weights 1/2, 1/4, 1/4 and shares that meet a border: what reaches top_p is kept and no more, u at a border draws the next token."""
    x = torch.tensor([[math.log(2), 0.0, 0.0]], dtype=F32)
    x = torch.cat([x, torch.zeros(1, 3)])
    rows = torch.zeros(6, 4, dtype=F32)                                       # four of one weight
    u = torch.tensor([0.0, 0.25, 0.5, 0.75, 1.0 - 2.0 ** -24, 0.4999999])
    assert call(rows.cuda(), u.cuda())[0].tolist() == [0, 1, 2, 3, 3, 1]
    for p, n in ((0.5, 2), (0.5000001, 3), (0.25, 1), (0.75, 3), (0.2, 1)):
        tokens, logprobs = call(rows.cuda(), u.cuda(), top_p=p)
        assert tokens.max() == n - 1 and abs(logprobs[0] + math.log(n)) < 1e-6
    assert call(rows.cuda(), torch.tensor([-1.0, float("nan"), 1.0, 2.0, math.inf, 0.3]).cuda())[0].tolist() == [0, 0, 3, 3, 3, 1]


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_masks_and_rows_with_nothing_to_draw_from(dtype):
    x, u = logits(8, 5000, dtype, 4)
    x[:, ::2] = -math.inf
    for how in (dict(), dict(k=4000), dict(p=0.9), dict(k=10, p=0.5), dict(T=0.0)):
        check(x, u, **how)
    lowest = x.clone()
    lowest[:, ::2] = torch.finfo(dtype).min
    check(lowest, u, p=0.9)
    check(lowest, u, T=1e30)
    x[1], x[2, 17], x[3, 4999], x[4, 3:] = -math.inf, float("nan"), math.inf, -math.inf
    x[4, 1] = -5.0
    for how in (dict(), dict(top_k=3), dict(top_p=0.5), dict(temperature=0.0)):
        tokens, logprobs = call(x.cuda(), u.cuda(), **how)
        assert tokens[1] == tokens[2] == tokens[3] == -1 and logprobs[1:4].isnan().all()
        assert tokens[4] == 1 and logprobs[4] == 0 and (tokens[5:] >= 0).all()


def test_strides_and_optional_outputs():
    x, u = logits(5, 1001, BF16, 5)
    wide = torch.full((5, 1040), float("nan"), dtype=BF16, device="cuda")
    wide[:, 3:1004] = x.cuda()
    want = call(x.cuda(), u.cuda(), top_p=0.9)
    got = call(wide[:, 3:1004], u.cuda(), top_p=0.9)
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
    tokens = torch.zeros(5, dtype=torch.int32, device="cuda")
    rl.sample_tokens(x.cuda(), u.cuda(), tokens, top_p=0.9)
    assert torch.equal(tokens.cpu(), want[0])
    one = x[:1].cuda().expand(5, 1001)
    assert torch.equal(call(one, u.cuda())[0], call(one.contiguous(), u.cuda())[0])
    assert call(x[:0].cuda(), u[:0].cuda())[0].numel() == 0


def test_shares_of_many_draws():
    """One row drawn by evenly spaced numbers: every token as often as its probability says, one draw more or less for each border."""
    x, _ = logits(1, 300, F32, 6, 2.0)
    n = 4096
    u = (torch.arange(n) + 0.5) / n
    for how in (dict(), dict(T=0.8, p=0.9)):
        keep = dict(T=1.0, k=0, p=1.0, m=0.0, **{}) | how
        w = torch.where(kept(x[0], **keep), weights(x[0], keep["T"]), 0.0)
        tokens, _ = call(x.cuda().expand(n, 300), u.cuda(), temperature=keep["T"], top_p=keep["p"])
        count = torch.bincount(tokens.long(), minlength=300)
        assert ((count - n * w / w.sum()).abs() <= 1 + 1e-6).all()


def test_recorded_calls_draw_by_the_numbers_of_the_replay():
    x, u = logits(9, 20000, BF16, 7)
    x, u = x.cuda(), u.cuda()
    tokens, logprobs = torch.zeros(9, dtype=torch.int32, device="cuda"), torch.zeros(9, device="cuda")
    work = torch.zeros(max(1, rl.rlkv_sample_tokens_workspace(9, 20000)), dtype=torch.uint8, device="cuda")
    run = lambda: rl.sample_tokens(x, u, tokens, temperature=0.9, top_k=300, top_p=0.9, logprobs=logprobs, workspace=work)      # noqa: E731
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i in range(4):
        u.copy_(torch.rand(9, generator=torch.Generator().manual_seed(i)))
        work.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        got = tokens.clone(), logprobs.clone()
        run()
        torch.cuda.synchronize()
        assert torch.equal(got[0], tokens) and torch.equal(got[1], logprobs)
    with torch.cuda.stream(torch.cuda.Stream()):
        other = call(x, u, temperature=0.9, top_k=300, top_p=0.9)
    assert torch.equal(other[0], tokens.cpu())


@pytest.mark.parametrize("k", [1, 2, 5, 12, 13, 191, 192, 193, 384, 500, 1000])
@pytest.mark.parametrize("vocab", [7, 8, 130, 8193, 30000, 131071])
def test_top_k_of_any_number(vocab, k):
    """Around the numbers up to which a top_k is found among the largest logits of groups of tokens."""
    x, u = logits(6, vocab, F32, seed=vocab + k)
    check(x, u, T=0.9, k=k, p=0.97, m=1e-3)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_top_k_where_most_tokens_are_masked(dtype):
    """Tokens of a few chunks only, of one chunk, every 500th, fewer than top_k; and many equal ones where the cut falls."""
    x, u = logits(6, 100003, dtype, seed=11)
    x[0, 4000:] = -math.inf
    x[1, :70000] = x[1, 70090:] = -math.inf
    x[2, torch.arange(100003) % 500 != 3] = -math.inf
    x[3, 9:] = -math.inf
    x[4] = (x[4] / 4).round() * 4
    x[5] = x[5].clamp(max=0.5)
    for k in (20, 50, 180):
        check(x, u, k=k)
        check(x, u, T=1.3, k=k, p=0.8)


def test_top_k_of_negative_logits_and_zeros():
    x, u = logits(4, 20000, F32, seed=12)
    x[0] = -x[0].abs() - 100
    x[1, x[1] > 0] = -0.0
    x[2, x[2] > 0] = 0.0
    x[3] = 1e-40 * x[3]
    for k in (3, 64):
        check(x, u, k=k)


@pytest.mark.parametrize("equal", [150, 300, 700, 2000, 2100])
def test_top_k_among_equal_logits(equal):
    """Lists of the most likely tokens that are far longer than top_k."""
    x, u = logits(8, 40000, F32, seed=13)
    x[:, torch.randperm(40000, generator=torch.Generator().manual_seed(equal))[:equal]] = 20.0
    x[::2, 777] = 21.0
    for k in (40, 170, 600):
        check(x, u, k=k)
        check(x, u, k=k, p=0.73, T=0.5, m=0.01)


def test_temperatures_next_to_nothing():
    """As good as greedy, without infinities of what is divided by them."""
    x, u = logits(6, 30000, F32, seed=14)
    for T in (1e-30, 1e-45, 5e-324):
        for how in (dict(), dict(k=300), dict(k=20), dict(p=0.9), dict(m=0.5)):
            check(x, u, T=T, **how)
