"""Gradient of log probabilities and entropies of logits far from 0: with lse given, the distance to it is what counts, not the logits' size.

p = exp(scale x - lse) with scale x - lse rounded once (one fused operation; |scale x - lse| = D), times log2(e), whose constant is rounded too: the
exponent is off by 3 * 2^-24 D, the exponential by 2^-23, so p by (3 D + 2) 2^-24 of itself.  The factor g + gh (log p + H) takes D's error
once more and six roundings of its parts' sizes: (3 D + 8) 2^-24 of size = p (|g| + |gh| (|log p| + |H|)) covers each, twice that both; the token's own
g two roundings; then the output's.
"""
import pytest
import torch

import paper_2510_08525_amd as rl

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("shift", [0.0, 300.0, -2.0e3, 3.0e4])
@pytest.mark.parametrize("scale", [1.0, 0.7])
@pytest.mark.parametrize("rows,vocab,dtype", [(3, 1000, torch.float32), (2, 32003, torch.float32), (5, 777, torch.bfloat16)])
def test_gradient(rows, vocab, dtype, scale, shift):
    g = torch.Generator().manual_seed(vocab)
    x = (torch.randn(rows, vocab, generator=g) * 3 + shift).to(dtype).cuda()
    tokens = torch.randint(0, vocab, (rows,), generator=g, dtype=torch.int32).cuda()
    scale32 = float(torch.tensor(scale, dtype=torch.float32))
    z = x.double() * scale32
    lse = torch.logsumexp(z, -1).float()
    lp = z - lse.double()[:, None]
    p = lp.exp()
    h = torch.special.entr(torch.softmax(z, -1)).sum(-1).float()
    gl, gh = (torch.randn(rows, generator=g).cuda() for _ in range(2))
    part = lp + h.double()[:, None]
    want = -p * (gl.double()[:, None] + gh.double()[:, None] * part)
    hot = torch.zeros_like(want)
    hot.scatter_(1, tokens.long()[:, None], gl.double()[:, None])
    size = p * (gl.double().abs()[:, None] + gh.double().abs()[:, None] * (lp.abs() + h.double()[:, None]))
    want, tol = scale32 * (want + hot), scale32 * (2 * (3 * lp.abs() + 8) * U * size + 2 * U * hot.abs())
    half = 2.0 ** -8 if dtype == torch.bfloat16 else U
    out = torch.empty_like(x)
    rl.token_logprobs_grad(x, tokens, lse, gl, out, scale=scale, entropy=h, grad_entropy=gh)
    err, tol = (out.double() - want).abs(), tol + half * want.abs() + 1e-37
    assert (err <= tol).all(), float((err / tol).max())
