"""The policy's operators on tensors whose rows lie past 2^32 bytes and 2^31 elements of their beginnings, and at their largest vocabulary."""
import packed_reference as ref
import pytest
import torch

import paper_2510_08525_amd as rl
from test_gpu_packed_attention import BF, D, SCALE

pytestmark = pytest.mark.gpu
TOKENS, WIDE = 2 ** 19 + 100, 8192              # 2^32 elements and more


def _views(how, tokens, rows):
    """Eight tensors of 8, 2, 2, 8, 8, 8, 2, 2 heads in one buffer of zeros, far rows or far heads, and the buffer."""
    buffer = torch.zeros(TOKENS * WIDE, dtype=BF, device="cuda")
    heads, out, at = (8, 2, 2, 8, 8, 8, 2, 2), [], 0
    far = TOKENS * WIDE // 8 // 8 * 8           # from head to head: seven times that is past 2^31
    for h in heads:
        if how == "tokens":
            out.append(buffer.as_strided((tokens, h, D), (WIDE, D, 1), at * D))
            at += h
        else:
            out.append(buffer.as_strided((tokens, h, D), (D, far, 1), at))
            at += tokens * D
    return out, buffer


@pytest.mark.parametrize("how", ["tokens", "heads"])
def test_attention_and_its_gradient(how):
    tokens = TOKENS if how == "tokens" else 900
    lengths, mask, sink, recent = [333, 1, 0, 290], [1, 0], 5, 70
    rows, first = sum(lengths), tokens - 7 - sum(lengths)
    (q, k, v, g, out, dq, dk, dv), buffer = _views(how, tokens, rows)
    inside = slice(first, first + rows)
    gen = torch.Generator().manual_seed(1)
    small = [torch.randn(rows, t.shape[1], D, generator=gen).to(BF) for t in (q, k, v, g)]
    for t, x in zip((q, k, v, g), small):
        t[inside] = x.cuda()
    offsets = torch.tensor([0] + lengths).cumsum(0).add(first).int().cuda()
    lse = torch.full((8, tokens), 7.0, device="cuda")
    how = dict(mask=mask, sink=sink, recent=recent)
    rl.packed_attention(q, k, v, offsets, out, SCALE, lse=lse, **how)
    rl.packed_attention_grad(q, k, v, offsets, out, lse, g, dq, dk, dv, SCALE, **how)
    torch.cuda.synchronize()
    want, want_lse, tol, lse_tol = ref.attention(*small[:3], lengths, mask, sink, recent, SCALE)
    ref.near(out[inside], want, tol)
    ref.near(lse[:, inside], want_lse, lse_tol)
    grads, tols = ref.gradient(*small[:3], out[inside].cpu(), lse[:, inside].cpu(), small[3], lengths, mask, sink, recent, SCALE)
    for x, y, t in zip((dq, dk, dv), grads, tols):
        ref.near(x[inside], y, t)
    # nothing else was written
    assert (lse[:, :first] == 7).all() and (lse[:, first + rows:] == 7).all()
    for t in (q, k, v, g, out, dq, dk, dv):
        t[inside] = 0
    assert all(not part.any() for part in buffer.split(2 ** 30))


def test_norm_and_rotation():
    """The bits of a small call on the same last rows."""
    heads, last = (8, 2, 2), 300
    tokens, buffer = 2 ** 19 + 100, torch.zeros(TOKENS * WIDE, dtype=BF, device="cuda")
    qkv = buffer.as_strided((tokens, 12 * D), (WIDE, 1), 0)
    q, k, v = (buffer.as_strided((tokens, h, D), (WIDE, D, 1), at * D) for h, at in zip(heads, (12, 20, 22)))
    grad = buffer.as_strided((tokens, 12 * D), (WIDE, 1), 24 * D)
    g = torch.Generator().manual_seed(2)
    qkv[-last:] = torch.randn(last, 12 * D, generator=g).to(BF).cuda()
    positions = torch.randint(0, 5000, (tokens,), generator=g, dtype=torch.int32).cuda()
    rotary = rl.Rotary([500000.0 ** (-i / 64) for i in range(64)])
    rl.head_norm_rotary(qkv, positions, rotary, q, k, v_out=v, eps=1e-5)
    rl.head_norm_rotary_grad(qkv, positions, rotary, q, k, grad, grad_v=v, eps=1e-5)
    small = qkv[-last:].contiguous()
    a, b, c = (torch.empty(last, h, D, dtype=BF, device="cuda") for h in heads)
    rl.head_norm_rotary(small, positions[-last:].contiguous(), rotary, a, b, v_out=c, eps=1e-5)
    back = torch.empty_like(small)
    rl.head_norm_rotary_grad(small, positions[-last:].contiguous(), rotary, a, b, back, grad_v=c, eps=1e-5)
    for x, y in ((q, a), (k, b), (v, c), (grad, back)):
        assert torch.equal(x[-last:], y) and y.any()


@pytest.mark.parametrize("how", [dict(), dict(top_p=0.9), dict(top_k=30, min_p=0.01)])
def test_rows_of_logits(how):
    rows, stride, vocab = 20000, 160000, 1000
    buffer = torch.empty(rows * stride, device="cuda")
    x = buffer.as_strided((rows, vocab), (stride, 1))
    g = torch.Generator().manual_seed(3)
    small = (3 * torch.randn(rows, vocab, generator=g)).cuda()
    x.copy_(small)
    u = torch.rand(rows, generator=g).cuda()
    a, b = (torch.empty(rows, dtype=torch.int32, device="cuda") for _ in range(2))
    rl.sample_tokens(x, u, a, **how)
    rl.sample_tokens(small, u, b, **how)
    assert torch.equal(a, b) and (a >= 0).all() and len(a.unique()) > 500


def test_the_largest_vocabulary():
    """2^24 tokens, weights of 2^-38: rounded to half of that each, so their sum is off by 2^-15 of the largest weight at most."""
    vocab = 2 ** 24
    x = 2 * torch.randn(vocab, generator=torch.Generator().manual_seed(4))
    w = torch.exp(x.double() - x.double().max())
    u = torch.tensor([0.0, 0.3, 0.77, 0.999999])
    tokens, logprobs = torch.empty(4, dtype=torch.int32, device="cuda"), torch.empty(4, device="cuda")
    rows = x.cuda().expand(4, vocab).contiguous()
    rl.sample_tokens(rows, u.cuda(), tokens, logprobs=logprobs)
    cum = torch.cumsum(w, 0)
    for t, lp, r in zip(tokens.tolist(), logprobs.tolist(), u.double().tolist()):
        assert cum[t] - w[t] - 2.0 ** -15 <= r * cum[-1] <= cum[t] + 2.0 ** -15
        assert abs(lp - float(torch.log(w[t] / cum[-1]))) <= 2.0 ** -24 * abs(lp) + 2.0 ** -15 / float(cum[-1]) + 1e-9
    best, order = torch.sort(x, descending=True, stable=True)
    for how, kept in ((dict(top_k=40), 40), (dict(top_k=40, top_p=0.5), None)):
        rl.sample_tokens(rows, u.cuda(), tokens, logprobs=logprobs, **how)
        v = torch.exp(best[:40].double() - best[0].double())
        if kept is None:
            kept = int((torch.cumsum(v, 0) - v < 0.5 * v.sum()).sum())
        inside = torch.zeros(vocab, dtype=torch.float64)
        inside[order[:kept]] = w[order[:kept]]
        cum = torch.cumsum(inside, 0)
        for t, r in zip(tokens.tolist(), u.double().tolist()):
            assert inside[t] > 0 and cum[t] - inside[t] - 2.0 ** -30 <= r * cum[-1] <= cum[t] + 2.0 ** -30
