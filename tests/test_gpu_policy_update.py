"""The policy's operators as a training loop runs them one behind the other: sampling, norm with rotation, both attentions with their blend,
log probabilities, and the whole way back; and the same calls from a graph.

Against the formulas in 64 bits from the projections on.  Eleven values on the way are rounded to bf16 (q, k, weights, both outputs, their blend, its gradient,
the shares of it, z, the gradients of an attention, their sum, the result), each by at most 2^-8 of it.  Where z = w (dp - delta) subtracts, errors of dp count
up to twice: a gradient is off by at most 22 * 2^-8 of it in the 2-norm.  (Where a query has one key dp is delta and z is 0 by the formula, on the GPU what
two sums of 128 products in fp32 differ by, 2 * 128 * 2^-24 = 2^-16 of |grad_out| |v|: through z k and the norm, whose rows have a root mean square
above 1/2 here, 2^-15 scale |grad_out| |v| |k| comes on top.)  A gate's gradient is a sum of grad_out (full - local) whose
parts were rounded independently: off by at most 22 * 2^-8 of the root of the sum of (|grad_out| (|full| + |local|))^2.  Log probabilities: the
blend's rounding and what it carries (five of the eleven, 5 * 2^-8 of a component at most), through products with `head` of rows of norm 1,
is in the 2-norm over a row's components at most 5 * 2^-8 |blend|, twice (the token's logit and the log-sum-exp)."""
import math
import os
import sys

import pytest
import torch

import paper_2510_08525_amd as rl

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
D = 128


def reference(layer, head, qkv, positions, lengths, tokens, advantage):
    """Log probabilities, the blend, the gradients by autograd in 64 bits on the CPU, and what the bounds are made of."""
    Hq, H = layer.heads
    leaves = [t.detach().double().cpu().requires_grad_() for t in (qkv, *layer.weights, layer.gates)]
    x, wq, wk, gates = leaves
    x = x.view(x.shape[0], Hq + 2 * H, D)
    t = positions.cpu().double()[:, None, None] * torch.tensor([500000.0 ** (-2 * i / D) for i in range(D // 2)], dtype=torch.float64)

    def head_rows(x, w):
        y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-5) * w
        a, b = y[..., :D // 2], y[..., D // 2:]
        return torch.cat([a * t.cos() - b * t.sin(), b * t.cos() + a * t.sin()], -1)

    q, k, v = head_rows(x[:, :Hq], wq), head_rows(x[:, Hq:Hq + H], wk), x[:, Hq + H:]
    k, v = (y.repeat_interleave(layer.group, 1) for y in (k, v))
    blends, fulls, locals_ = [], [], []
    at = 0
    for n in lengths:
        rows = slice(at, at + n)
        s = torch.stack([q[rows, h] @ k[rows, h].t() for h in range(Hq)]) * layer.scale
        i, j = torch.arange(n)[:, None], torch.arange(n)[None]
        causal = j <= i
        near = causal & ((j < layer.local["sink"]) | (i - j < layer.local["recent"]))
        values = v[rows].transpose(0, 1)
        full, local = (torch.matmul(torch.softmax(s.masked_fill(~m, -math.inf), -1), values).transpose(0, 1) for m in (causal, near))
        gate = gates.repeat_interleave(layer.group)[:, None]
        blends.append(gate * full + (1 - gate) * local)
        fulls.append(full)
        locals_.append(local)
        at += n
    blend, full, local = (torch.cat(y) for y in (blends, fulls, locals_))
    blend.retain_grad()
    logprob = torch.log_softmax(blend.reshape(blend.shape[0], -1) @ head.double().cpu().t(), -1).gather(1, tokens.long().cpu()[:, None])[:, 0]
    (-(advantage.double().cpu() * logprob).sum()).backward()
    spread = (blend.grad.abs() * (full.abs() + local.abs())).detach().pow(2).sum((0, 2)).view(H, -1).sum(1).sqrt()
    rows = [y.detach().norm(dim=-1).max() for y in (k, v)]
    return logprob.detach(), blend.detach(), [y.grad for y in leaves], spread, 2.0 ** -15 * layer.scale * blend.grad.norm() * rows[0] * rows[1]


def setup(lengths, heads, seed=0):
    from policy_update import GatedAttention, rollouts

    g = torch.Generator().manual_seed(seed)
    T = sum(lengths)
    tokens, old, positions, offsets = rollouts(lengths, 500, g)
    layer = GatedAttention(T, len(lengths), *heads, seed=seed)
    qkv = torch.randn(T, layer.grad_qkv.shape[1], generator=g).bfloat16().cuda()
    head = torch.randn(500, heads[0] * D, generator=g)
    head = (head / head.norm(dim=1, keepdim=True)).cuda()
    return tokens, positions, offsets, layer, qkv, head, torch.randn(T, generator=g).cuda()


@pytest.mark.parametrize("lengths, heads", [([70, 1, 333, 129], (8, 2)), ([1], (4, 4)), ([65, 64, 63, 2, 200], (14, 2))])
def test_an_update_against_autograd(lengths, heads):
    from policy_update import update

    tokens, positions, offsets, layer, qkv, head, advantage = setup(lengths, heads)
    assert ((tokens >= 0) & (tokens < 500)).all()
    logprob, grads = update(layer, head, qkv, positions, offsets, tokens, advantage)
    want, blend, wants, spread, least = reference(layer, head, qkv, positions, lengths, tokens, advantage)
    part = 22 * 2.0 ** -8
    assert ((logprob.double().cpu() - want).abs() <= 2 * 5 * 2.0 ** -8 * blend.flatten(1).norm(dim=1) + 1e-5).all()
    for name, x, y in zip(("projections", "query weight", "key weight"), grads, wants):
        off = (x.double().cpu() - y).norm()
        assert off <= part * y.norm() + least, f"{name}: {off / y.norm():.4f}"
    assert ((grads[3].double().cpu() - wants[3]).abs() <= part * spread + 1e-30).all()


def test_gates_by_differences():
    """The loss (in 64 bits from the kernels' own outputs, so without their roundings) along a step of the gates changes as their gradient says."""
    from policy_update import update

    tokens, positions, offsets, layer, qkv, head, advantage = setup([90, 40, 211], (8, 2), 3)
    _, (_, _, _, grad) = update(layer, head, qkv, positions, offsets, tokens, advantage)
    full, local = (out.double().cpu() for out in layer.outs)

    def loss(gates):
        gate = gates.repeat_interleave(layer.group)[:, None]
        logits = (gate * full + (1 - gate) * local).flatten(1) @ head.double().cpu().t()
        return -(advantage.double().cpu() * torch.log_softmax(logits, -1).gather(1, tokens.long().cpu()[:, None])[:, 0]).sum()

    gates, spread = layer.gates.double().cpu(), reference(layer, head, qkv, positions, [90, 40, 211], tokens, advantage)[3]
    for h in range(2):
        step = torch.zeros(2, dtype=torch.float64)
        step[h] = 1e-4
        slope = (loss(gates + step) - loss(gates - step)) / 2e-4
        # (the blend is rounded before the logits, its gradient behind them: two of the roundings above)
        assert abs(slope - grad[h].double().cpu()) <= 2 * 2.0 ** -8 * spread[h] + 1e-6


def test_a_layer_from_a_graph():
    """Recorded once and replayed on other inputs, with eager calls of the same layer between: the bits of the eager calls."""
    lengths = [70, 1, 333, 129]
    tokens, positions, offsets, layer, qkv, head, advantage = setup(lengths, (8, 2), 5)
    grad = torch.randn(sum(lengths), 8, D, generator=torch.Generator().manual_seed(6)).bfloat16().cuda()

    def run():
        out = layer.forward(qkv, positions, offsets)
        return [out, *layer.backward(grad)[:3]]

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        recorded = run()
    for turn in range(3):
        g = torch.Generator().manual_seed(100 + turn)
        qkv.copy_(torch.randn(qkv.shape, generator=g))
        grad.copy_(torch.randn(grad.shape, generator=g))
        want = [t.clone() for t in run()]
        for t in (layer.grad_qkv, *layer.grad_weights, *layer.outs):
            t.fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(recorded, want):
            assert torch.equal(x, y), turn


def test_what_is_drawn_in_a_rollout():
    """Tokens are among those that the filters keep; with a temperature of 0 they are the greedy rollout's."""
    from decoder_rollout import Decoder

    prompts = torch.randint(0, 1000, (3, 64), generator=torch.Generator().manual_seed(3)).cuda()
    counts = [40, 64, 7]
    greedy = Decoder().rollout(prompts, counts, 5)
    assert torch.equal(Decoder().rollout(prompts, counts, 5, dict(temperature=0.0))[0], greedy[0])
    how = dict(temperature=1.5, top_k=20)
    tokens, _, _, _, logits = Decoder().rollout(prompts, counts, 5, how, seed=1)
    assert torch.equal(tokens, Decoder().rollout(prompts, counts, 5, how, seed=1)[0])
    best = logits.topk(20, -1).indices
    assert (best == tokens[..., None]).any(-1).all() and not torch.equal(tokens, greedy[0])


def test_on_a_stream_of_the_callers():
    """The calls run on torch's current stream: what the other stream holds back, they wait for."""
    lengths = [70, 1, 333, 129]
    tokens, positions, offsets, layer, qkv, head, advantage = setup(lengths, (8, 2), 7)
    grad = torch.randn(sum(lengths), 8, D, generator=torch.Generator().manual_seed(8)).bfloat16().cuda()
    want = [t.clone() for t in (layer.forward(qkv, positions, offsets), *layer.backward(grad)[:3])]
    values, stream = qkv.clone(), torch.cuda.Stream()
    qkv.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        big = torch.randn(4096, 4096, device="cuda")
        for _ in range(20):
            big = big @ big * 1e-4
        qkv.copy_(values)
        got = [layer.forward(qkv, positions, offsets), *layer.backward(grad)[:3]]
    stream.synchronize()
    for x, y in zip(got, want):
        assert torch.equal(x, y)
