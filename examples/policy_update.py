"""An update of a policy and of the gates of its heads on packed rollouts: one attention layer forward and back through the library's operators.

  logits -> drawn tokens;  packed projections -> norm and rotation of the heads -> full and local attention over the packed sequences ->
  their blend by a gate for each KV head -> product to the vocabulary -> log probabilities; and back: to the blend, to both attentions, to
  the gates, through the rotation and the norm to the projections and the norm's weights.

A gate of 1 is a head that keeps its whole past, one of 0 a head that keeps the first `sink` and the last `recent` positions: what the gates learn decides
which heads get a full cache.  Weights are random; torch supplies memory, the products with the vocabulary and the sums.

    python examples/policy_update.py
"""
from __future__ import annotations

import math
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2510_08525_amd as rl  # noqa: E402

D, EPS = 128, 1e-5


class GatedAttention:
    """out = gate full + (1 - gate) local over sequences packed one behind the other, and its gradient."""

    def __init__(self, tokens, sequences, q_heads=8, kv_heads=2, sink=4, recent=60, seed=0):
        g = torch.Generator().manual_seed(seed)
        new = lambda *shape, dtype=torch.bfloat16: torch.empty(*shape, dtype=dtype, device="cuda")       # noqa: E731
        self.heads = (q_heads, kv_heads)
        self.group, self.scale = q_heads // kv_heads, 1 / math.sqrt(D)
        self.local = dict(mask=[0] * kv_heads, sink=sink, recent=recent)
        self.rotary = rl.Rotary([500000.0 ** (-2 * i / D) for i in range(D // 2)])
        self.weights = [(1 + 0.1 * torch.randn(D, generator=g)).bfloat16().cuda() for _ in range(2)]
        self.gates = torch.rand(kv_heads, generator=g).cuda()
        # (all that the calls write, so that a graph may hold them)
        self.q, self.k, self.v = (new(tokens, h, D) for h in (q_heads, kv_heads, kv_heads))
        self.outs = [new(tokens, q_heads, D) for _ in range(2)]
        self.lses = [new(q_heads, tokens, dtype=torch.float32) for _ in range(2)]
        self.grads = [[torch.zeros_like(t) for t in (self.q, self.k, self.v)] for _ in range(2)]
        self.grad_qkv = new(tokens, (q_heads + 2 * kv_heads) * D)
        self.grad_weights = [new(D, dtype=torch.float32) for _ in range(2)]
        self.attention_work = new(max(1, rl.rlkv_packed_attention_grad_workspace(tokens, q_heads, kv_heads)), dtype=torch.uint8)
        self.norm_work = new(max(1, rl.rlkv_head_norm_rotary_grad_workspace(tokens, q_heads, kv_heads)), dtype=torch.uint8)

    def _gates(self):
        return self.gates.repeat_interleave(self.group)[:, None]

    def forward(self, qkv, positions, offsets):
        self.saved = (qkv, positions, offsets)
        rl.head_norm_rotary(qkv, positions, self.rotary, self.q, self.k, v_out=self.v, q_weight=self.weights[0], k_weight=self.weights[1], eps=EPS)
        for out, lse, how in zip(self.outs, self.lses, ({}, self.local)):
            rl.packed_attention(self.q, self.k, self.v, offsets, out, self.scale, lse=lse, **how)
        gate = self._gates()
        return (gate * self.outs[0] + (1 - gate) * self.outs[1]).bfloat16()

    def backward(self, grad_out):
        """Gradients of the projections, the two weights of the norm and the gates."""
        qkv, positions, offsets = self.saved
        gate = self._gates()
        for out, lse, grads, how, share in zip(self.outs, self.lses, self.grads, ({}, self.local), (gate, 1 - gate)):
            rl.packed_attention_grad(self.q, self.k, self.v, offsets, out, lse, (share * grad_out).bfloat16(), *grads, self.scale,
                                     workspace=self.attention_work, **how)
        grad_q, grad_k, grad_v = ((a.float() + b).bfloat16() for a, b in zip(*self.grads))
        rl.head_norm_rotary_grad(qkv, positions, self.rotary, grad_q, grad_k, self.grad_qkv, grad_v=grad_v, q_weight=self.weights[0],
                                 k_weight=self.weights[1], eps=EPS, grad_q_weight=self.grad_weights[0], grad_k_weight=self.grad_weights[1],
                                 workspace=self.norm_work)
        grad_gates = (grad_out.float() * (self.outs[0].float() - self.outs[1])).sum((0, 2)).view(-1, self.group).sum(1)
        return self.grad_qkv, *self.grad_weights, grad_gates


def update(layer, head, qkv, positions, offsets, tokens, advantage):
    """Log probabilities of `tokens` [rows] under the layer and the product with `head` [vocab, q heads * 128] (float32), and the gradients
    of - sum(advantage * log probability)."""
    rows = tokens.shape[0]
    logits = layer.forward(qkv, positions, offsets).view(rows, -1).float() @ head.t()
    logprob, lse = (torch.empty(rows, device="cuda") for _ in range(2))
    rl.token_logprobs(logits, tokens, logprob, lse=lse)
    grad_logits = torch.empty_like(logits)
    rl.token_logprobs_grad(logits, tokens, lse, -advantage, grad_logits)
    grad_out = (grad_logits @ head).bfloat16().view(rows, *layer.q.shape[1:])
    return logprob, layer.backward(grad_out)


def rollouts(lengths, vocab, generator):
    """Drawn tokens of sequences of these lengths, packed, their positions and where the sequences begin.  (Here from random logits.)"""
    rows = sum(lengths)
    logits = (3 * torch.randn(rows, vocab, generator=generator)).cuda()
    tokens, old = torch.empty(rows, dtype=torch.int32, device="cuda"), torch.empty(rows, device="cuda")
    rl.sample_tokens(logits, torch.rand(rows, generator=generator).cuda(), tokens, temperature=0.7, top_p=0.95, logprobs=old)
    positions = torch.cat([torch.arange(n, dtype=torch.int32) for n in lengths]).cuda()
    offsets = torch.tensor([0] + lengths).cumsum(0).int().cuda()
    return tokens, old, positions, offsets


def main():
    g = torch.Generator().manual_seed(0)
    lengths, vocab = [70, 1, 333, 129], 1000
    tokens, old, positions, offsets = rollouts(lengths, vocab, g)
    layer = GatedAttention(sum(lengths), len(lengths))
    qkv = torch.randn(sum(lengths), layer.grad_qkv.shape[1], generator=g).bfloat16().cuda()
    head = (torch.randn(vocab, layer.heads[0] * D, generator=g) / math.sqrt(layer.heads[0] * D)).cuda()
    advantage = torch.randn(sum(lengths), generator=g).cuda()
    logprob, (grad_qkv, grad_q_weight, grad_k_weight, grad_gates) = update(layer, head, qkv, positions, offsets, tokens, advantage)
    print(f"log probability of what was drawn {old.mean():.3f} where it was drawn, {logprob.mean():.3f} under the layer")
    print(f"norms of the gradients: projections {grad_qkv.float().norm():.3f}, norm's weights {grad_q_weight.norm():.3f} and "
          f"{grad_k_weight.norm():.3f}; gates {[round(x, 3) for x in grad_gates.tolist()]}")


if __name__ == "__main__":
    main()
