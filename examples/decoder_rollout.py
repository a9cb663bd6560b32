"""A rollout through the library's operators, as a serving or training loop would run it: an attention-only decoder with 8-bit weights.

  tokens -> embedding -> per layer: norm with residual into 8 bits, product to the packed projections, rotation and append to the head-mixed
  cache with the attention, quantising, product back -> norm -> product to the vocabulary -> log probabilities of what was said,
  entropy and alternatives; behind the rollout the gradient of a policy objective with respect to its logits.

Prompts go through `rotary` and the prefill attention, decode steps through `append_rotary` and the decode attention.  Weights are random
(there is nothing to say about what it says); torch supplies memory, the embedding lookup and the layout changes of a prompt.

    python examples/decoder_rollout.py
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

E4M3 = torch.float8_e4m3fn
D, GROUP, EPS = 128, 128, 1e-5


def block_quantize(w):
    """A weight [n, k] in 8 bits with one scale for each 128 x 128 block: done once, when weights are loaded."""
    n, k = w.shape
    pad = torch.nn.functional.pad(w.float(), (0, -k % GROUP, 0, -n % GROUP))
    blocks = pad.view(pad.shape[0] // GROUP, GROUP, pad.shape[1] // GROUP, GROUP)
    scales = (blocks.abs().amax((1, 3)) / 448).clamp(min=2.0 ** -126)
    q = (blocks / scales[:, None, :, None]).view(pad.shape)[:n, :k].to(E4M3).contiguous()
    return q, scales.contiguous()


class Decoder:
    def __init__(self, layers=2, q_heads=8, kv_heads=2, vocab=1000, batch=3, max_len=256, prompt=64, sink=4, recent=60, mask=None, seed=0,
                 page_tokens=0):
        self.layers, self.q_heads, self.kv_heads, self.batch, self.vocab = layers, q_heads, kv_heads, batch, vocab
        self.hidden = q_heads * D
        g = torch.Generator().manual_seed(seed)
        weight = lambda n, k: block_quantize((torch.randn(n, k, generator=g) / math.sqrt(k)).cuda())       # noqa: E731
        self.embedding = torch.randn(vocab, self.hidden, generator=g).bfloat16().cuda()
        self.norms = (1 + 0.1 * torch.randn(layers + 1, self.hidden, generator=g)).bfloat16().cuda()
        self.qkv = [weight((q_heads + 2 * kv_heads) * D, self.hidden) for _ in range(layers)]
        self.out = [weight(self.hidden, self.hidden) for _ in range(layers)]
        self.head = weight(vocab, self.hidden)
        mask = [[1] + [0] * (kv_heads - 1)] * layers if mask is None else mask
        pool = batch * -(-max_len // page_tokens) if page_tokens else 0
        self.cache = rl.Cache(layers, q_heads, kv_heads, D, batch, sink, recent, rl.RLKV_BF16, mask, [max_len] * batch, prefill_tokens=prompt,
                              page_tokens=page_tokens, pool_pages=pool)
        self.rotary = rl.Rotary([500000.0 ** (-2 * i / D) for i in range(D // 2)])

    def _eight_bits(self, x, norm=None, residual=None):
        """x (its norm, with the residual added in front) in 8 bits, the scales, and the sum that is the next residual."""
        rows, cols = x.shape
        q = torch.empty(rows, cols, dtype=E4M3, device="cuda")
        scales = torch.empty(-(-cols // GROUP), rows, device="cuda")
        if norm is None:
            rl.quantize(x, q, scales)
            return q, scales, None
        total = x if residual is None else torch.empty_like(x)
        rl.rms_norm(x, norm, EPS, q, scales=scales, residual=residual, sum_out=None if residual is None else total)
        return q, scales, total

    def forward(self, tokens, counts=None):
        """Logits [batch, T, vocab] of tokens [batch, T]: the prompts' first `counts` tokens, or one decode step."""
        B, T = tokens.shape
        scale = 1.0 / math.sqrt(D)
        x, residual = self.embedding[tokens.reshape(-1)], None
        for layer in range(self.layers):
            q8, s8, residual = self._eight_bits(x, self.norms[layer], residual)
            packed = torch.empty(B * T, (self.q_heads + 2 * self.kv_heads) * D, dtype=torch.bfloat16, device="cuda")
            rl.scaled_matmul(q8, s8, *self.qkv[layer], packed)
            packed = packed.view(B, T, -1)
            if counts is None:
                q, attn = (torch.empty(B, self.q_heads, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
                self.cache.append_rotary(layer, packed, None, self.rotary, q)
                self.cache.decode_attention(layer, q, attn, scale)
                attn = attn.view(B, -1)
            else:
                # (zeros: the rows past a prompt's end are not written)
                q, k, v = (torch.zeros(B, h, T, D, dtype=torch.bfloat16, device="cuda") for h in (self.q_heads, self.kv_heads, self.kv_heads))
                attn = torch.zeros_like(q)
                self.cache.rotary(layer, packed, counts, self.rotary, q, k, v)
                self.cache.prefill_attention(layer, q, k, v, counts, attn, scale)
                attn = attn.transpose(1, 2).reshape(B * T, -1)
            q8, s8, _ = self._eight_bits(attn)
            x = torch.empty(B * T, self.hidden, dtype=torch.bfloat16, device="cuda")
            rl.scaled_matmul(q8, s8, *self.out[layer], x)
        q8, s8, _ = self._eight_bits(x, self.norms[-1], residual)
        logits = torch.empty(B * T, self.vocab, device="cuda")
        rl.scaled_matmul(q8, s8, *self.head, logits)
        return logits.view(B, T, -1)

    def score(self, logits, tokens, top=0):
        """Log probabilities and entropies of `tokens` [rows] under logits [rows, vocab], lse, and the `top` most likely tokens."""
        rows = logits.shape[0]
        logprob, entropy, lse = (torch.empty(rows, device="cuda") for _ in range(3))
        best = (torch.empty(rows, top, device="cuda"), torch.empty(rows, top, dtype=torch.int32, device="cuda")) if top else None
        rl.token_logprobs(logits, tokens, logprob, entropy=entropy, lse=lse, top=best)
        return logprob, entropy, lse, best

    def rollout(self, prompts, counts, steps):
        """Greedy answers to ragged prompts: tokens, their log probabilities, entropies [batch, steps] and the logits they came from."""
        B = self.batch
        logits = self.forward(prompts, counts)
        last = logits[torch.arange(B, device="cuda"), torch.tensor(counts, device="cuda") - 1].contiguous()
        said = []
        for step in range(steps):
            if step:
                last = self.forward(said[-1][0].long().view(B, 1)).view(B, -1)
            _, _, _, (_, ids) = self.score(last, torch.full((B,), -1, dtype=torch.int32, device="cuda"), top=3)
            token = ids[:, 0].contiguous()
            logprob, entropy, lse, _ = self.score(last, token)
            said.append((token, logprob, entropy, lse, last))
        return [torch.stack(v, 1) for v in zip(*said)]


def policy_gradient(logits, tokens, lse, entropy, advantage, entropy_weight=0.01):
    """Gradient of - sum(advantage * log p(token) + entropy_weight * entropy) with respect to the logits of an answer [rows, vocab]."""
    grad = torch.empty_like(logits)
    rl.token_logprobs_grad(logits, tokens, lse, -advantage, grad, entropy=entropy, grad_entropy=torch.full_like(advantage, -entropy_weight))
    return grad


def main():
    model = Decoder()
    g = torch.Generator().manual_seed(1)
    counts = [40, 64, 7]
    prompts = torch.randint(0, model.vocab, (model.batch, 64), generator=g).cuda()
    tokens, logprob, entropy, lse, logits = model.rollout(prompts, counts, 12)
    advantage = torch.linspace(-1, 1, tokens.numel(), device="cuda")
    grad = policy_gradient(logits.reshape(-1, model.vocab), tokens.reshape(-1), lse.reshape(-1), entropy.reshape(-1), advantage)
    torch.cuda.synchronize()
    for b in range(model.batch):
        print(f"prompt of {counts[b]:3d} tokens -> {tokens[b].tolist()}  log probability {logprob[b].sum():.2f}, entropy {entropy[b].mean():.2f}")
    print(f"lengths {model.cache.lengths(0).tolist()}, norm of the gradient {grad.norm():.3f}")


if __name__ == "__main__":
    main()
