"""Attention over packed sequences, and its gradient, at sizes that no other test has: more KV heads than a word of the mask has bits, and 16384 keys."""
import packed_reference as ref
import pytest
import torch

from test_gpu_packed_attention import SCALE, check, inputs, run
from test_gpu_packed_attention_grad import check as check_grad
from test_gpu_packed_attention_grad import run as run_grad

pytestmark = pytest.mark.gpu

MASKS = {"all full": lambda n: [1] * n, "all local": lambda n: [0] * n, "every third": lambda n: [int(h % 3 == 0) for h in range(n)],
         "the last": lambda n: [0] * (n - 1) + [1], "but the first": lambda n: [0] + [1] * (n - 1), "a word": lambda n: [int(h // 64 == 1) for h in range(n)]}


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("kv_heads, group", [(64, 1), (65, 2), (100, 1), (129, 1), (256, 1), (256, 3)])
def test_many_heads(kv_heads, group, mask):
    check([30, 1, 60], kv_heads * group, kv_heads, MASKS[mask](kv_heads), 3, 9, tail=3, seed=kv_heads)
    check_grad([30, 1, 60], kv_heads * group, kv_heads, MASKS[mask](kv_heads), 3, 9, tail=3, seed=kv_heads)


def test_many_heads_not_divided():
    """(More than 256 workgroups of queries.)"""
    check([300, 70], 256, 256, MASKS["every third"](256), 20, 90, tail=300, seed=3)
    check_grad([300, 70], 256, 256, MASKS["every third"](256), 20, 90, tail=300, seed=3)


def _few(n):
    """Rows of a long sequence that are looked at: its first and last ones, and around tiles and workgroups."""
    return torch.tensor(sorted({0, 1, 63, 64, 4095, 8191, 8192, 8193, 10007, n - 257, n - 64, n - 2, n - 1}))


@pytest.mark.parametrize("q_heads, kv_heads, mask, sink, recent", [(4, 2, [1, 0], 64, 512), (2, 1, [1], 0, 0), (2, 1, [0], 5000, 3000)])
def test_16384_keys(q_heads, kv_heads, mask, sink, recent):
    """Some rows of each result against 64 bits (bounds as in packed_reference.py; the gradient's from out and lse as the forward call left them)."""
    n, group = 16384, q_heads // kv_heads
    q, k, v, go, offsets = inputs([n], q_heads, kv_heads, seed=5)
    out, lse = run(q, k, v, offsets, mask, sink, recent)
    dq, dk, dv = (t.cpu() for t in run_grad(q, k, v, out, lse, go, offsets, mask, sink, recent))
    q, k, v, go, out, lse = (t.cpu().double() for t in (q, k, v, go, out, lse))
    at, place = _few(n), torch.arange(n)
    delta, far_delta = (go * out).sum(-1), (go * out).abs().sum(-1)

    def admitted(i, j, h):
        near = j <= i
        return near if mask[h] else near & ((j < sink) | (i - j < recent))

    def pairs(i, j, head):
        """w, z of the query rows i and keys j [i, j] and their errors without the rounding to bf16."""
        h = head // group
        x, y, g, z = q[i, head], k[j, h], go[i, head], v[j, h]
        on = admitted(i[:, None], j[None], h)
        w = torch.exp(SCALE * x @ y.t() - lse[head, i, None]).masked_fill(~on, 0)
        e = 2.0 ** -17 * SCALE * (x.abs() @ y.abs().t()) + ref.FP32 * (1 + lse[head, i, None].abs())
        way = g @ z.t() - delta[i, head, None]
        ez = w * e * way.abs() + w * ref.FP32 * (g.abs() @ z.abs().t() + far_delta[i, head, None]) + on * ref.TINY * (way.abs() + 1)
        return w, w * way, w * e + on * ref.TINY, ez

    for head in range(q_heads):
        h = head // group
        s = (SCALE * q[at, head] @ k[:, h].t()).masked_fill(~admitted(at[:, None], place[None], h), float("-inf"))
        e = 2.0 ** -17 * SCALE * (q[at, head].abs() @ k[:, h].abs().t()).amax(-1, keepdim=True) + ref.FP32
        p = torch.softmax(s, -1)
        want = p @ v[:, h]
        ref.near(out[at, head], want, (ref.BF16 + 2 * e) * (p @ v[:, h].abs()) + ref.BF16 * want.abs() * (1 + ref.BF16))
        top = torch.logsumexp(s, -1)
        ref.near(lse[head, at], top, e[:, 0] + ref.FP32 * top.abs())
        _, z, _, ez = pairs(at, place, head)
        want = SCALE * z @ k[:, h]
        ref.near(dq[at, head], want, SCALE * (ref.BF16 * z.abs() + ez) @ k[:, h].abs() * (1 + ref.BF16) + ref.BF16 * want.abs())
    for h in range(kv_heads):
        wants, bounds = [0, 0], [0, 0]
        for head in range(h * group, (h + 1) * group):
            w, z, ew, ez = (t.t() for t in pairs(place, at, head))
            wants = [wants[0] + SCALE * z @ q[:, head], wants[1] + w @ go[:, head]]
            bounds = [bounds[0] + SCALE * (ref.BF16 * z.abs() + ez) @ q[:, head].abs() * (1 + ref.BF16),
                      bounds[1] + (ref.BF16 * w + ew) @ go[:, head].abs() * (1 + ref.BF16)]
        for got, want, bound in zip((dk, dv), wants, bounds):
            ref.near(got[at, h], want, bound + ref.BF16 * want.abs())
