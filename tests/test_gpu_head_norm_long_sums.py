"""Gradients of the norm's weights over so many tokens that a thread would add up more than 512 rows one behind the other."""
import pytest
import torch

import paper_2510_08525_amd as rl

pytestmark = pytest.mark.gpu
D, BF = 128, torch.bfloat16


@pytest.mark.parametrize("values", [False, True])
@pytest.mark.parametrize("tokens, q_heads, kv_heads", [(819200, 28, 4), (819200 * 7, 4, 1)])
def test_sums_of_like_rows(tokens, q_heads, kv_heads, values):
    """Rows of ones and gradients of ones: with eps = 2^-14 every row adds u = 1 - 2^-15 (to 2^-24).  Sums of up to 512 of them are exact in fp32, beyond
    each row would lose or gain 2^-15; what follows are five sums over lanes and wavefronts, off by 2^-24 each, and 64 bits."""
    if values:
        tokens //= 2
    qkv = torch.ones(tokens, (q_heads + 2 * kv_heads) * D, dtype=BF, device="cuda")
    one = torch.ones(1, 1, D, dtype=BF, device="cuda")
    gq, gk = one.expand(tokens, q_heads, D), one.expand(tokens, kv_heads, D)
    sums, back = [torch.zeros(D, device="cuda") for _ in range(2)], torch.empty_like(qkv)
    rl.head_norm_rotary_grad(qkv, None, None, gq, gk, back, grad_v=gk if values else None, eps=2.0 ** -14, grad_q_weight=sums[0], grad_k_weight=sums[1])
    for got, heads in zip(sums, (q_heads, kv_heads)):
        want = tokens * heads / (1 + 2.0 ** -14) ** 0.5
        assert (got.double().cpu() - want).abs().max() <= 2.0 ** -20 * want
    # (g w - u mean(g w u)) / sqrt(..) = u (1 - u^2): what is left of 1 - u^2 = 2^-14 in fp32 is off by 2^-22
    assert (back[:, :(q_heads + kv_heads) * D].float() - 2.0 ** -14).abs().max() <= 2.0 ** -21
