"""The workspace of the heads' gradient: 512 bytes a workgroup of 32 rows side by side, of which none is to add up more than 512 one behind the other."""
import pytest

import paper_2510_08525_amd as rl

need = rl.rlkv_head_norm_rotary_grad_workspace


@pytest.mark.parametrize("q_heads, kv_heads", [(28, 4), (32, 8), (1, 1), (1024, 1), (1, 300)])
def test_no_smaller_for_more_tokens(q_heads, kv_heads):
    last = 0
    for tokens in (1, 63, 70, 1800, 2047, 2048, 2100, 10 ** 5, 424857, 424858, 528264, 528265, 10 ** 6, 10 ** 7):
        if tokens * (q_heads + 2 * kv_heads) < 2 ** 29:
            assert need(tokens, q_heads, kv_heads) >= last
            last = need(tokens, q_heads, kv_heads)


@pytest.mark.parametrize("tokens, q_heads, kv_heads", [(14 * 10 ** 6, 28, 4), (10 ** 7, 32, 8), (2 ** 28 // 3, 1, 1)])
def test_grows_with_the_rows(tokens, q_heads, kv_heads):
    assert need(tokens, q_heads, kv_heads) >= tokens * (q_heads + kv_heads) // (32 * 512) * 512
