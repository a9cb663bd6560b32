"""The rollout example: prompts and steps agree with each other, scores with their formulas, the gradient with its own."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_steps_say_what_the_prompt_says():
    """The logits of a prompt's tokens, all at once and token by token: the same operations on the same values.  What may differ is the order of
    attention's sums and the way of the 8-bit products of many rows, both below the rounding of the bf16 activations; two layers of those
    and the final product leave the logits within 5 % of their 2-norm."""
    from decoder_rollout import Decoder

    tokens = torch.randint(0, 1000, (3, 40), generator=torch.Generator().manual_seed(2)).cuda()
    whole, single = Decoder(), Decoder()
    a = whole.forward(tokens, [40, 40, 40])
    b = torch.cat([single.forward(tokens[:, i:i + 1]) for i in range(40)], 1)
    assert (a - b).norm() <= 0.05 * b.norm()
    assert (whole.cache.lengths(1) == single.cache.lengths(1)).all()


@pytest.mark.parametrize("page", [0, 32])
def test_rollout(page):
    from decoder_rollout import Decoder, policy_gradient

    model = Decoder(page_tokens=page)
    prompts = torch.randint(0, 1000, (3, 64), generator=torch.Generator().manual_seed(3)).cuda()
    tokens, logprob, entropy, lse, logits = model.rollout(prompts, [40, 64, 7], 10)
    assert model.cache.lengths(0).tolist() == [49, 73, 16]
    lp = torch.log_softmax(logits.double(), -1)
    assert torch.equal(tokens.long(), lp.argmax(-1))
    assert torch.allclose(logprob.double(), lp.amax(-1), atol=1e-5) and torch.allclose(entropy.double(), -(lp.exp() * lp).sum(-1), atol=1e-5)
    adv = torch.randn(30, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    z = logits.reshape(30, -1)
    grad = policy_gradient(z, tokens.reshape(-1), lse.reshape(-1), entropy.reshape(-1), adv, 0.1)
    x = z.double().cpu().requires_grad_()
    l = torch.log_softmax(x, -1)
    (-(adv.double().cpu() * l.gather(1, tokens.reshape(-1, 1).long().cpu())[:, 0]).sum() + 0.1 * (l.exp() * l).sum()).backward()
    assert torch.allclose(grad.double().cpu(), x.grad, atol=1e-5)


def test_it_runs_as_a_program(capsys):
    import decoder_rollout

    decoder_rollout.main()
    out = capsys.readouterr().out
    assert out.count("prompt of") == 3 and "norm of the gradient" in out
