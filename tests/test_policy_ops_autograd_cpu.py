"""The policy's operators are calls that autograd does not see: while gradients are recorded, a tensor that asks for one is refused, wherever it
stands; where none are recorded it is not.  (Without a GPU the first tensor of a call; a tensor on the CPU is refused for that.)"""
import pytest
import torch

import paper_2510_08525_amd as rl

B = torch.bfloat16


def _attention(device, which, back):
    q, k, v, out, g = (torch.zeros(4, h, 128, dtype=B, device=device) for h in (2, 1, 1, 2, 2))
    offsets, lse = torch.zeros(2, dtype=torch.int32, device=device), torch.zeros(2, 4, device=device)
    named = dict(q=q, k=k, v=v, out=out, lse=lse, grad_out=g)
    named[which].requires_grad_()
    if not back:
        return lambda: rl.packed_attention(q, k, v, offsets, out, 1.0, lse=lse)
    return lambda: rl.packed_attention_grad(q, k, v, offsets, out, lse, g, torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v), 1.0,
                                            workspace=torch.zeros(1, dtype=torch.uint8, device=device))


def _norm(device, which, back):
    qkv = torch.zeros(4, 512, device=device)
    q, k, v = (torch.zeros(4, h, 128, device=device) for h in (2, 1, 1))
    weights = {name: torch.zeros(128, device=device) for name in ("q_weight", "k_weight")}
    dict(qkv=qkv, q=q, k=k, v=v, **weights)[which].requires_grad_()
    if not back:
        return lambda: rl.head_norm_rotary(qkv, None, None, q, k, v_out=v, eps=1e-5, **weights)
    return lambda: rl.head_norm_rotary_grad(qkv, None, None, q, k, torch.zeros_like(qkv), grad_v=v, eps=1e-5, workspace=torch.zeros(1, dtype=torch.uint8, device=device),
                                            **weights)


def _sample(device, which):
    x, u, t = torch.zeros(4, 50, device=device), torch.zeros(4, device=device), torch.ones(4, device=device)
    n = torch.zeros(4, dtype=torch.int32, device=device)
    dict(logits=x, uniforms=u, temperature=t)[which].requires_grad_()
    return lambda: rl.sample_tokens(x, u, n, temperature=t, workspace=torch.zeros(1, dtype=torch.uint8, device=device))


CALLS = [(_attention, w, back) for back in (False, True) for w in ("q", "k", "v", "out", "lse") + (("grad_out",) if back else ())]
CALLS += [(_norm, w, back) for back in (False, True) for w in ("qkv", "q", "k", "v", "q_weight", "k_weight")]
CALLS += [(_sample, w) for w in ("logits", "uniforms", "temperature")]


def _refused(call):
    with pytest.raises(ValueError, match="requires a gradient"):
        call()


@pytest.mark.parametrize("make, how", [(_attention, ("q", False)), (_attention, ("q", True)), (_norm, ("qkv", False)), (_norm, ("qkv", True)),
                                       (_sample, ("logits",))])
def test_what_requires_a_gradient_is_refused(make, how):
    call = make("cpu", *how)
    _refused(call)
    for mode in (torch.no_grad, torch.inference_mode):
        with mode(), pytest.raises(ValueError, match="on the GPU|on cuda"):
            call()


@pytest.mark.gpu
@pytest.mark.parametrize("make, how", [(c[0], c[1:]) for c in CALLS])
def test_wherever_it_stands(make, how):
    _refused(make("cuda", *how))
