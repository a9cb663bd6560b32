"""What the operators' calls write counts as changed in place, whatever the mode; inputs do not."""
import numpy as np
import pytest
import torch

import paper_2510_08525_amd as rl

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn


def _new(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype, device="cuda")


def _calls():
    """name -> (call, tensors it writes, tensors it reads)"""
    x, r, w, out, total = _new(4, 256), _new(4, 256), _new(256), _new(4, 256), _new(4, 256)
    q, s = _new(4, 256, dtype=torch.uint8).view(E4M3), _new(2, 4)
    b, sb, y = _new(128, 256, dtype=torch.uint8).view(E4M3), _new(1, 2), _new(4, 128)
    tokens, lp, h, lse = _new(4, dtype=torch.int32), _new(4), _new(4), _new(4)
    top, g, grad = (_new(4, 3), _new(4, 3, dtype=torch.int32)), _new(4), _new(4, 256)
    yield "rms_norm", lambda: rl.rms_norm(x, w, 1e-5, out, residual=r, sum_out=total), [out, total], [x, r, w]
    yield "8 bits", lambda: rl.rms_norm(x, w, 1e-5, q, scales=s), [q, s], [x, w]
    yield "quantize", lambda: rl.quantize(x, q, s), [q, s], [x]
    yield "scaled_matmul", lambda: rl.scaled_matmul(q, s, b, sb, y), [y], [q, s, b, sb]
    yield ("token_logprobs", lambda: rl.token_logprobs(x, tokens, lp, entropy=h, lse=lse, top=top), [lp, h, lse, *top], [x, tokens])
    yield ("token_logprobs_grad", lambda: rl.token_logprobs_grad(x, tokens, lse, g, grad, entropy=h, grad_entropy=g), [grad], [x, tokens, lse, h, g])


def test_versions_of_what_is_written():
    for name, call, writes, reads in _calls():
        before = [t._version for t in writes], [t._version for t in reads]
        call()
        with torch.no_grad():
            call()
        assert [t._version for t in writes] == [v + 2 for v in before[0]], name
        assert [t._version for t in reads] == before[1], name
    torch.cuda.synchronize()


def test_versions_of_a_caches_outputs():
    c = rl.Cache(1, 4, 2, 128, 2, 4, 16, rl.RLKV_BF16, [1, 0], [20] * 2)
    rot = rl.Rotary([1.0] * 64)
    qkv = _new(2, 3, 8 * 128, dtype=torch.bfloat16)
    q, k, v = (_new(2, h, 3, 128, dtype=torch.bfloat16) for h in (4, 2, 2))
    c.rotary(0, qkv, None, rot, q, k, v)
    c.append_rotary(0, qkv, np.array([3, 1]), rot, q)
    c.append_rotary(0, qkv, None, rot)
    torch.cuda.synchronize()
    assert (q._version, k._version, v._version, qkv._version) == (2, 1, 1, 0)
    c.close()


def test_a_refused_call_writes_nothing():
    x, s = _new(4, 256), _new(2, 4)
    with pytest.raises(rl.RlkvError):
        rl.rms_norm(x, None, -1.0, x)
    assert x._version == 0 and s._version == 0


def test_what_autograd_saved_is_known_to_be_gone():
    """The gradient over the logits themselves, which the caller's graph still needs."""
    z = torch.randn(4, 256, device="cuda", requires_grad=True)
    x = z * 1.0
    loss = (x * x).sum()
    tokens, one = _new(4, dtype=torch.int32), torch.ones(4, device="cuda")
    with torch.no_grad():
        rl.token_logprobs_grad(x.detach(), tokens, one, one, x)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_tensors_of_inference_mode():
    with torch.inference_mode():
        x, out = torch.randn(4, 256, device="cuda"), _new(4, 256)
        rl.rms_norm(x, None, 1e-5, out)
    rl.rms_norm(x, None, 1e-5, out)
    y = x / (x.pow(2).mean(1, keepdim=True) + 1e-5).sqrt()
    assert torch.allclose(out, y, rtol=1e-5, atol=1e-6)
