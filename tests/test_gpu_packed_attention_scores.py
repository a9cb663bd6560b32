"""Attention over packed sequences whose scores are large: a score in the log2 domain is a product that fp32 rounds by far more than weights may be off."""
import packed_reference as ref
import pytest
import torch

from test_gpu_packed_attention import BF, D, SCALE, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tail", [0, 66000])             # keys divided between the halves of a workgroup, and (beyond 256 workgroups) not
@pytest.mark.parametrize("two", [4.0, 8.0, 16.0])
def test_two_large_scores_next_to_each_other(two, tail):
    """Two keys of a sequence, 97 apart, whose products with the queries are 2^25 to 2^26, the second's `two` more; all others' are 0.  Products are
    exact in fp32, so the weights' ratio is that of the formula to 2^-18; each is rounded to bf16, and so is the output."""
    n, where = 128, (3, 100)
    q, k, v = (torch.zeros(n + tail, 1, D, dtype=BF) for _ in range(3))
    q[:n, 0, 0], q[:, 0, 1] = 4096 * (1 + torch.arange(n) / 128), two / 2
    k[where[0], 0, 0] = k[where[1], 0, 0] = 8192
    k[where[1], 0, 1] = 2
    v[where[0]], v[where[1]] = 1, -1
    out, lse = run(q, k, v, torch.tensor([0, n], dtype=torch.int32))
    s = torch.tensor([0, two], dtype=torch.float64) * SCALE
    p = torch.softmax(s, 0)
    want = float(p[0] - p[1])
    assert (out[where[0]:where[1]].double().cpu() - 1).abs().max() <= 2 * ref.BF16
    assert (out[where[1]:n].double().cpu() - want).abs().max() <= ref.BF16 * (1 + abs(want)) + ref.FP32
    full = SCALE * q[where[1]:n, 0, 0].double() * 8192 + torch.logsumexp(s, 0)
    assert (lse[0, where[1]:n].double().cpu() - full).abs().le(ref.FP32 * full).all()
