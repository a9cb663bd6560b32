"""The largest number of sequences that the packed attention takes, nearly all of them empty: places in the offsets of which no two, and no step between
them, may be added up in 31 bits."""
import pytest
import torch

from test_gpu_packed_attention import inputs, run
from test_gpu_packed_attention_grad import run as run_grad

pytestmark = pytest.mark.gpu
MOST = 2 ** 31 - 2


@pytest.mark.parametrize("at", [0, 12345, 2 ** 30 - 1, 2 ** 30 + 70, MOST - 1000, MOST - 3])
def test_attention_and_its_gradient(at):
    """Sequences number `at` and the two behind it, of 100, 0 and 200 tokens: the bits of a call with these three alone."""
    mask, sink, recent = [0, 1], 5, 40
    q, k, v, go, few = inputs([100, 0, 200], 4, 2)
    out, lse = run(q, k, v, few, mask, sink, recent)
    grads = run_grad(q, k, v, out, lse, go, few, mask, sink, recent)
    offsets = torch.empty(MOST + 1, dtype=torch.int32, device="cuda")
    offsets[:at + 1], offsets[at + 1:at + 3], offsets[at + 3:] = 0, 100, 300
    same, same_lse = run(q, k, v, offsets, mask, sink, recent)
    assert torch.equal(same, out) and torch.equal(same_lse, lse)
    assert all(torch.equal(x, y) for x, y in zip(run_grad(q, k, v, out, lse, go, offsets, mask, sink, recent), grads))
