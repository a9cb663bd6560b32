"""Attention over packed sequences whose scores are large: from 2^24 on a score in the log2 domain is a whole number, and its distance from the
product before its rounding grows beyond what an exponential takes (128 from 2^31 on)."""
import packed_reference as ref
import pytest
import torch

from test_gpu_packed_attention import BF, D, SCALE, inputs, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tail", [0, 17000])             # keys divided between the halves of a workgroup, and (beyond 256 workgroups) not
@pytest.mark.parametrize("size", [1e4, 1e6, 1e8, 3e9, 1e10, 1e15, 1e30])
def test_the_largest_score_has_all_the_weight(size, tail):
    """Scores of some `size`.  fp32 sums leave each within 2^-17 of scale sum |q k| (packed_reference.py), and where the largest admitted one is more than
    two of that and 60 above all others, those have e^-60 of the weight: the output is the largest one's value, rounded with its weight."""
    lengths, mask, sink, recent = [300, 40, 1], [0, 1], 5, 40
    q, k, v, _, offsets = inputs(lengths, 4, 2, seed=1, tail=tail)
    q = (q.float() * size).to(BF)
    out, lse = (t.cpu().double() for t in run(q, k, v, offsets, mask, sink, recent))
    clear = rows = 0
    for a, b in ref.spans(lengths):
        for h in range(4):
            near = ref.admitted(b - a, mask[h // 2], sink, recent)
            x, y, z = q[a:b, h].double(), k[a:b, h // 2].double(), v[a:b, h // 2].double()
            s = (SCALE * x @ y.t()).masked_fill(~near, float("-inf"))
            off = 2.0 ** -17 * SCALE * (x.abs() @ y.abs().t()).masked_fill(~near, 0).amax(-1)
            best, second = s.max(-1), s.scatter(1, s.argmax(-1, keepdim=True), float("-inf")).amax(-1)
            sure = best.values - second > 2 * off + 60
            got, want = out[a:b, h], z[best.indices]
            assert (got[sure] - want[sure]).abs().le(2 * ref.BF16 * (1 + ref.BF16) * want[sure].abs() + 1e-20).all()
            assert (got.abs() <= z.abs().max() * (1 + 2.0 ** -6)).all()                # (of the others: none is not a number)
            assert (lse[h, a:b] - torch.logsumexp(s, -1)).abs().le(off + ref.FP32 * (1 + best.values.abs())).all()
            clear, rows = clear + int(sure.sum()), rows + b - a
    assert clear > 0.9 * rows


@pytest.mark.parametrize("tail", [0, 5000])              # (16 heads)
def test_scores_that_rise_from_far_below(tail):
    """A first tile of keys whose scores are all some -2^33 to -2^31 in the log2 domain and whose values are so small that no product with them is
    infinite; the other keys' scores are 0, their values 1."""
    n = 128
    q, k, v = torch.zeros(n + tail, 16, D, dtype=BF), torch.zeros(n + tail, 1, D, dtype=BF), torch.ones(n + tail, 1, D, dtype=BF)
    q[:n, :, 0] = (2.0 ** 17 * (1 + 3 * torch.rand(n, 16, generator=torch.Generator().manual_seed(2)))).to(BF)
    k[:64, 0, 0], v[:64] = -(2.0 ** 17), 1e-25
    out, lse = run(q, k, v, torch.tensor([0, n], dtype=torch.int32))
    assert (out[64:n].cpu() == 1).all()
    want = torch.log(torch.arange(1.0, 65.0, dtype=torch.float64)).expand(16, 64)
    assert (lse[:, 64:n].cpu().double() - want).abs().max() <= ref.FP32 * (1 + want.max())
    assert (out[:64].cpu().float() - 1e-25).abs().max() <= 2 * ref.BF16 * 1e-25 * (1 + ref.BF16)


@pytest.mark.parametrize("tail", [0, 66000])
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
