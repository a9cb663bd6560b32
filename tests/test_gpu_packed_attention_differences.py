"""Gradient of the attention over packed sequences against differences of the attention itself in 64 bits.

Along the signs of a gradient the derivative is the sum of its sizes, to which the elements' bounds add up to less than a tenth of it, so that a gradient that is
0, of another size, or in part of another sign is none of it.  The bounds: those of the formulas (packed_reference.py) from out and lse as they are handed over,
and what out's rounding to bf16 leaves in delta, 2^-8 of sum |grad_out out|, spread over the admitted pairs by their weights."""
import packed_reference as ref
import pytest
import torch

from test_gpu_packed_attention import BF, SCALE, inputs

LENGTHS, SINK, RECENT = [60, 21, 1, 130], 3, 17


def case(mask, seed):
    """Inputs, the derivative along the signs of each gradient by differences, the signs and the sums of bounds."""
    q, k, v, go, offsets = inputs(LENGTHS, 4, 2, seed)
    out, lse, _, _ = ref.attention(q, k, v, LENGTHS, mask, SINK, RECENT, SCALE)
    out, lse = out.to(BF), lse.float()
    grads, tols = ref.gradient(q, k, v, out, lse, go, LENGTHS, mask, SINK, RECENT, SCALE)
    off = ref.BF16 * (go.double() * out.double()).abs().sum(-1)
    more = [torch.zeros_like(t) for t in tols]
    for a, b in ref.spans(LENGTHS):
        for h in range(4):
            x, y = q[a:b, h].double(), k[a:b, h // 2].double()
            w = torch.exp(SCALE * x @ y.t() - lse[h, a:b, None].double()).masked_fill(~ref.admitted(b - a, mask[h // 2], SINK, RECENT), 0) * off[a:b, h, None]
            more[0][a:b, h] += SCALE * w @ y.abs()
            more[1][a:b, h // 2] += SCALE * w.t() @ x.abs()
    ways, slopes = [g.sign() for g in grads], []
    for which, way in enumerate(ways):
        def f(step):
            x = [t.double() for t in (q, k, v)]
            x[which] = x[which] + step * way
            return (ref.attention(*x, LENGTHS, mask, SINK, RECENT, SCALE)[0] * go.double()).sum()
        # the step's square times a third derivative, taken out by a second step: what is left is of the fourth power
        near, far = (f(1e-4) - f(-1e-4)) / 2e-4, (f(2e-4) - f(-2e-4)) / 4e-4
        slopes.append(float(near + (near - far) / 3))
    # (a bound is one of every element; 1.05: the gradient that it is taken from is off by the same)
    bounds = [float((1.05 * (t + m) * w.abs()).sum()) + 1e-6 * abs(s) for t, m, w, s in zip(tols, more, ways, slopes)]
    return (q, k, v, out, lse, go, offsets), ways, slopes, bounds, grads


CASES = [([0, 1], 0), ([1, 1], 1), ([0, 0], 2)]


@pytest.mark.parametrize("mask, seed", CASES)
def test_what_the_bounds_leave(mask, seed):
    """The formulas' gradients meet them; none, half, the opposite, and one without a head, a sequence or a tenth of it do not."""
    _, ways, slopes, bounds, grads = case(mask, seed)
    for i, (g, way, slope, bound) in enumerate(zip(grads, ways, slopes, bounds)):
        assert 0 < bound < 0.1 * slope
        off = lambda x: abs(float((x * way).sum()) - slope)                     # noqa: E731
        assert off(g) <= bound
        headless, shorter = g.clone(), g.clone()
        headless[:, 0], shorter[:60] = 0, 0
        for wrong in (0 * g, g / 2, -g, headless, shorter, 0.9 * g, 1.1 * g):
            assert off(wrong) > bound


@pytest.mark.gpu
@pytest.mark.parametrize("mask, seed", CASES)
def test_against_differences(mask, seed):
    from test_gpu_packed_attention_grad import run

    (q, k, v, out, lse, go, offsets), ways, slopes, bounds, _ = case(mask, seed)
    for got, way, slope, bound in zip(run(q, k, v, out, lse, go, offsets, mask, SINK, RECENT), ways, slopes, bounds):
        assert abs(float((got.double().cpu() * way).sum()) - slope) <= bound
