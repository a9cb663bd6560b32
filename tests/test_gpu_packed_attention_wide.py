"""The cases of the packed attention's tests in buffers of so many rows that workgroups walk over their keys in one piece (small launches divide them
between the halves of a workgroup), and lengths around that change."""
import packed_reference as ref
import pytest
import torch

from test_gpu_packed_attention import D, SCALE, check, inputs, run

pytestmark = pytest.mark.gpu


def rows(q_heads):
    """More than 256 workgroups of 256 columns."""
    return 66000 // q_heads + 300


@pytest.mark.parametrize("q_heads, kv_heads", [(4, 4), (8, 2), (7, 1), (10, 2)])
@pytest.mark.parametrize("lengths", [[1], [1, 1, 1], [0, 5, 0, 0, 33, 0], [64], [63, 65, 1], [256, 300], [257]])
def test_lengths_and_groups(lengths, q_heads, kv_heads):
    check(lengths, q_heads, kv_heads, seed=len(lengths), first=len(lengths) % 3, tail=rows(q_heads))


@pytest.mark.parametrize("sink, recent", [(0, 1), (1, 1), (4, 60), (33, 70), (64, 256), (200, 3), (1000, 1000), (0, 2 ** 31 - 1), (2 ** 31 - 1, 1)])
def test_local_heads(sink, recent):
    check([700, 3, 129, 0, 300, 64], 8, 4, [1, 0, 0, 1], sink, recent, tail=rows(8))


def test_scores_far_apart():
    check([300, 40], 4, 2, scale=3.0, scale_q=2.0, tail=rows(4))
    check([300, 40], 4, 2, [0, 1], 5, 40, scale=1e-6, tail=rows(4))


@pytest.mark.parametrize("n", [64, 65, 128, 129, 191, 192, 193, 2047, 2048, 2049])
def test_lengths_around_a_tile(n):
    check([n], 32, 2, [1, 0], 70, 100, seed=n)                             # (up to 2048 rows the keys are divided)
    check([n - 1, 1], 16, 1, seed=n)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("mask", [[1, 1], [0, 0]])
@pytest.mark.parametrize("tail", [20, rows(4)])
def test_what_is_not_admitted_does_not_count(bad, mask, tail):
    """Not finite values in either half's tiles: the rows that do not admit them are what they are without."""
    lengths, sink, recent = [40, 200, 7], 4, 30
    q, k, v, _, offsets = inputs(lengths, 4, 2, tail=tail)
    keep = torch.ones(247, dtype=torch.bool)
    for place in (39, 70, 139, 200):
        v[place, :, 3::5] = bad
        k[place, 1, ::2] = bad
        a, b = next(s for s in ref.spans(lengths) if s[0] <= place < s[1])
        keep[a:b] &= ~ref.admitted(b - a, mask[0], sink, recent)[:, place - a]
    k[247:], v[247:], q[247:] = bad, bad, bad
    out, lse = run(q, k, v, offsets, mask, sink, recent)
    clean = [torch.nan_to_num(t[:247], 0, 0, 0) for t in (q, k, v)]
    want, want_lse, tol, lse_tol = ref.attention(*clean, lengths, mask, sink, recent, SCALE)
    ref.near(out[:247][keep], want[keep], tol[keep])
    ref.near(lse[:, :247][:, keep], want_lse[:, keep], lse_tol[:, keep])
    assert ((~torch.isfinite(out[:247, :, 3]).all(-1)).cpu() == ~keep).all()
    assert (out[247:] == 7).all()


def test_offsets_that_make_no_sense_stay_inside_the_tensors():
    n = 60 + rows(4)
    q, k, v, _, _ = inputs([n], 4, 2)
    whole = torch.full((n + 140, 4, D), 7.0, dtype=torch.bfloat16, device="cuda")
    for offsets in ([0, -5, 40], [50, 20, 10], [2 ** 31 - 1, 0, 2 ** 31 - 1], [-(2 ** 31), 2 ** 31 - 1]):
        run(q, k, v, torch.tensor(offsets, dtype=torch.int32), [0, 1], 3, 9, out=whole[70:n + 70])
        assert (whole[:70] == 7).all() and (whole[n + 70:] == 7).all()


@pytest.mark.parametrize("lengths", [[1500], [1000, 500], [750, 0, 750], [100] * 15, [1499, 1]])
def test_sequences_in_the_middle(lengths):
    """Between 128 and 256 workgroups, where it depends on the lengths whether keys are divided."""
    check(lengths, 28, 4, [1, 0, 0, 1], 30, 200, seed=len(lengths))
