"""Attention over packed sequences against 64 bits on the CPU (packed_reference.py has the bounds and where they come from)."""
import packed_reference as ref
import pytest
import torch

import paper_2510_08525_amd as rl

pytestmark = pytest.mark.gpu
D, BF = 128, torch.bfloat16
SCALE = D ** -0.5


def inputs(lengths, q_heads, kv_heads, seed=0, first=0, tail=0, scale_q=1.0):
    """q, k, v of packed projections, and the gradient of the output, on the CPU; offsets."""
    n = first + sum(lengths) + tail
    g = torch.Generator().manual_seed(seed)
    new = lambda h: torch.randn(n, h, D, generator=g).to(BF)                   # noqa: E731
    q, k, v, go = new(q_heads) * scale_q, new(kv_heads), new(kv_heads), new(q_heads)
    offsets = torch.tensor([first] + [b for _, b in ref.spans(lengths, first)], dtype=torch.int32)
    return q, k, v, go, offsets


def run(q, k, v, offsets, mask=None, sink=0, recent=0, scale=SCALE, out=None):
    q, k, v = (t.cuda() for t in (q, k, v))
    out = torch.full(q.shape, 7.0, dtype=BF, device="cuda") if out is None else out
    lse = torch.full((q.shape[1], q.shape[0]), 7.0, device="cuda")
    rl.packed_attention(q, k, v, offsets.cuda(), out, scale, lse=lse, mask=mask, sink=sink, recent=recent)
    torch.cuda.synchronize()
    return out, lse


def check(lengths, q_heads, kv_heads, mask=None, sink=0, recent=0, scale=SCALE, first=0, tail=0, seed=0, scale_q=1.0):
    q, k, v, _, offsets = inputs(lengths, q_heads, kv_heads, seed, first, tail, scale_q)
    out, lse = run(q, k, v, offsets, mask, sink, recent, scale)
    want, want_lse, tol, lse_tol = ref.attention(q, k, v, lengths, mask or [1] * kv_heads, sink, recent, scale, first)
    inside = slice(first, first + sum(lengths))
    ref.near(out[inside], want[inside], tol[inside])
    ref.near(lse[:, inside], want_lse[:, inside], lse_tol[:, inside])
    for rest in (slice(0, first), slice(first + sum(lengths), None)):              # rows of no sequence: left as they were
        assert (out[rest] == 7).all() and (lse[:, rest] == 7).all()


@pytest.mark.parametrize("q_heads, kv_heads", [(1, 1), (4, 4), (8, 2), (7, 1), (16, 1), (10, 2)])
@pytest.mark.parametrize("lengths", [[1], [1, 1, 1], [0, 5, 0, 0, 33, 0], [64], [63, 65, 1], [256, 300], [257]])
def test_lengths_and_groups(lengths, q_heads, kv_heads):
    check(lengths, q_heads, kv_heads, seed=len(lengths), first=len(lengths) % 3, tail=5 * (len(lengths) % 2))


@pytest.mark.parametrize("sink, recent", [(0, 1), (1, 1), (4, 60), (33, 70), (64, 256), (200, 3), (1000, 1000), (0, 2 ** 31 - 1), (2 ** 31 - 1, 1)])
def test_local_heads(sink, recent):
    check([700, 3, 129, 0, 300, 64], 8, 4, [1, 0, 0, 1], sink, recent)


def test_long_sequence():
    check([3000], 4, 1, [0], 64, 512)
    check([2000, 1100], 3, 1)


def test_many_short_sequences():
    check([i % 4 for i in range(1500)], 2, 1, [0], 1, 2, tail=3)              # more offsets than the kernel holds close by
    check([i % 7 for i in range(1022)], 2, 2, [0, 1], 1, 2)


def test_scores_far_apart():
    check([300, 40], 4, 2, scale=3.0, scale_q=2.0)
    check([300, 40], 4, 2, [0, 1], 5, 40, scale=1e-6)


def test_no_sequences_and_no_tokens():
    q, k, v, _, _ = inputs([5], 2, 1)
    out, lse = run(q, k, v, torch.tensor([0], dtype=torch.int32))
    assert (out == 7).all()
    out, lse = run(q[:0], k[:0], v[:0], torch.tensor([0, 0], dtype=torch.int32))
    out, lse = run(q, k, v, torch.tensor([3, 3, 3], dtype=torch.int32))
    assert (out == 7).all() and (lse == 7).all()


@pytest.mark.parametrize("offsets", [[0, -5, 40], [-3, 20, 20], [50, 20, 10], [0, 1000], [2 ** 31 - 1, 0, 2 ** 31 - 1], [-(2 ** 31), 2 ** 31 - 1], [90, 95]])
def test_offsets_that_make_no_sense_stay_inside_the_tensors(offsets):
    """The calls end, and rows around the tensors are as they were."""
    q, k, v, go, _ = inputs([60], 4, 2)
    whole = torch.full((200, 4, D), 7.0, dtype=BF, device="cuda")
    run(q, k, v, torch.tensor(offsets, dtype=torch.int32), [0, 1], 3, 9, out=whole[70:130])
    assert (whole[:70] == 7).all() and (whole[130:] == 7).all()


def test_strides():
    """Views of packed projections, heads in front, one row for all tokens: the same bits."""
    q, k, v, _, offsets = inputs([100, 33], 6, 2)
    want, want_lse = run(q, k, v, offsets)
    packed = torch.cat([q.view(133, -1), k.view(133, -1), v.view(133, -1), torch.zeros(133, 8, dtype=BF)], 1).cuda()
    a, b, c = packed[:, :6 * D].view(133, 6, D), packed[:, 6 * D:8 * D].view(133, 2, D), packed[:, 8 * D:10 * D].view(133, 2, D)
    front = torch.empty(6, 133, D, dtype=BF, device="cuda").transpose(0, 1)
    out, lse = run(a, b, c, offsets, out=front)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    one = v[:1].cuda().expand(133, 2, D)
    out, _ = run(q, k, one, offsets)
    same, _ = run(q, k, one.contiguous(), offsets)
    assert torch.equal(out, same)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("mask", [[1, 1], [0, 0]])
def test_what_is_not_admitted_does_not_count(bad, mask):
    """Values and keys at 4 places, and all rows behind the last sequence, are not finite: the rows that do not admit them keep their bits."""
    lengths, sink, recent = [40, 200, 7], 4, 30
    q, k, v, _, offsets = inputs(lengths, 4, 2, tail=20)
    want, want_lse = run(q, k, v, offsets, mask, sink, recent)
    rows = torch.ones(247, dtype=torch.bool)
    for place in (39, 100, 139, 246):
        v[place, :, 3::5] = bad
        k[place, 1, ::2] = bad
        a, b = next(s for s in ref.spans(lengths) if s[0] <= place < s[1])
        rows[a:b] &= ~ref.admitted(b - a, mask[0], sink, recent)[:, place - a]
    k[247:], v[247:], q[247:] = bad, bad, bad
    out, lse = run(q, k, v, offsets, mask, sink, recent)
    # (the products of a tile with such values are taken one by one, sums in another order: a rounding of fp32 may move one of bf16)
    keep = torch.cat([rows, torch.zeros(20, dtype=torch.bool)])
    want64, want_lse64, tol, lse_tol = ref.attention(torch.nan_to_num(q, 0, 0, 0), torch.nan_to_num(k, 0, 0, 0), torch.nan_to_num(v, 0, 0, 0), lengths,
                                                     mask, sink, recent, SCALE)
    ref.near(out[keep], want64[keep], tol[keep])
    ref.near(lse[:, keep], want_lse64[:, keep], lse_tol[:, keep])
    hit = ~torch.isfinite(out[:247, :, 3]).all(-1)
    assert (hit.cpu() == ~rows).all()
    assert (out[247:] == 7).all()


def test_equal_calls_give_equal_bits_also_on_another_stream():
    q, k, v, _, offsets = inputs([500, 77, 300], 8, 2)
    a = run(q, k, v, offsets, [0, 1], 10, 100)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        b = run(q, k, v, offsets, [0, 1], 10, 100)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_recorded_calls_take_the_offsets_of_the_replay():
    q, k, v, _, _ = inputs([200], 4, 2, tail=0)
    q, k, v = (t.cuda() for t in (q, k, v))
    offsets = torch.tensor([0, 200, 200, 200], dtype=torch.int32, device="cuda")
    out, lse = torch.zeros_like(q), torch.zeros(4, 200, device="cuda")
    call = lambda: rl.packed_attention(q, k, v, offsets, out, SCALE, lse=lse, mask=[0, 1], sink=4, recent=50)     # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for new in ([0, 200, 200, 200], [0, 70, 71, 190], [5, 5, 100, 200], [0, 1, 2, 3]):
        offsets.copy_(torch.tensor(new, dtype=torch.int32))
        out.fill_(3)
        lse.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone()
        out.fill_(3)
        lse.fill_(3)
        call()
        torch.cuda.synchronize()
        assert torch.equal(got[0], out) and torch.equal(got[1], lse)
