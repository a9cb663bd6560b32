"""Gradient of the attention over packed sequences: against its formulas in 64 bits (packed_reference.py), against autograd, against differences."""
import packed_reference as ref
import pytest
import torch

import paper_2510_08525_amd as rl
from test_gpu_packed_attention import BF, D, SCALE, inputs

pytestmark = pytest.mark.gpu


def run(q, k, v, out, lse, go, offsets, mask=None, sink=0, recent=0, scale=SCALE, grads=None, workspace=None):
    q, k, v, out, lse, go = (t.cuda() for t in (q, k, v, out, lse, go))
    grads = [torch.full(t.shape, 7.0, dtype=BF, device="cuda") for t in (q, k, v)] if grads is None else grads
    rl.packed_attention_grad(q, k, v, offsets.cuda(), out, lse, go, *grads, scale, mask=mask, sink=sink, recent=recent, workspace=workspace)
    torch.cuda.synchronize()
    return grads


def prepared(lengths, q_heads, kv_heads, mask, sink, recent, scale=SCALE, first=0, tail=0, seed=0, scale_q=1.0):
    q, k, v, go, offsets = inputs(lengths, q_heads, kv_heads, seed, first, tail, scale_q)
    out, lse, _, _ = ref.attention(q, k, v, lengths, mask, sink, recent, scale, first)
    return q, k, v, out.to(BF), lse.float(), go, offsets


def check(lengths, q_heads, kv_heads, mask=None, sink=0, recent=0, scale=SCALE, first=0, tail=0, seed=0, scale_q=1.0):
    mask = mask or [1] * kv_heads
    q, k, v, out, lse, go, offsets = prepared(lengths, q_heads, kv_heads, mask, sink, recent, scale, first, tail, seed, scale_q)
    got = run(q, k, v, out, lse, go, offsets, mask, sink, recent, scale)
    want, tol = ref.gradient(q, k, v, out, lse, go, lengths, mask, sink, recent, scale, first)
    inside = slice(first, first + sum(lengths))
    for x, y, t in zip(got, want, tol):
        ref.near(x[inside], y[inside], t[inside])
        assert (x[:first] == 7).all() and (x[first + sum(lengths):] == 7).all()


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
    check([i % 4 for i in range(1500)], 2, 1, [0], 1, 2, tail=3)
    check([i % 7 for i in range(1022)], 2, 2, [0, 1], 1, 2)


def test_scores_far_apart():
    check([300, 40], 4, 2, scale=3.0, scale_q=2.0)
    check([300, 40], 4, 2, [0, 1], 5, 40, scale=1e-6)


@pytest.mark.parametrize("mask", [[1, 1], [0, 0], [0, 1]])
def test_against_autograd(mask):
    """Through the library's own forward pass, whose out is rounded: delta is off by 2^-8 of sum |grad_out out|, beside what the formulas allow."""
    lengths, sink, recent = [150, 31], 4, 40
    q, k, v, go, offsets = inputs(lengths, 6, 2)
    out, lse = torch.zeros(181, 6, D, dtype=BF, device="cuda"), torch.zeros(6, 181, device="cuda")
    rl.packed_attention(q.cuda(), k.cuda(), v.cuda(), offsets.cuda(), out, SCALE, lse=lse, mask=mask, sink=sink, recent=recent)
    got = run(q, k, v, out, lse, go, offsets, mask, sink, recent)
    x = [t.double().requires_grad_() for t in (q, k, v)]
    parts = []
    for a, b in ref.spans(lengths):
        for h in range(6):
            s = SCALE * x[0][a:b, h] @ x[1][a:b, h // 3].t()
            s = s.masked_fill(~ref.admitted(b - a, mask[h // 3], sink, recent), float("-inf"))
            parts.append((torch.softmax(s, -1) @ x[2][a:b, h // 3] * go[a:b, h].double()).sum())
    sum(parts).backward()
    _, tol = ref.gradient(q, k, v, out.cpu(), lse.cpu(), go, lengths, mask, sink, recent, SCALE)
    # what the rounding of out leaves in delta, spread over the admitted pairs
    off = 2 * ref.BF16 * (go.double() * out.double().cpu()).abs().sum(-1)
    more = [torch.zeros_like(t) for t in tol]
    for a, b in ref.spans(lengths):
        for h in range(6):
            w = torch.exp(SCALE * x[0][a:b, h].detach() @ x[1][a:b, h // 3].detach().t() - lse[h, a:b, None].cpu().double())
            w = w.masked_fill(~ref.admitted(b - a, mask[h // 3], sink, recent), 0) * off[a:b, h, None]
            more[0][a:b, h] += SCALE * w @ x[1][a:b, h // 3].detach().abs()
            more[1][a:b, h // 3] += SCALE * w.t() @ x[0][a:b, h].detach().abs()
    for y, t, m, u in zip(got, x, more, tol):
        ref.near(y, t.grad, u * 1.05 + m)


def test_against_differences():
    """The derivative of sum(out * grad_out) along a direction: central differences of the 64-bit forward, 1e-4 off by the step's square alone."""
    lengths, mask, sink, recent = [60, 21], [0, 1], 3, 17
    q, k, v, out, lse, go, offsets = prepared(lengths, 4, 2, mask, sink, recent)
    got = run(q, k, v, out, lse, go, offsets, mask, sink, recent)
    _, tol = ref.gradient(q, k, v, out, lse, go, lengths, mask, sink, recent, SCALE)
    g = torch.Generator().manual_seed(5)
    for which in range(3):
        way = torch.randn(got[which].shape, generator=g).double()
        def f(step):
            x = [t.double() for t in (q, k, v)]
            x[which] = x[which] + step * way
            return (ref.attention(*x, lengths, mask, sink, recent, SCALE)[0] * go.double()).sum()
        slope = (f(1e-4) - f(-1e-4)) / 2e-4
        # bounds of independent values add up as a random walk does at most where signs are random; taken whole they hold always
        assert abs((got[which].double().cpu() * way).sum() - slope) <= (2 * tol[which] * way.abs()).sum() + 1e-4 * abs(slope)


@pytest.mark.parametrize("offsets", [[0, -5, 40], [-3, 20, 20], [50, 20, 10], [0, 1000], [2 ** 31 - 1, 0, 2 ** 31 - 1], [-(2 ** 31), 2 ** 31 - 1], [90, 95]])
def test_offsets_that_make_no_sense_stay_inside_the_tensors(offsets):
    q, k, v, go, _ = inputs([60], 4, 2)
    whole = [torch.full((200, h, D), 7.0, dtype=BF, device="cuda") for h in (4, 2, 2)]
    run(q, k, v, q, torch.zeros(4, 60), go, torch.tensor(offsets, dtype=torch.int32), [0, 1], 3, 9, grads=[t[70:130] for t in whole])
    for t in whole:
        assert (t[:70] == 7).all() and (t[130:] == 7).all()


def test_strides():
    mask, lengths = [0, 1], [100, 33]
    q, k, v, out, lse, go, offsets = prepared(lengths, 6, 2, mask, 4, 30)
    want = run(q, k, v, out, lse, go, offsets, mask, 4, 30)
    packed = torch.cat([t.view(133, -1) for t in (q, k, v)], 1).cuda()
    a, b, c = packed[:, :6 * D].view(133, 6, D), packed[:, 6 * D:8 * D].view(133, 2, D), packed[:, 8 * D:].view(133, 2, D)
    front = lambda t: t.cuda().transpose(0, 1).contiguous().transpose(0, 1)                   # noqa: E731
    grad = torch.zeros(133, 10 * D, dtype=BF, device="cuda")
    grads = [grad[:, :6 * D].view(133, 6, D), torch.zeros(2, 133, D, dtype=BF, device="cuda").transpose(0, 1), grad[:, 8 * D:].view(133, 2, D)]
    got = run(a, b, c, front(out), lse, front(go), offsets, mask, 4, 30, grads=grads)
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    assert (grad[:, 6 * D:8 * D] == 0).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("mask", [[1, 1], [0, 0]])
def test_what_is_not_admitted_does_not_count(bad, mask):
    """One token's key and value, another's query and gradient are not finite, and all rows behind the last sequence: gradients that no admitted pair
    ties to them are as without."""
    lengths, sink, recent = [40, 200, 7], 4, 30
    q, k, v, out, lse, go, offsets = prepared(lengths, 4, 2, mask, sink, recent, tail=20)
    clean = [t.clone() for t in (q, k, v, out, lse, go)]
    near = torch.zeros(247, 247, dtype=torch.bool)
    for a, b in ref.spans(lengths):
        near[a:b, a:b] = ref.admitted(b - a, mask[0], sink, recent)
    k[100, :, ::3], v[100, :, 1::4] = bad, bad
    q[150, :, 5], go[150, :, ::7] = bad, bad
    for t in (q, k, v, out, go):
        t[247:] = bad
    lse[:, 247:] = bad
    got = run(q, k, v, out, lse, go, offsets, mask, sink, recent)
    want, tol = ref.gradient(*clean, lengths, mask, sink, recent, SCALE)
    free_q = ~near[:, 100]
    free_q[150] = False
    free_k = ~near[150] & ~near[free_q.logical_not().nonzero()[:, 0]].any(0)           # (rows that see key 100 pass it on)
    free_k[100] = False
    assert free_q.sum() > 90 and free_k.sum() > 40
    ref.near(got[0][:247][free_q], want[0][:247][free_q], tol[0][:247][free_q])
    for i in (1, 2):
        ref.near(got[i][:247][free_k], want[i][:247][free_k], tol[i][:247][free_k])
        assert (got[i][247:] == 7).all()
    assert not torch.isfinite(got[0][150]).any() and not torch.isfinite(got[1][100]).any()


def test_equal_calls_give_equal_bits_also_on_another_stream():
    mask = [0, 1]
    q, k, v, out, lse, go, offsets = prepared([300, 77, 200], 8, 2, mask, 10, 100)
    a = run(q, k, v, out, lse, go, offsets, mask, 10, 100)
    with torch.cuda.stream(torch.cuda.Stream()):
        b = run(q, k, v, out, lse, go, offsets, mask, 10, 100)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_recorded_calls_and_a_workspace_of_any_contents():
    mask = [0, 1]
    q, k, v, out, lse, go, offsets = (t.cuda() for t in prepared([150, 50], 4, 2, mask, 4, 50))
    grads = [torch.zeros_like(t) for t in (q, k, v)]
    work = torch.full((rl.rlkv_packed_attention_grad_workspace(200, 4, 2),), 255, dtype=torch.uint8, device="cuda")
    call = lambda: rl.packed_attention_grad(q, k, v, offsets, out, lse, go, *grads, SCALE, mask=mask, sink=4, recent=50, workspace=work)  # noqa: E731
    call()
    torch.cuda.synchronize()
    want = [t.clone() for t in grads]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for byte in (0, 255, 127):
        work.fill_(byte)
        for t in grads:
            t.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(grads, want))


@pytest.mark.parametrize("lengths", [[1500], [750, 0, 750], [100] * 15])
def test_sequences_in_the_middle(lengths):
    """Between 128 and 256 workgroups, where it depends on the lengths whether the queries' keys are divided."""
    check(lengths, 28, 4, [1, 0, 0, 1], 30, 200, seed=len(lengths))


@pytest.mark.parametrize("lengths, mask", [([1], None), ([0, 5, 0, 33, 0], None), ([63, 65, 1], None), ([300, 40, 129], [1, 0, 0, 1])])
def test_in_a_buffer_of_many_rows(lengths, mask):
    """More than 256 workgroups: keys are not divided."""
    check(lengths, 8, 4, mask, 33, 70, first=2, tail=8600, seed=len(lengths))


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("tail", [20, 16800])
def test_not_finite_rows_that_are_not_admitted(bad, tail):
    """In either half's tiles, with keys divided and not: gradients of rows that have nothing to do with them are what they are without."""
    lengths, mask, sink, recent = [200, 150], [0, 0], 4, 30
    q, k, v, go, offsets = inputs(lengths, 4, 2, tail=tail)
    out, lse, _, _ = ref.attention(q[:350], k[:350], v[:350], lengths, mask, sink, recent, SCALE)
    full = lambda t, fill: torch.cat([t, torch.full((tail, *t.shape[1:]), fill, dtype=t.dtype)])      # noqa: E731
    out, lse = full(out.to(BF), 0.0), torch.cat([lse.float(), torch.zeros(4, tail)], 1)
    clean = [t[:350].clone() for t in (q, k, v, go)]
    want, tol = ref.gradient(*clean[:3], out[:350], lse[:, :350], clean[3], lengths, mask, sink, recent, SCALE)
    v[70], k[70] = bad, bad                                             # (admitted by 70 .. 99 of the first sequence alone)
    q[350:], k[350:], v[350:], go[350:] = bad, bad, bad, bad
    got = run(q, k, v, out, lse, go, offsets, mask, sink, recent)
    rows = torch.ones(350, dtype=torch.bool)
    rows[70:100] = False                                                # queries that see it
    ref.near(got[0][:350][rows], want[0][rows], tol[0][rows])
    keys = torch.ones(350, dtype=torch.bool)
    keys[:4] = keys[41:100] = False                                     # keys that those queries see
    for x, y, t in zip(got[1:], want[1:], tol[1:]):
        ref.near(x[:350][keys], y[keys], t[keys])
    for x in got:
        assert (x[350:] == 7).all()
