"""A recorded rotation runs at every replay over the lengths cached by then, whichever of the two copies of the lengths the appends in between
have left them in: the bits of every replay are those of the same call made then."""
import pytest
import torch

import paper_2510_08525_amd as rl

pytestmark = pytest.mark.gpu
D = 128


@pytest.mark.parametrize("dtype", [rl.RLKV_BF16, rl.RLKV_F32])
@pytest.mark.parametrize("counts", [None, [2, 0, 3]])
def test_replays_follow_the_lengths(dtype, counts):
    t = torch.bfloat16 if dtype == rl.RLKV_BF16 else torch.float32
    Hq, H, B, T = 8, 2, 3, 3
    c = rl.Cache(1, Hq, H, D, B, 4, 30, dtype, [1, 0], [400] * B)
    rot = rl.Rotary([500000.0 ** (-i / 64) for i in range(64)])
    qkv = torch.randn(B, T, (Hq + 2 * H) * D, device="cuda").to(t)
    new = lambda: [torch.full((B, h, T, D), 7.0, dtype=t, device="cuda") for h in (Hq, H, H)]       # noqa: E731
    kv = lambda n: [torch.randn(B, H, n, D, device="cuda").to(t) for _ in range(2)]                  # noqa: E731
    c.append_ragged(0, *kv(9), [9, 5, 2])
    eager, outs = new(), new()
    c.rotary(0, qkv, counts, rot, *eager)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.rotary(0, qkv, counts, rot, *outs)

    def check(what):
        qkv.copy_(torch.randn(B, T, (Hq + 2 * H) * D, device="cuda").to(t))
        for o in outs + eager:
            o.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        c.rotary(0, qkv, counts, rot, *eager)
        torch.cuda.synchronize()
        for a, b in zip(outs, eager):
            assert torch.equal(a, b), (what, c.lengths(0).tolist())

    check("as recorded")
    q, o = (torch.randn(B, Hq, D, device="cuda").to(t) for _ in range(2))
    for i in range(3):
        c.append(0, *kv(4))
        check("an append")
        c.append_rotary(0, qkv, [1, 0, 2], rot)
        check("a ragged append of rotated rows")
        c.append_decode(0, *kv(1), q, o, D ** -0.5)
        check("a step in one call")
    c.reset(1)
    check("one sequence reset")
    c.append_ragged(0, *kv(6), [0, 6, 1])
    check("and filled again")
    c.reset()
    check("all reset")
    c.append_ragged(0, *kv(200), [200, 1, 7])
    check("a prompt")
    c.close()
