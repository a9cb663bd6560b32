"""Attention over packed sequences and its gradient in 64 bits on the CPU, with how far a kernel may be from them by the roundings it makes.

A rounding to bf16 is off by at most 2^-8 of the value.  The kernels round the weights w (and z, of the gradient) to bf16 before their products and
the result once, so an output is off by at most 2^-8 (sum of |w v| / l + |out|).  What happens in fp32 comes on top: the scores' sums of 128 products,
off by at most 128 * 2^-24 of sum |q k| each, and a weight by that times the scale; the exponential's and the sums' own errors, 2^-18 of
each term, are far above what a chain of 2^-24's over some thousand terms makes of them.

Below 2^-126 fp32 has no normal numbers, and the exponential and the matrix instructions take such values for 0: a weight w is off by up to 2^-126
besides, z = w (dp - delta) by up to 2^-126 (|dp - delta| + 1), and a result by 2^-126.  (Scores far apart give gradients of 1e-38.)"""
import torch

BF16, FP32, TINY = 2.0 ** -8, 2.0 ** -18, 2.0 ** -126
D = 128


def spans(lengths, first=0):
    at, out = first, []
    for n in lengths:
        out.append((at, at + n))
        at += n
    return out


def admitted(n, full, sink, recent):
    i, j = torch.arange(n)[:, None], torch.arange(n)[None]
    return (j <= i) if full else (j <= i) & ((j < sink) | (i - j < recent))


def attention(q, k, v, lengths, mask, sink, recent, scale, first=0):
    """(out, lse, bound of out, bound of lse) [tokens, q heads, ...] of tensors on the CPU; rows of no sequence are 0."""
    q, k, v = (t.double() for t in (q, k, v))
    T, Hq, _ = q.shape
    group = Hq // k.shape[1]
    out, tol = torch.zeros(T, Hq, D, dtype=torch.float64), torch.zeros(T, Hq, D, dtype=torch.float64)
    lse, lse_tol = torch.zeros(Hq, T, dtype=torch.float64), torch.zeros(Hq, T, dtype=torch.float64)
    for a, b in spans(lengths, first):
        for h in range(Hq if b > a else 0):
            g = h // group
            s = scale * (q[a:b, h] @ k[a:b, g].t())
            near = admitted(b - a, mask[g], sink, recent)
            s = s.masked_fill(~near, float("-inf"))
            e = 2.0 ** -17 * scale * (q[a:b, h].abs() @ k[a:b, g].abs().t()).masked_fill(~near, 0).amax(-1, keepdim=True) + FP32
            p = torch.softmax(s, -1)
            out[a:b, h] = p @ v[a:b, g]
            far = p @ v[a:b, g].abs()
            tol[a:b, h] = (BF16 + 2 * e) * far + BF16 * out[a:b, h].abs() * (1 + BF16)
            lse[h, a:b] = torch.logsumexp(s, -1)
            lse_tol[h, a:b] = e[:, 0] + FP32 * lse[h, a:b].abs()
    return out, lse, tol, lse_tol


def gradient(q, k, v, out, lse, g, lengths, mask, sink, recent, scale, first=0):
    """((dq, dk, dv), their bounds) of the formulas, with out and lse as they are given."""
    q, k, v, out, lse, g = (t.double() for t in (q, k, v, out, lse, g))
    T, Hq, _ = q.shape
    H = k.shape[1]
    new = lambda n: torch.zeros(T, n, D, dtype=torch.float64)           # noqa: E731
    dq, dk, dv, tq, tk, tv = new(Hq), new(H), new(H), new(Hq), new(H), new(H)
    for a, b in spans(lengths, first):
        for h in range(Hq if b > a else 0):
            c = h * H // Hq
            qq, kk, vv, gg = q[a:b, h], k[a:b, c], v[a:b, c], g[a:b, h]
            near = admitted(b - a, mask[c], sink, recent)
            w = torch.exp(scale * (qq @ kk.t()) - lse[h, a:b, None]).masked_fill(~near, 0)
            e = 2.0 ** -17 * scale * (qq.abs() @ kk.abs().t()) + FP32 * (1 + lse[h, a:b, None].abs())
            dp, far = gg @ vv.t(), gg.abs() @ vv.abs().t()
            delta, dfar = (gg * out[a:b, h]).sum(-1, keepdim=True), (gg * out[a:b, h]).abs().sum(-1, keepdim=True)
            z = w * (dp - delta)
            ez = w * e * (dp - delta).abs() + w * FP32 * (far + dfar) + near * TINY * ((dp - delta).abs() + 1)
            dq[a:b, h] = scale * z @ kk
            tq[a:b, h] = scale * (BF16 * z.abs() + ez) @ kk.abs() * (1 + BF16) + BF16 * dq[a:b, h].abs()
            dk[a:b, c] += scale * z.t() @ qq
            tk[a:b, c] += scale * (BF16 * z.abs() + ez).t() @ qq.abs() * (1 + BF16)
            dv[a:b, c] += w.t() @ gg
            tv[a:b, c] += (BF16 * w + w * e + near * TINY).t() @ gg.abs() * (1 + BF16)
    return (dq, dk, dv), (tq, tk + BF16 * dk.abs(), tv + BF16 * dv.abs())


def near(x, y, tol):
    """Every value within its bound, none not a number."""
    far = (x.double().cpu() - y).abs()
    assert (far <= tol + TINY).all(), f"off by {far.max():.3g}, {(far / (tol + TINY)).max():.3g} of the bound"
