"""Operators of the policy's training loop whose speed is measured, next to those of operators.py: rollouts are sampled, then the policy is
updated on them, packed one behind the other.

  sample      tokens drawn from rows of logits by given random numbers: temperature, top-k, top-p, min-p, and the log probability of
              the token in the distribution it was drawn from
  heads       packed projections as the attention takes them: norm of every query and key head, rotation by given positions
  heads_grad  the way back, with the gradients of the norms' weights
  attn        attention over whole sequences packed one behind the other, under the causal mask (full heads) or the local one (sinks and
              recent positions), with log-sum-exp
  attn_grad   its way back: gradients of queries, keys and values

Shapes are those of the library's own workloads (32 query / 8 KV heads and 28 / 4, head_dim 128) and generic ones.  `run` computes the
plain form, or with `own` calls the library.
"""
import math

import torch

own = False

D = 128
SCALE = 1.0 / math.sqrt(D)
EPS = 1e-6
SCORES = 2 ** 31          # scores that the plain attention holds at once


# ---- the cases ---------------------------------------------------------------------------------------------------

def _sample(name, rows, vocab, dtype="bf16", temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, per_row=False, masked=False):
    """per_row: every request of the batch brings its own temperature and filters, spread around the given ones."""
    return dict(name=name, kind="sample", rows=rows, vocab=vocab, dtype=dtype, temperature=temperature, top_k=top_k, top_p=top_p,
                min_p=min_p, per_row=per_row, masked=masked)


def _heads(name, kind, tokens, q_heads, kv_heads, dtype="bf16", norm=True, rotary=D, interleaved=False, values=False):
    return dict(name=name, kind=kind, tokens=tokens, q_heads=q_heads, kv_heads=kv_heads, dtype=dtype, norm=norm, rotary=rotary,
                interleaved=interleaved, values=values)


def _attn(name, kind, q_heads, kv_heads, pct, batch, lo, hi, sink=64, recent=256, tail=0):
    """pct: of the KV heads, how many see sinks and recent positions only; tail: rows of the buffers behind the last sequence."""
    return dict(name=name, kind=kind, q_heads=q_heads, kv_heads=kv_heads, pct=pct, batch=batch, lo=lo, hi=hi, sink=sink, recent=recent,
                tail=tail)


def listed():
    return [
        # One user's next token under a usual setting: latency.
        _sample("sample_b1", 1, 131072, "f32", 0.7, 0, 0.95),
        # A serving batch whose requests all have filters of their own; a vocabulary of odd size.
        _sample("sample_requests_48", 48, 128011, "f32", 0.8, 50, 0.9, 0.05, per_row=True),
        # A step of a rollout batch: the policy itself, without filters.
        _sample("sample_rollouts_512", 512, 131072),
        # One user's decode step of a layer, what stands between the projections and the fused append and attention.  The smallest call.
        _heads("heads_b1", "heads", 1, 32, 8, values=True),
        # A batch of packed rollouts.
        _heads("heads_16k", "heads", 16384, 28, 4),
        # The same way back, for one short answer and for the batch.
        _heads("heads_grad_333", "heads_grad", 333, 28, 4),
        _heads("heads_grad_16k", "heads_grad", 16384, 32, 8),
        # One short prompt.
        _attn("attn_333", "attn", 28, 4, 0, 1, 333, 333),
        # Ragged rollouts under a mask with half the KV heads local, behind them the rest of a buffer of fixed size.
        _attn("attn_packed_24_100_2000", "attn", 28, 4, 50, 24, 100, 2000, tail=77),
        # A long reasoning trace, every head full: the largest product.
        _attn("attn_16k", "attn", 32, 8, 0, 1, 16384, 16384),
        # The update on short ragged answers, and on a long trace of which half the heads are local.
        _attn("attn_grad_packed_12_50_700", "attn_grad", 28, 4, 50, 12, 50, 700),
        _attn("attn_grad_2x8k", "attn_grad", 32, 8, 50, 2, 8192, 8192, 64, 512),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["sample", "sample", "sample", "heads", "heads", "heads_grad", "heads_grad", "attn", "attn", "attn", "attn_grad",
                       "attn_grad", "attn_grad"])
    if kind == "sample":
        vocab = _log_int(rng, 1000, 262144)
        rows = _log_int(rng, 1, min(512, 2 ** 26 // vocab))
        c = _sample("", rows, vocab, rng.choice(["bf16", "f32"]), rng.choice([0.0, 0.3, 0.6, 0.8, 1.0, 1.0, 1.0, 1.3]),
                    rng.choice([0, 0, 0, 1, 20, 50, 1000]), rng.choice([1.0, 1.0, 0.95, 0.9, 0.5]), rng.choice([0.0, 0.0, 0.02, 0.1]),
                    rng.random() < 0.4, rng.random() < 0.2)
        if c["dtype"] == "f32":
            c["rows"] = max(1, rows // 2)
    else:
        q_heads, kv_heads = rng.choice([(32, 8), (28, 4), (32, 8), (28, 4), (8, 8), (12, 4), (16, 1)])
        if kind in ("heads", "heads_grad"):
            c = _heads("", kind, _log_int(rng, 1, 16384 * 36 // (q_heads + 2 * kv_heads + 4)), q_heads, kv_heads,
                       rng.choice(["bf16", "bf16", "f32"]), rng.random() < 0.75, rng.choice([128, 128, 128, 64, 32, 96]),
                       rng.random() < 0.3, kind == "heads" and rng.random() < 0.3)
            if c["dtype"] == "f32":
                c["tokens"] = max(1, c["tokens"] // 2)
        else:
            batch = _log_int(rng, 1, 64)
            hi = _log_int(rng, 1, (16384 if kind == "attn" else 8192) // batch)
            sink, recent = rng.choice([(16, 112), (64, 256), (64, 512), (33, 70), (4, 1000), (0, 1)])
            c = _attn("", kind, q_heads, kv_heads, rng.choice([0, 0, 25, 50, 75, 100]), batch, rng.randint(0, hi), hi, sink, recent,
                      rng.choice([0, 0, 5, 300]))
    del c["name"]
    return c


# ---- inputs ------------------------------------------------------------------------------------------------------

def _dtype(name):
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def _gen(seed, what):
    return torch.Generator(device="cuda").manual_seed(seed * 16 + what)


def _randn(seed, what, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=_gen(seed, what), device="cuda", dtype=dtype)


def _rand(seed, what, *shape):
    return torch.rand(*shape, generator=_gen(seed, what), device="cuda")


def _lengths(c):
    """Length of every sequence: spread over [lo, hi] in a scattered order, the first one the longest."""
    n, lo, hi = c["batch"], c["lo"], c["hi"]
    return [hi if b == 0 else lo + int((hi - lo) * ((b * 0.6180339887498949 + 0.5) % 1.0) + 0.5) for b in range(n)]


def _mask(c):
    """[kv_heads], 1 = full."""
    n = c["pct"] * c["kv_heads"] // 100
    return [0 if h < n else 1 for h in range(c["kv_heads"])]


def _inv_freq(c):
    half = c["rotary"] // 2
    return [500000.0 ** (-i / half) for i in range(half)]


def _sample_inputs(c, seed):
    """Logits of rows that are more and less sure of what comes next, in a padded buffer as a projection leaves them."""
    R, V, dt = c["rows"], c["vocab"], _dtype(c["dtype"])
    sharp = 1.5 * 2.5 ** _rand(seed, 1, R, 1)
    x = torch.zeros(R, -(-V // 64) * 64, device="cuda", dtype=dt)[:, :V]
    x.copy_(_randn(seed, 2, R, V) * sharp)
    if c["masked"]:                                                            # an answer of a given form: most tokens are forbidden
        off = _rand(seed, 3, V) < 0.7
        off[V // 2] = False
        x.masked_fill_(off, -math.inf)
    u = _rand(seed, 4, R)
    T, k, p, m = c["temperature"], c["top_k"], c["top_p"], c["min_p"]
    if c["per_row"]:
        T = T * (0.5 + _rand(seed, 5, R))
        k = (k * 2 * _rand(seed, 6, R)).int()                                  # (0: this request has no such limit)
        p = torch.where(_rand(seed, 7, R) < 0.25, 1.0, p * (0.9 + 0.1 * _rand(seed, 8, R)))
        m = m * (2 * _rand(seed, 9, R) - 0.5).clamp(min=0)
    return x, u, (T, k, p, m)


def _heads_inputs(c, seed):
    """Packed projections of sequences one behind the other, with the positions that go with them."""
    T, Hq, H, dt = c["tokens"], c["q_heads"], c["kv_heads"], _dtype(c["dtype"])
    qkv = _randn(seed, 1, T, (Hq + 2 * H) * D, dtype=dt) * 1.5
    pos = torch.arange(T, device="cuda", dtype=torch.int32)
    pos = pos % (T // 3 + 1) + (4000 if T == 1 else 0)
    w = [(1 + 0.2 * _randn(seed, 2 + i, D)).to(dt) if c["norm"] else None for i in range(2)]
    dq, dk = _randn(seed, 4, T, Hq, D, dtype=dt), _randn(seed, 5, T, H, D, dtype=dt)
    return qkv, pos, w, dq, dk


def _attn_inputs(c, seed):
    """Queries and keys as the rotation leaves them, values where the projections have them; keys of the first positions larger, as sinks are."""
    n, Hq, H = sum(_lengths(c)) + c["tail"], c["q_heads"], c["kv_heads"]
    q = _randn(seed, 1, n, Hq, D, dtype=torch.bfloat16)
    k = _randn(seed, 2, n, H, D, dtype=torch.bfloat16)
    at = 0
    for length in _lengths(c):
        k[at:at + min(4, length)] *= 2
        at += length
    v = _randn(seed, 3, n, (Hq + 2 * H) * D, dtype=torch.bfloat16)[:, (Hq + H) * D:].view(n, H, D)
    g = _randn(seed, 4, n, Hq, D, dtype=torch.bfloat16)
    return q, k, v, g


class State:
    pass


def prepare(case, seed):
    c, s = case, State()
    s.case = c
    new = lambda *shape, dtype: torch.zeros(*shape, device="cuda", dtype=dtype)          # noqa: E731
    if c["kind"] == "sample":
        s.x, s.u, s.how = _sample_inputs(c, seed)
        s.tokens, s.logprobs = new(c["rows"], dtype=torch.int32), new(c["rows"], dtype=torch.float32)
        if own:
            import paper_2510_08525_amd as rl

            s.workspace = new(max(1, rl.rlkv_sample_tokens_workspace(c["rows"], c["vocab"])), dtype=torch.uint8)
    elif c["kind"] in ("heads", "heads_grad"):
        T, Hq, H, dt = c["tokens"], c["q_heads"], c["kv_heads"], _dtype(c["dtype"])
        s.qkv, s.pos, (s.wq, s.wk), s.dq, s.dk = _heads_inputs(c, seed)
        s.inv_freq = torch.tensor(_inv_freq(c), device="cuda", dtype=torch.float64)
        if c["kind"] == "heads":
            s.q, s.k = new(T, Hq, D, dtype=dt), new(T, H, D, dtype=dt)
            s.v = new(T, H, D, dtype=dt) if c["values"] else None
        else:
            s.dqkv = new(T, (Hq + 2 * H) * D, dtype=dt)                        # (the values' columns: what the attention left there)
            s.dwq, s.dwk = (new(D, dtype=torch.float32) if c["norm"] else None for _ in range(2))
        if own:
            import paper_2510_08525_amd as rl

            s.rotary = rl.Rotary(_inv_freq(c), interleaved=c["interleaved"])
            s.workspace = new(max(1, rl.rlkv_head_norm_rotary_grad_workspace(T, Hq, H)), dtype=torch.uint8)
    else:
        Hq, H, ns = c["q_heads"], c["kv_heads"], _lengths(c)
        n, bf = sum(ns) + c["tail"], torch.bfloat16
        s.q, s.k, s.v, s.g = _attn_inputs(c, seed)
        s.offsets = torch.tensor([sum(ns[:i]) for i in range(len(ns) + 1)], device="cuda", dtype=torch.int32)
        s.seq = torch.repeat_interleave(torch.arange(len(ns), device="cuda"), torch.tensor(ns, device="cuda"))
        s.pos = torch.arange(sum(ns), device="cuda") - s.offsets.long()[s.seq]
        s.local = ~torch.tensor(_mask(c), device="cuda", dtype=torch.bool)
        s.out, s.lse = new(n, Hq, D, dtype=bf), new(Hq, n, dtype=torch.float32)
        if c["kind"] == "attn_grad":
            s.out, s.lse = _plain_attention(s)
            s.dq, s.dk = new(n, Hq, D, dtype=bf), new(n, H, D, dtype=bf)
            s.dv = new(n, (Hq + 2 * H) * D, dtype=bf)[:, (Hq + H) * D:].view(n, H, D)
            if own:
                import paper_2510_08525_amd as rl

                s.workspace = new(max(1, rl.rlkv_packed_attention_grad_workspace(n, Hq, H)), dtype=torch.uint8)
    torch.cuda.synchronize()
    return s


def run(s):
    return _run_own(s) if own else _run_plain(s)


# ---- the library's calls -------------------------------------------------------------------------------------------

def _run_own(s):
    import paper_2510_08525_amd as rl

    c = s.case
    if c["kind"] == "sample":
        T, k, p, m = s.how
        rl.sample_tokens(s.x, s.u, s.tokens, temperature=T, top_k=k, top_p=p, min_p=m, logprobs=s.logprobs, workspace=s.workspace)
        return [s.tokens, s.logprobs]
    eps = EPS if c.get("norm") else None
    if c["kind"] == "heads":
        rl.head_norm_rotary(s.qkv, s.pos, s.rotary, s.q, s.k, v_out=s.v, q_weight=s.wq, k_weight=s.wk, eps=eps)
        return [s.q, s.k, s.v]
    if c["kind"] == "heads_grad":
        rl.head_norm_rotary_grad(s.qkv, s.pos, s.rotary, s.dq, s.dk, s.dqkv, q_weight=s.wq, k_weight=s.wk, eps=eps,
                                 grad_q_weight=s.dwq, grad_k_weight=s.dwk, workspace=s.workspace)
        return [s.dqkv, s.dwq, s.dwk]
    how = dict(mask=_mask(c), sink=c["sink"], recent=c["recent"])
    if c["kind"] == "attn":
        rl.packed_attention(s.q, s.k, s.v, s.offsets, s.out, SCALE, lse=s.lse, **how)
        return [s.out, s.lse]
    rl.packed_attention_grad(s.q, s.k, s.v, s.offsets, s.out, s.lse, s.g, s.dq, s.dk, s.dv, SCALE, workspace=s.workspace, **how)
    return [s.dq, s.dk, s.dv]


# ---- the plain form ------------------------------------------------------------------------------------------------

def _plain_sample(s):
    """Weights and their sums in 64 bits: a random number falls next to a border of two tokens now and then."""
    R, V = s.x.shape
    T, k, p, min_p = (torch.as_tensor(v, device="cuda").double().expand(R)[:, None] for v in s.how)
    x, best = s.x.double(), s.x.double().amax(-1, keepdim=True)
    w = torch.where(T > 0, torch.exp((x - best) / torch.where(T > 0, T, 1.0)), (x == best).double())
    order = torch.sort(s.x, dim=-1, descending=True, stable=True).indices
    ws = w.gather(1, order)
    rank = torch.arange(V, device="cuda")
    keep = torch.where(T > 0, (rank < k) | (k <= 0), rank < 1)
    ws = torch.where(keep, ws, 0.0)
    cum = torch.cumsum(ws, -1)
    before = torch.cat([torch.zeros_like(best), cum[:, :-1]], -1)
    keep = keep & ((before < p * cum[:, -1:]) | (p >= 1)) & (ws >= min_p)
    keep[:, 0] = True
    w = torch.where(torch.zeros_like(keep).scatter(1, order, keep), w, 0.0)
    cum = torch.cumsum(w, -1)
    total = cum[:, -1:]
    token = (cum <= s.u.double()[:, None] * total).sum(-1, keepdim=True).clamp(max=V - 1)
    return [token[:, 0].int(), torch.log(w.gather(1, token) / total)[:, 0].float()]


def _plain_turn(x, pos, inv_freq, interleaved):
    """x [T, heads, D] in 32 bits; angles in 64 bits."""
    half = inv_freq.numel()
    angle = pos.double()[:, None, None] * inv_freq
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    r = x.clone()
    if interleaved:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        r[..., 0:2 * half:2], r[..., 1:2 * half:2] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., :half], x[..., half:2 * half]
        r[..., :half], r[..., half:2 * half] = a * cos - b * sin, b * cos + a * sin
    return r


def _plain_heads(s, x, w):
    y = x.float()
    if w is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * w.float()
    return _plain_turn(y, s.pos, s.inv_freq, s.case["interleaved"]).to(x.dtype)


def _plain_heads_grad(s, x, w, g):
    """(gradient of the heads, of the weight)"""
    g = _plain_turn(g.float(), -s.pos, s.inv_freq, s.case["interleaved"])
    if w is None:
        return g.to(x.dtype), None
    y = x.float()
    r = torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS)
    unit, gw = y * r, g * w.float()
    return ((gw - unit * (gw * unit).mean(-1, keepdim=True)) * r).to(x.dtype), (g * unit).sum((0, 1))


def _padded(s, x):
    """[rows, heads, D] of the packed sequences as [sequences, heads, longest, D] in 32 bits."""
    c = s.case
    p = torch.zeros(c["batch"], c["hi"], x.shape[1], D, device="cuda")
    p[s.seq, s.pos] = x[:s.seq.numel()].float()
    return p.transpose(1, 2).contiguous()


def _packed(s, p, like):
    """The way back, rounded; rows behind the last sequence are zero."""
    out = torch.zeros_like(like)
    out[:s.seq.numel()] = p.transpose(1, 2)[s.seq, s.pos].to(like.dtype)
    return out


def _admitted(s):
    """[kv heads, 1, longest, longest]"""
    c = s.case
    j = torch.arange(c["hi"], device="cuda")
    i = j[:, None]
    near = (j <= i) & ((j < c["sink"]) | (i - j < c["recent"]))
    return torch.where(s.local[:, None, None, None], near, j <= i)


def _kv_heads_at_once(c):
    return max(1, min(c["kv_heads"], SCORES // (c["batch"] * c["hi"] ** 2 * (c["q_heads"] // c["kv_heads"]))))


def _plain_attention(s):
    c = s.case
    B, L, H, step = c["batch"], c["hi"], c["kv_heads"], _kv_heads_at_once(c)
    q, k, v, admit = _padded(s, s.q).view(B, H, -1, D), _padded(s, s.k), _padded(s, s.v), _admitted(s)
    out, lse = torch.empty_like(q), torch.empty(B, H, q.shape[2], device="cuda")
    for h in range(0, H, step):                                                # (all heads at once unless memory forbids)
        part = slice(h, h + step)
        x = torch.matmul(q[:, part] * SCALE, k[:, part].transpose(-1, -2).contiguous()).view(B, -1, c["q_heads"] // H, L, L)
        x = x.masked_fill_(~admit[part], -math.inf)
        best = x.amax(-1, keepdim=True)
        p = torch.exp_(x.sub_(best))
        total = p.sum(-1, keepdim=True)
        out[:, part] = torch.matmul(p.view(B, -1, q.shape[2], L), v[:, part]) / total.view(B, -1, q.shape[2], 1)
        lse[:, part] = (best + torch.log(total)).view(B, -1, q.shape[2])
    rows = torch.zeros(c["q_heads"], s.q.shape[0], device="cuda")
    rows[:, :s.seq.numel()] = lse.view(B, -1, L).transpose(0, 1)[:, s.seq, s.pos]
    return _packed(s, out.view(B, -1, L, D), s.q), rows


def _plain_attention_grad(s):
    c = s.case
    B, L, H, step = c["batch"], c["hi"], c["kv_heads"], _kv_heads_at_once(c)
    G = c["q_heads"] // H
    q, g, o = (_padded(s, t).view(B, H, G * L, D) for t in (s.q, s.g, s.out))
    k, v, admit = _padded(s, s.k), _padded(s, s.v), _admitted(s)
    lse = torch.zeros(B, L, c["q_heads"], device="cuda")
    lse[s.seq, s.pos] = s.lse[:, :s.seq.numel()].t()
    lse = lse.transpose(1, 2).reshape(B, H, G * L, 1)
    delta = (g * o).sum(-1, keepdim=True)
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    for h in range(0, H, step):                                                # (all heads at once unless memory forbids)
        part = slice(h, h + step)
        p = torch.matmul(q[:, part] * SCALE, k[:, part].transpose(-1, -2).contiguous())
        p = torch.exp_(p.sub_(lse[:, part])).view(B, -1, G, L, L).masked_fill_(~admit[part], 0.0).view(B, -1, G * L, L)
        dv[:, part] = torch.matmul(p.transpose(-1, -2), g[:, part])
        d = torch.matmul(g[:, part], v[:, part].transpose(-1, -2).contiguous()).sub_(delta[:, part]).mul_(p)
        dq[:, part] = torch.matmul(d, k[:, part]) * SCALE
        dk[:, part] = torch.matmul(d.transpose(-1, -2), q[:, part]) * SCALE
    return [_packed(s, dq.view(B, -1, L, D), s.q), _packed(s, dk, s.k), _packed(s, dv, s.k)]


def _run_plain(s):
    c = s.case
    if c["kind"] == "sample":
        return _plain_sample(s)
    if c["kind"] in ("heads", "heads_grad"):
        x = s.qkv.view(c["tokens"], -1, D)
        Hq, H = c["q_heads"], c["kv_heads"]
        q, k, v = x[:, :Hq], x[:, Hq:Hq + H], x[:, Hq + H:]
        if c["kind"] == "heads":
            return [_plain_heads(s, q, s.wq), _plain_heads(s, k, s.wk), v.clone() if c["values"] else None]
        dq, dwq = _plain_heads_grad(s, q, s.wq, s.dq)
        dk, dwk = _plain_heads_grad(s, k, s.wk, s.dk)
        return [torch.cat([dq, dk, torch.zeros_like(v)], 1).view(c["tokens"], -1), dwq, dwk]
    return list(_plain_attention(s)) if c["kind"] == "attn" else _plain_attention_grad(s)


# ---- what a pass cannot do without -----------------------------------------------------------------------------------

def _pairs(c):
    """Admitted pairs of a query and a key, over all query heads."""
    S, W = c["sink"], c["sink"] + c["recent"]
    full = sum(n * (n + 1) // 2 for n in _lengths(c))
    near = sum(min(n, W) * (min(n, W) + 1) // 2 + max(0, n - W) * W for n in _lengths(c))
    return c["q_heads"] // c["kv_heads"] * sum(full if f else near for f in _mask(c))


def work(case):
    c = case
    e = {"f32": 4, "bf16": 2}.get(c.get("dtype"), 2)
    if c["kind"] == "sample":
        n = c["rows"] * c["vocab"]
        return {"bytes": n * e + 12 * c["rows"], "flops": 20 * n}
    Hq, H = c["q_heads"], c["kv_heads"]
    if c["kind"] in ("heads", "heads_grad"):
        n = c["tokens"] * (Hq + H) * D
        if c["kind"] == "heads":
            return {"bytes": 2 * e * (n + c["values"] * c["tokens"] * H * D) + 4 * c["tokens"], "flops": 8 * n}
        return {"bytes": (3 if c["norm"] else 2) * e * n + 4 * c["tokens"], "flops": 16 * n}
    n = sum(_lengths(c))
    if c["kind"] == "attn":
        return {"bytes": 2 * n * (2 * Hq + 2 * H) * D + 4 * n * Hq, "flops": 4 * D * _pairs(c)}
    return {"bytes": 2 * n * (4 * Hq + 4 * H) * D + 4 * n * Hq, "flops": 10 * D * _pairs(c)}


# ---- the same in 64 bits ---------------------------------------------------------------------------------------------

def _exact_sample(c, seed):
    """Row by row from the definition: thresholds instead of positions in a sorted row."""
    x, u, how = _sample_inputs(c, seed)
    logprobs = []
    T, k, p, m = (torch.as_tensor(v, device="cuda").double().expand(c["rows"]).tolist() for v in how)
    for r in range(c["rows"]):
        z = x[r].double()
        if T[r] <= 0:
            logprobs.append(torch.zeros((), device="cuda", dtype=torch.float64))
            continue
        z = torch.log_softmax(z / T[r], 0)
        # equal logits stand in order of their tokens
        ranked = torch.argsort(torch.argsort(-x[r].double(), stable=True))
        kept = ranked < (k[r] if k[r] > 0 else z.numel())
        if p[r] < 1:
            q = torch.softmax(torch.where(kept, z, -math.inf), 0)
            q_sorted = torch.zeros_like(q).scatter(0, ranked, q)
            enough = torch.cumsum(q_sorted, 0)
            n = int((enough < p[r]).sum()) + 1
            kept &= ranked < n
        kept &= (torch.exp(z - z.max()) >= m[r]) | (ranked == 0)
        q = torch.softmax(torch.where(kept, z, -math.inf), 0)
        i = torch.searchsorted(torch.cumsum(q, 0), u[r].double(), right=True).clamp(max=z.numel() - 1)
        logprobs.append(torch.log(q[i]))
    return [None, torch.stack(logprobs)]


def _turned64(c, x, pos):
    """x [T, heads, D] in 64 bits, as products of complex numbers."""
    f = torch.tensor(_inv_freq(c), dtype=torch.float64, device="cuda")
    half = f.numel()
    angle = torch.outer(pos.double(), f)
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]
    part = x[..., :2 * half]
    pairs = part.unflatten(-1, (half, 2)) if c["interleaved"] else part.unflatten(-1, (2, half)).transpose(-1, -2)
    z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
    z = z.flatten(-2) if c["interleaved"] else z.transpose(-1, -2).flatten(-2)
    return torch.cat([z, x[..., 2 * half:]], -1)


def _exact_heads(c, seed):
    """The way back is autograd's."""
    qkv, pos, w, dq, dk = _heads_inputs(c, seed)
    T, Hq, H = c["tokens"], c["q_heads"], c["kv_heads"]
    x = qkv.double().view(T, -1, D).requires_grad_()
    w = [None if t is None else t.double().requires_grad_() for t in w]
    parts = []
    for y, t in zip((x[:, :Hq], x[:, Hq:Hq + H]), w):
        if t is not None:
            y = y / torch.sqrt(y.square().sum(-1, keepdim=True) / D + EPS) * t
        parts.append(_turned64(c, y, pos))
    if c["kind"] == "heads":
        return [parts[0].detach(), parts[1].detach(), x[:, Hq + H:].detach() if c["values"] else None]
    torch.autograd.backward(parts, [dq.double(), dk.double()])
    return [x.grad.view(T, -1)] + [None if t is None else t.grad for t in w]


def _exact_attn(c, seed):
    """A sequence and a query head after the other; the way back is the derivative of the softmax row by row."""
    q, k, v, g = _attn_inputs(c, seed)
    Hq, H, n = c["q_heads"], c["kv_heads"], q.shape[0]
    new = lambda *shape: torch.zeros(*shape, device="cuda", dtype=torch.float64)          # noqa: E731
    out, lse, dq, dk, dv = new(n, Hq, D), new(Hq, n), new(n, Hq, D), new(n, H, D), new(n, H, D)
    at = 0
    for length in _lengths(c):
        rows = slice(at, at + length)
        i = torch.arange(length, device="cuda")
        past = i[None] <= i[:, None]
        near = past & ((i[None] < c["sink"]) | (i[:, None] - i[None] < c["recent"]))
        for h in range(Hq if length else 0):
            kv = h * H // Hq
            a, b, w = q[rows, h].double(), k[rows, kv].double(), v[rows, kv].double()
            z = (a @ b.t()).mul_(SCALE).masked_fill_(~(past if _mask(c)[kv] else near), -math.inf)
            lse[h, rows] = torch.logsumexp(z, -1)
            p = torch.softmax(z, -1)
            if c["kind"] == "attn":
                out[rows, h] = p @ w
                continue
            go = g[rows, h].double()
            dv[rows, kv] += p.t() @ go
            dp = go @ w.t()
            ds = p * (dp - (p * dp).sum(-1, keepdim=True))
            dq[rows, h] = ds @ b * SCALE
            dk[rows, kv] += ds.t() @ a * SCALE
        at += length
    return [out, lse] if c["kind"] == "attn" else [dq, dk, dv]


def exact(case, seed):
    if case["kind"] == "sample":
        return _exact_sample(case, seed)
    return _exact_heads(case, seed) if case["kind"] in ("heads", "heads_grad") else _exact_attn(case, seed)
