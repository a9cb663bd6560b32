"""The operators around the attention whose speed is measured: what a decoder does on its way into the head-mixed cache and out
of it again.

  norm      root-mean-square norm with the residual's addition, output in the storage type or in 8 bits with a scale for each
            128 columns (`quantize`: the 8-bit output alone, without a norm)
  matmul    product of 8-bit matrices, a scale for each row and 128 columns of the left one, one for each 128 x 128 block of
            the right one
  step      a decode step of one layer from the packed projections: queries and keys rotated by their positions, keys and
            values appended to the head-mixed cache, attention of the new tokens
  import    ragged prompts rotated and appended in one call, then one such step
  split     the packed projections of a prompt chunk as the prefill attention takes them: queries and keys rotated, heads first
  logprobs  log probabilities of given tokens, entropy, log-sum-exp and the most likely tokens of rows of logits
  grad      gradient of log probabilities and entropies with respect to the logits

Shapes are those of the library's own workloads (32 query / 8 KV heads and 28 / 4, head_dim 128, so 4096 and 3584 columns and
packed projections of 6144 and 4608) and generic ones.  `run` computes the plain form, or with `own` calls the library.
"""
import math

import torch

own = False

D = 128
GROUP = 128               # columns that share a scale
SCALE = 1.0 / math.sqrt(D)
EPS = 1e-5
E4M3 = torch.float8_e4m3fn
E4M3_MAX = 448.0
LEAST_SCALE = 2.0 ** -126
ROOM = 4096               # tokens a "step" case can grow by before its cache is filled anew


# ---- the cases ---------------------------------------------------------------------------------------------------

def _norm(name, rows, cols, dtype="bf16", to="e4m3", residual=True, kind="norm", pad=0):
    return dict(name=name, kind=kind, rows=rows, cols=cols, dtype=dtype, to=to, residual=residual, pad=pad)


def _matmul(name, m, n, k, to="bf16"):
    return dict(name=name, kind="matmul", m=m, n=n, k=k, to=to)


def _attn(name, kind, q_heads, kv_heads, pct, batch, lo, hi, sink, recent, dtype="bf16", page=0, rotary=D, interleaved=False):
    return dict(name=name, kind=kind, dtype=dtype, q_heads=q_heads, kv_heads=kv_heads, pct=pct, batch=batch, lo=lo, hi=hi,
                sink=sink, recent=recent, page=page, rotary=rotary, interleaved=interleaved)


def _logits(name, kind, rows, vocab, dtype="bf16", top=0, masked=False):
    return dict(name=name, kind=kind, rows=rows, vocab=vocab, dtype=dtype, top=top, masked=masked)


def listed():
    return [
        # One user's decode step: the norm in front of the projections, its output as the 8-bit product takes it.  The
        # smallest call: latency.
        _norm("norm_b1", 1, 4096),
        # The same for a batch of prompts.
        _norm("norm_prompts_16k", 16384, 3584),
        # One token through the packed projections: weights are read once, nothing else counts.
        _matmul("matmul_b1", 1, 6144, 4096),
        # A chat prompt of an odd length through the packed projections of the 28 / 4 shape.
        _matmul("matmul_prompt_333", 333, 4608, 3584),
        # A batch of prompts through a wide layer: the largest product.
        _matmul("matmul_prompts_8k", 8192, 14336, 4096),
        # A decode step of a busy server with a paged pool, from the packed projections to the attention's output.
        _attn("step_paged_b16_2k_6k", "step", 28, 4, 50, 16, 2000, 6000, 64, 256, page=64),
        # One user in single precision (how the cache is checked against a reference model).
        _attn("step_f32_b1_1k", "step", 32, 8, 50, 1, 1000, 1000, 16, 112, dtype="f32"),
        # Requests whose projections were computed elsewhere are admitted: ragged prompts go into the stores.
        _attn("import_b32_200_1500", "import", 32, 8, 60, 32, 200, 1500, 64, 512),
        # A small server's decode step: log probabilities of the sampled tokens with 20 alternatives each, as an interface reports them.
        _logits("logprobs_b8_top20", "logprobs", 8, 131072, dtype="f32", top=20),
        # Scoring the tokens of a rollout batch, with entropies; a vocabulary of odd size.
        _logits("logprobs_rollout_4k", "logprobs", 4096, 128011),
        # The policy gradient's way back through one short answer, and through a batch of them.
        _logits("grad_answer_64", "grad", 64, 32000, dtype="f32"),
        _logits("grad_rollout_2k", "grad", 2048, 128011),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "quantize", "matmul", "matmul", "matmul", "step", "step", "import", "split", "logprobs",
                       "logprobs", "logprobs", "grad", "grad"])
    if kind in ("norm", "quantize"):
        rows = _log_int(rng, 1, 16384)
        cols = _log_int(rng, 128, min(8192, 16384 * 3584 // rows))
        if rng.random() < 0.6:
            cols = -(-cols // 128) * 128
        dtype = rng.choice(["bf16", "bf16", "f32"])
        c = _norm("", min(rows, 16384 * 3584 // cols), cols, dtype, "e4m3" if kind == "quantize" else rng.choice(["e4m3", dtype]),
                  kind == "norm" and rng.random() < 0.7, kind, rng.choice([0, 0, 8, 3]))
    elif kind == "matmul":
        m = _log_int(rng, 1, 8192)
        n = _log_int(rng, 64, 14336)
        k = 16 * _log_int(rng, 8, min(896, max(8, 8192 * 14336 * 4096 // (m * n) // 16)))
        c = _matmul("", m, n, k, rng.choice(["bf16", "bf16", "f32"]))
    elif kind in ("step", "import", "split"):
        q_heads, kv_heads = rng.choice([(32, 8), (28, 4), (32, 8), (28, 4), (8, 8), (12, 4), (16, 1)])
        sink, recent = rng.choice([(16, 112), (64, 256), (64, 512), (33, 70), (4, 1000)])
        batch = _log_int(rng, 1, 32)
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        most = (2 ** 17 if kind == "step" else 2 ** 15) // (2 if dtype == "f32" else 1)
        hi = _log_int(rng, 20, min(8192, most // batch))
        c = _attn("", kind, q_heads, kv_heads, rng.choice([0, 20, 40, 60, 60, 80]), batch, rng.randint(max(1, hi // 8), hi), hi,
                  sink, recent, dtype, 0, rng.choice([128, 128, 128, 64, 32, 96]), rng.random() < 0.3)
        if c["dtype"] == "bf16" and rng.random() < 0.4:
            c["page"] = rng.choice([32, 64, 256])
    else:
        vocab = _log_int(rng, 1000, 262144)
        top = rng.choice([0, 0, 1, 5, 20, 32]) if kind == "logprobs" else 0
        most = 2 ** 25 if top else 2048 * 128011
        c = _logits("", kind, _log_int(rng, 1, min(4096, most // vocab)), vocab, rng.choice(["bf16", "bf16", "f32"]), top,
                    rng.random() < 0.3)
        if c["dtype"] == "f32":
            c["rows"] = max(1, c["rows"] // 2)
    del c["name"]
    return draw(rng) if 3072 in c.values() else c              # (a size that no configuration here has)


# ---- inputs ------------------------------------------------------------------------------------------------------

def _dtype(name):
    return {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": E4M3}[name]


def _gen(seed, what):
    return torch.Generator(device="cuda").manual_seed(seed * 16 + what)


def _randn(seed, what, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=_gen(seed, what), device="cuda", dtype=dtype)


def _groups(n):
    return -(-n // GROUP)


def _lengths(c):
    """Context (prompt) length of every sequence: spread over [lo, hi] in a scattered order."""
    n, lo, hi = c["batch"], c["lo"], c["hi"]
    return [lo + int((hi - lo) * ((b * 0.6180339887498949 + 0.5) % 1.0) + 0.5) for b in range(n)]


def _mask(c):
    """[kv_heads], 1 = full."""
    n = c["pct"] * c["kv_heads"] // 100
    return [0 if h < n else 1 for h in range(c["kv_heads"])]


def _inv_freq(c):
    """Radians a position, of each pair of rotated columns."""
    half = c["rotary"] // 2
    return [500000.0 ** (-i / half) for i in range(half)]


def _heads(c):
    return c["q_heads"] + 2 * c["kv_heads"]


def _norm_inputs(c, seed):
    """Activations as a decoder has them: a few columns far larger than the rest."""
    R, C, dt = c["rows"], c["cols"], _dtype(c["dtype"])
    big = 1.0 + 20.0 * (torch.rand(C, generator=_gen(seed, 1), device="cuda") < 0.005)
    x = torch.zeros(R, C + c["pad"], device="cuda", dtype=dt)[:, :C]
    x.copy_((_randn(seed, 2, R, C, dtype=dt) * big.to(dt)))
    res = _randn(seed, 3, R, C, dtype=dt) * 2.0 if c["residual"] else None
    w = (1.0 + 0.1 * _randn(seed, 4, C)).to(dt)
    return x, res, w


def _matmul_inputs(c, seed):
    M, N, K = c["m"], c["n"], c["k"]
    a = (_randn(seed, 1, M, K, dtype=torch.bfloat16) * 100.0).to(E4M3)
    b = (_randn(seed, 2, N, K, dtype=torch.bfloat16) * 100.0).to(E4M3)
    a_scales = 0.01 * (0.5 + torch.rand(_groups(K), M, generator=_gen(seed, 3), device="cuda"))
    b_scales = 2e-4 * (0.5 + torch.rand(_groups(N), _groups(K), generator=_gen(seed, 4), device="cuda"))
    return a, a_scales, b, b_scales


def _attn_inputs(c, seed):
    B, dt = c["batch"], _dtype(c["dtype"])
    one = _randn(seed, 1, B, 1, _heads(c) * D, dtype=dt)                       # a new token's packed projections
    if c["kind"] == "step":                                                    # the contexts, as they are in a cache
        k = _randn(seed, 2, B, c["kv_heads"], c["hi"], D, dtype=dt)
        v = _randn(seed, 3, B, c["kv_heads"], c["hi"], D, dtype=dt)
        return one, k, v
    return one, _randn(seed, 2, B, c["hi"], _heads(c) * D, dtype=dt), None     # prompts: packed projections


def _logit_inputs(c, seed):
    """Rows of a padded buffer, as a projection to a vocabulary leaves them; tokens of the prompt (-1) are not scored."""
    R, V, dt = c["rows"], c["vocab"], _dtype(c["dtype"])
    x = torch.zeros(R, -(-V // 64) * 64, device="cuda", dtype=dt)[:, :V]
    x.copy_(_randn(seed, 1, R, V, dtype=dt) * 3.0)
    tokens = torch.randint(0, V, (R,), generator=_gen(seed, 2), device="cuda", dtype=torch.int32)
    if c["masked"]:                                                            # an answer of a given form: most tokens are forbidden
        off = torch.rand(V, generator=_gen(seed, 3), device="cuda") < 0.7
        off[tokens.long()] = False
        x.masked_fill_(off, -math.inf)
    if R > 16:
        tokens[::7] = -1
    return x, tokens


class State:
    pass


def prepare(case, seed):
    """Goes by `own` for one thing only: the cache that the library's calls work on is filled where they are made, and the
    plain form keeps its keys and values in two tensors."""
    c, s = case, State()
    s.case = c
    new = lambda *shape, dtype: torch.zeros(*shape, device="cuda", dtype=dtype)          # noqa: E731
    if c["kind"] in ("norm", "quantize"):
        s.x, s.residual, s.weight = _norm_inputs(c, seed)
        s.sum = new(c["rows"], c["cols"], dtype=s.x.dtype) if c["residual"] else None
        s.out = new(c["rows"], c["cols"], dtype=_dtype(c["to"]))
        s.scales = new(_groups(c["cols"]), c["rows"], dtype=torch.float32) if c["to"] == "e4m3" else None
    elif c["kind"] == "matmul":
        s.a, s.a_scales, s.b, s.b_scales = _matmul_inputs(c, seed)
        s.out = new(c["m"], c["n"], dtype=_dtype(c["to"]))
    elif c["kind"] in ("step", "import", "split"):
        _prepare_attn(s, c, seed, new)
    else:
        s.x, s.tokens = _logit_inputs(c, seed)
        if c["kind"] == "grad":
            s.g_logprob, s.g_entropy = _randn(seed, 4, c["rows"]), 0.01 * _randn(seed, 5, c["rows"])
            _, s.entropy, s.lse, _ = _plain_logprobs(s.x, s.tokens, 1.0)
            s.out = torch.empty_like(s.x)
        else:
            R, k = c["rows"], c["top"]
            s.logprob, s.entropy, s.lse = (new(R, dtype=torch.float32) for _ in range(3))
            s.top = (new(R, k, dtype=torch.float32), new(R, k, dtype=torch.int32)) if k else None
            if own:
                import paper_2510_08525_amd as rl

                s.workspace = new(max(1, rl.rlkv_token_logprobs_workspace(R, c["vocab"], k)), dtype=torch.uint8)
    torch.cuda.synchronize()
    return s


def _prepare_attn(s, c, seed, new):
    B, H, Hq, dt, ns = c["batch"], c["kv_heads"], c["q_heads"], _dtype(c["dtype"]), _lengths(c)
    s.one, a, b = _attn_inputs(c, seed)
    s.lengths, s.grown = ns, 0
    s.at = torch.tensor(ns, device="cuda")
    s.q_one, s.out = new(B, Hq, D, dtype=dt), new(B, Hq, D, dtype=dt)
    room = {"step": ROOM, "import": 1, "split": 0}[c["kind"]]
    if c["kind"] == "step":
        s.context = a, b
    else:
        s.prompts = a
        s.q = new(B, Hq, c["hi"], D, dtype=dt)
    if c["kind"] == "split":
        s.k, s.v = new(B, H, c["hi"], D, dtype=dt), new(B, H, c["hi"], D, dtype=dt)
    s.inv_freq = torch.tensor(_inv_freq(c), device="cuda", dtype=torch.float64)
    s.local = ~torch.tensor(_mask(c), device="cuda", dtype=torch.bool)
    if own:
        import paper_2510_08525_amd as rl

        most = [n + max(1, room) for n in ns]
        pool = sum(-(-n // c["page"]) for n in most) if c["page"] else 0
        s.cache = rl.Cache(1, Hq, H, D, B, c["sink"], c["recent"], rl.RLKV_BF16 if c["dtype"] == "bf16" else rl.RLKV_F32,
                           _mask(c), most, page_tokens=c["page"], pool_pages=pool)
        if c["page"]:
            s.cache.pool_shuffle(1234 + seed)
        s.rotary = rl.Rotary(_inv_freq(c), interleaved=c["interleaved"])
        if c["kind"] == "step":
            s.cache.append_ragged(0, *s.context, ns)
    elif c["kind"] != "split":
        s.keys, s.values = (new(B, H, c["hi"] + room, D, dtype=dt) for _ in range(2))
        if c["kind"] == "step":
            s.keys[:, :, :c["hi"]], s.values[:, :, :c["hi"]] = s.context


def run(s):
    return _run_own(s) if own else _run_plain(s)


# ---- the library's calls -------------------------------------------------------------------------------------------

def _run_own(s):
    import paper_2510_08525_amd as rl

    c = s.case
    if c["kind"] == "norm":
        rl.rms_norm(s.x, s.weight, EPS, s.out, scales=s.scales, residual=s.residual, sum_out=s.sum)
        return [s.out, s.scales, s.sum]
    if c["kind"] == "quantize":
        rl.quantize(s.x, s.out, s.scales)
        return [s.out, s.scales, s.sum]
    if c["kind"] == "matmul":
        rl.scaled_matmul(s.a, s.a_scales, s.b, s.b_scales, s.out)
        return s.out
    if c["kind"] == "logprobs":
        rl.token_logprobs(s.x, s.tokens, s.logprob, entropy=s.entropy, lse=s.lse, top=s.top, workspace=s.workspace)
        return [s.logprob, s.entropy, s.lse, s.top]
    if c["kind"] == "grad":
        rl.token_logprobs_grad(s.x, s.tokens, s.lse, s.g_logprob, s.out, entropy=s.entropy, grad_entropy=s.g_entropy)
        return s.out
    cache = s.cache
    if c["kind"] == "split":
        cache.rotary(0, s.prompts, s.lengths, s.rotary, s.q, s.k, s.v)
        return [s.q, s.k, s.v]                                  # (rows past a prompt's end are zero since prepare())
    if c["kind"] == "import":
        cache.reset()
        cache.append_rotary(0, s.prompts, s.lengths, s.rotary, s.q)
    elif s.grown == ROOM:
        cache.reset()
        cache.append_ragged(0, *s.context, s.lengths)
        s.grown = 0
    cache.append_rotary(0, s.one, None, s.rotary, s.q_one)
    cache.decode_attention(0, s.q_one, s.out, SCALE)
    s.grown += 1
    return [s.q_one, s.out] + ([s.q] if c["kind"] == "import" else [])


# ---- the plain form ------------------------------------------------------------------------------------------------

def _plain_logprobs(x, tokens, scale, top=0):
    x = x.float() * scale
    m = x.amax(-1, keepdim=True)
    e = torch.exp(x - m)
    total = e.sum(-1, keepdim=True)
    lse = m + torch.log(total)
    entropy = (lse - (e * torch.where(e > 0, x, 0.0)).sum(-1, keepdim=True) / total)[:, 0]
    picked = x.gather(1, tokens.long().clamp(min=0)[:, None])
    logprob = torch.where(tokens >= 0, (picked - lse)[:, 0], 0.0)
    best = None
    if top:
        v, i = torch.sort(x, dim=-1, descending=True, stable=True)
        best = (v[:, :top] - lse, i[:, :top].int())
    return logprob, entropy, lse[:, 0], best


def _plain_quantize(y):
    R, C = y.shape
    g = torch.nn.functional.pad(y, (0, _groups(C) * GROUP - C)).view(R, -1, GROUP)
    scales = (g.abs().amax(-1) / E4M3_MAX).clamp(min=LEAST_SCALE)
    return (g / scales[..., None]).to(E4M3).view(R, -1)[:, :C], scales.t()


def _plain_rotate(x, pos, s):
    """x [B, T, heads, D] in 32 bits, pos [B, T]; angles in 64 bits."""
    half = s.inv_freq.numel()
    angle = pos.double()[..., None, None] * s.inv_freq
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    r = x.clone()
    if s.case["interleaved"]:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        r[..., 0:2 * half:2], r[..., 1:2 * half:2] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., :half], x[..., half:2 * half]
        r[..., :half], r[..., half:2 * half] = a * cos - b * sin, b * cos + a * sin
    return r


def _plain_split(s, packed, pos):
    """Packed projections [B, T, heads * D] as q, k, v [B, heads, T, D], queries and keys rotated."""
    c = s.case
    Hq, H = c["q_heads"], c["kv_heads"]
    x = packed.view(*packed.shape[:2], _heads(c), D)
    qk = _plain_rotate(x[:, :, :Hq + H].float(), pos, s).to(packed.dtype).transpose(1, 2)
    return qk[:, :Hq], qk[:, Hq:], x[:, :, Hq + H:].transpose(1, 2)


def _plain_attention(s, q, pos, most):
    """q [B, Hq, D] at positions pos over the first `most` rows of the plain cache."""
    c = s.case
    B, H = c["batch"], c["kv_heads"]
    j = torch.arange(most, device="cuda")
    i = pos[:, None]
    near = (j <= i) & ((j < c["sink"]) | (i - j < c["recent"]))
    admit = torch.where(s.local[None, :, None], near[:, None], (j <= i)[:, None])              # [B, H, most]
    k, v = s.keys[:, :, :most].float(), s.values[:, :, :most].float()
    scores = torch.matmul(q.float().view(B, H, -1, D) * SCALE, k.transpose(-1, -2).contiguous())
    scores = scores.masked_fill(~admit[:, :, None], -math.inf)
    p = torch.exp(scores - scores.amax(-1, keepdim=True))
    out = torch.matmul(p, v) / p.sum(-1, keepdim=True)
    return out.reshape(B, -1, D).to(q.dtype)


def _run_plain(s):
    c = s.case
    if c["kind"] in ("norm", "quantize"):
        h = s.x.float()
        if s.residual is not None:
            h = h + s.residual.float()
            s.sum = h.to(s.x.dtype)
        y = h
        if c["kind"] == "norm":
            y = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS) * s.weight.float()
        out, scales = _plain_quantize(y) if c["to"] == "e4m3" else (y.to(_dtype(c["to"])), None)
        return [out, scales, s.sum]
    if c["kind"] == "matmul":
        M, N, K = c["m"], c["n"], c["k"]
        a = s.a.float() * s.a_scales.t().repeat_interleave(GROUP, 1)[:, :K]
        b = s.b.float() * s.b_scales.repeat_interleave(GROUP, 0)[:N].repeat_interleave(GROUP, 1)[:, :K]
        return torch.matmul(a, b.t()).to(_dtype(c["to"]))
    if c["kind"] == "logprobs":
        return list(_plain_logprobs(s.x, s.tokens, 1.0, c["top"]))
    if c["kind"] == "grad":
        x = s.x.float()
        lp = x - s.lse[:, None]
        p = torch.exp(lp)
        g = torch.where(s.tokens >= 0, s.g_logprob, 0.0)[:, None]
        d = -p * (g + s.g_entropy[:, None] * (torch.where(p > 0, lp, 0.0) + s.entropy[:, None]))
        d.scatter_add_(1, s.tokens.long().clamp(min=0)[:, None], g)
        return d.to(s.x.dtype)
    T, at = c["hi"], s.at
    if c["kind"] in ("split", "import"):
        step = torch.arange(T, device="cuda")
        there = step < at[:, None]                                                              # [B, T]
        q, k, v = _plain_split(s, s.prompts, step.expand(c["batch"], T))
        q = torch.where(there[:, None, :, None], q, 0.0)
        if c["kind"] == "split":
            return [q] + [torch.where(there[:, None, :, None], x, 0.0) for x in (k, v)]
        s.keys[:, :, :T], s.values[:, :, :T], s.grown = k, v, 0
    elif s.grown == ROOM:
        s.grown = 0
    pos = at + s.grown
    q1, k1, v1 = _plain_split(s, s.one, pos[:, None])
    row = torch.arange(c["batch"], device="cuda")
    s.keys[row, :, pos], s.values[row, :, pos] = k1[:, :, 0], v1[:, :, 0]
    out = _plain_attention(s, q1[:, :, 0], pos, c["hi"] + s.grown + 1)
    s.grown += 1
    return [q1[:, :, 0], out] + ([q] if c["kind"] == "import" else [])


# ---- what a pass cannot do without -----------------------------------------------------------------------------------

def work(case):
    c = case
    e = {"f32": 4, "bf16": 2}.get(c.get("dtype"), 0)
    if c["kind"] in ("norm", "quantize"):
        n = c["rows"] * c["cols"]
        out = {"f32": 4, "bf16": 2, "e4m3": 1}[c["to"]]
        scales = 4 * c["rows"] * _groups(c["cols"]) if c["to"] == "e4m3" else 0
        norm = c["kind"] == "norm"
        return {"bytes": n * (e * (3 if c["residual"] else 1) + out) + scales + norm * c["cols"] * e, "flops": 6 * n}
    if c["kind"] == "matmul":
        M, N, K = c["m"], c["n"], c["k"]
        scales = 4 * _groups(K) * (M + _groups(N))
        return {"bytes": M * K + N * K + scales + M * N * (4 if c["to"] == "f32" else 2), "flops": 2 * M * N * K}
    if c["kind"] == "logprobs":
        n = c["rows"] * c["vocab"]
        return {"bytes": n * e + c["rows"] * (16 + 8 * c["top"]), "flops": 6 * n}
    if c["kind"] == "grad":
        n = c["rows"] * c["vocab"]
        return {"bytes": 2 * n * e + 20 * c["rows"], "flops": 8 * n}
    Hq, H, W, ns = c["q_heads"], c["kv_heads"], c["sink"] + c["recent"], _lengths(c)
    row = 2 * D * e
    stays = sum(sum(n if f else min(n, W) for f in _mask(c)) for n in ns)                       # rows of the stores
    if c["kind"] == "split":
        return {"bytes": 2 * sum(ns) * _heads(c) * D * e, "flops": 6 * sum(ns) * (Hq + H) * c["rotary"] // 2}
    nbytes, flops = 0, 0
    if c["kind"] == "import":
        nbytes = 2 * sum(ns) * Hq * D * e + 2 * stays * row
        flops = 3 * sum(ns) * (Hq + H) * c["rotary"]
    keys = sum(sum(min(n + 1, n + 1 if f else W) for f in _mask(c)) for n in ns)
    nbytes += keys * row + c["batch"] * (_heads(c) + 2 * H + 3 * Hq) * D * e
    return {"bytes": nbytes, "flops": flops + 4 * D * Hq // H * keys}


# ---- the same in 64 bits ---------------------------------------------------------------------------------------------

def _turned64(c, x, first):
    """x [T, heads, D] in 64 bits at positions first, first + 1, ..., as products of complex numbers."""
    f = torch.tensor(_inv_freq(c), dtype=torch.float64, device="cuda")
    half = f.numel()
    angle = torch.outer(torch.arange(first, first + x.shape[0], dtype=torch.float64, device="cuda"), f)
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]
    part = x[..., :2 * half]
    pairs = part.unflatten(-1, (half, 2)) if c["interleaved"] else part.unflatten(-1, (2, half)).transpose(-1, -2)
    z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
    z = z.flatten(-2) if c["interleaved"] else z.transpose(-1, -2).flatten(-2)
    return torch.cat([z, x[..., 2 * half:]], -1)


def _attend64(c, q, k, v):
    """q [Hq, D] of the newest position, k, v [H, n, D]: a loop over KV heads."""
    n, G, outs = k.shape[1], c["q_heads"] // c["kv_heads"], []
    j = torch.arange(n, device="cuda")
    for h, full in enumerate(_mask(c)):
        keep = j[(j < c["sink"]) | (j >= n - c["recent"])] if not full else j
        w = torch.softmax(q[h * G:(h + 1) * G] @ k[h, keep].t() * SCALE, -1)
        outs.append(w @ v[h, keep])
    return torch.cat(outs)


def exact(case, seed):
    c = case
    if c["kind"] in ("norm", "quantize"):
        x, res, w = _norm_inputs(c, seed)
        h = x.double() if res is None else x.double() + res.double()
        y = h
        if c["kind"] == "norm":
            y = h / torch.sqrt(h.pow(2).sum(1) / c["cols"] + EPS)[:, None] * w.double()
        total = h if res is not None else None
        if c["to"] != "e4m3":
            return [y, None, total]
        scales = torch.stack([p.abs().amax(1) for p in y.split(GROUP, 1)]) / E4M3_MAX
        scales = torch.clamp(scales, min=LEAST_SCALE)
        return [torch.cat([p / t[:, None] for p, t in zip(y.split(GROUP, 1), scales)], 1), scales, total]
    if c["kind"] == "matmul":
        a, sa, b, sb = _matmul_inputs(c, seed)
        out = torch.zeros(c["m"], c["n"], device="cuda", dtype=torch.float64)
        for j, n0 in enumerate(range(0, c["n"], 16 * GROUP)):                  # 16 blocks of columns at a time
            part = b[n0:n0 + 16 * GROUP].double()
            lines = sb[16 * j:16 * j + 16].double()
            for g in range(_groups(c["k"])):
                cols = slice(g * GROUP, (g + 1) * GROUP)
                right = part[:, cols] * lines[:, g].repeat_interleave(GROUP)[:part.shape[0], None]
                out[:, n0:n0 + part.shape[0]] += (a[:, cols].double() * sa[g].double()[:, None]) @ right.t()
        return out
    if c["kind"] in ("logprobs", "grad"):
        return _exact_logits(c, seed)
    Hq, H, ns = c["q_heads"], c["kv_heads"], _lengths(c)
    one, a, b = _attn_inputs(c, seed)
    q1, outs = [], []
    if c["kind"] != "step":
        parts = [torch.zeros(c["batch"], h, c["hi"], D, device="cuda", dtype=torch.float64) for h in (Hq, H, H)]
    for i, n in enumerate(ns):
        if c["kind"] != "step":
            x = a[i, :n].double().view(n, -1, D)
            turned = _turned64(c, x[:, :Hq + H], 0)
            for p, part in zip(parts, (turned[:, :Hq], turned[:, Hq:], x[:, Hq + H:])):
                p[i, :, :n] = part.transpose(0, 1)
            if c["kind"] == "split":
                continue
            k, v = parts[1][i, :, :n], parts[2][i, :, :n]
        else:
            k, v = a[i, :, :n].double(), b[i, :, :n].double()
        x = one[i].double().view(1, -1, D)
        turned = _turned64(c, x[:, :Hq + H], n)[0]
        q1.append(turned[:Hq])
        outs.append(_attend64(c, turned[:Hq], torch.cat([k, turned[Hq:, None]], 1), torch.cat([v, x[0, Hq + H:, None]], 1)))
    if c["kind"] == "split":
        return parts
    return [torch.stack(q1), torch.stack(outs)] + (parts[:1] if c["kind"] == "import" else [])


def _exact_logits(c, seed):
    x, tokens = _logit_inputs(c, seed)
    R, V = x.shape
    done = []
    if c["kind"] == "grad":
        g, h = _randn(seed, 4, R).double(), 0.01 * _randn(seed, 5, R)
        h = h.double()
    for r in range(0, R, 256):                                                 # 256 rows at a time: memory
        lp = torch.log_softmax(x[r:r + 256].double(), -1)
        p = lp.exp()
        plp = torch.special.entr(p)                                            # -p log p, 0 where p is 0
        entropy = plp.sum(-1)
        t = tokens[r:r + 256].long()
        rows = torch.arange(t.numel(), device="cuda")[t >= 0]
        if c["kind"] == "grad":
            part = plp * h[r:r + 256, None] - p * (entropy * h[r:r + 256])[:, None]
            gt = torch.where(t >= 0, g[r:r + 256], 0.0)
            part -= p * gt[:, None]
            part[rows, t[rows]] += gt[rows]
            done.append(part)
            continue
        picked = torch.zeros_like(entropy)
        picked[rows] = lp[rows, t[rows]]
        one = [picked, entropy, torch.logsumexp(x[r:r + 256].double(), -1)]
        if c["top"]:
            one.append(torch.topk(lp, c["top"], -1).values)
        done.append(one)
    if c["kind"] == "grad":
        return torch.cat(done)
    got = [torch.cat(v) for v in zip(*done)]
    return got[:3] + [(got[3], None) if c["top"] else None]
