"""The operators around the SBVR products in a decode step that verifies
drafted tokens, as they are timed and checked: the plan of a batch (pages,
slots, tree masks), the cache write, attention for a tree of drafted tokens
over the paged cache, the norms around a block with its gate and residual
scale, and the adjustment of logits before sampling.

A case names an operator (``op``) and its sizes.  ``run`` makes one pass:
through the package's public calls where ``own`` is true, through elementary
torch operations in binary32 where it is false.  ``exact`` gives the same
outputs from the definitions in binary64.
"""
import math

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one sequence, one new token: the plan's latency
        dict(name="plan_1", op="plan", requests=1, new=1, context=900, page=16, tree=False),
        # the largest batch served at once, trees of up to 64 drafted tokens
        dict(name="plan_4096_trees", op="plan", requests=4096, new=64, context=8192, page=16, tree=True),
        # one verification step's keys and values: eight drafted tokens, 8 kv heads of 128
        dict(name="write_8", op="write", tokens=8, kv_heads=8, dim=128, page=16, dtype="f16", layout="token"),
        # a prompt chunk written at once, pages kept head by head
        dict(name="write_16384", op="write", tokens=16384, kv_heads=8, dim=128, page=64, dtype="bf16", layout="head"),
        # plain decoding of one sequence with the 8B head layout: a single token, latency
        dict(name="attn_1x1_4k", op="attn", requests=1, new=1, context=4096, heads=32, kv_heads=8, dim=128, page=16,
             dtype="f16", layout="token", ragged=False),
        # eight sequences of the 8B layout, each verifying eight drafted tokens, ragged contexts
        dict(name="attn_8x8_8k", op="attn", requests=8, new=8, context=8192, heads=32, kv_heads=8, dim=128, page=64,
             dtype="f16", layout="token", ragged=True),
        # a busy server: 64 sequences decoding one token each on short ragged contexts, heads of 64
        dict(name="attn_64x1_2k", op="attn", requests=64, new=1, context=2047, heads=32, kv_heads=8, dim=64, page=32,
             dtype="bf16", layout="head", ragged=True),
        # four long contexts with the 70B head layout, trees of sixteen
        dict(name="attn_4x16_128k", op="attn", requests=4, new=16, context=131072, heads=64, kv_heads=8, dim=128,
             page=64, dtype="bf16", layout="token", ragged=False),
        # one token between two blocks of the 8B model: latency
        dict(name="norm_1x4096", op="norm", tokens=1, width=4096, dtype="f16", stream="f32", post=True, gate="none"),
        # a prompt chunk through the 70B width with norms on both sides and a gate per token
        dict(name="norm_4096x8192", op="norm", tokens=4096, width=8192, dtype="bf16", stream="bf16", post=True,
             gate="token"),
        # one sequence's next token on a vocabulary of odd size, all adjustments
        dict(name="logits_1x50001", op="logits", requests=1, new=1, vocab=50001, history=1500, dtype="f16", out="f32",
             grammar=1.0),
        # 32 sequences verifying trees of eight on a large vocabulary, a quarter of the rows under a grammar
        dict(name="logits_32x8x131072", op="logits", requests=32, new=8, vocab=131072, history=4000, dtype="f16",
             out="f32", grammar=0.25),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("plan", "write", "attn", "attn", "attn", "norm", "logits"))
    if op == "plan":
        return dict(op=op, requests=_log_int(rng, 1, 4096), new=_log_int(rng, 1, 64),
                    context=_log_int(rng, 1, 8192), page=2 ** rng.randint(4, 8), tree=rng.random() < 0.7)
    if op == "write":
        return dict(op=op, tokens=_log_int(rng, 1, 16384), kv_heads=rng.choice((1, 2, 4, 8)),
                    dim=rng.choice((64, 80, 96, 128)), page=2 ** rng.randint(4, 8), dtype=rng.choice(("f16", "bf16")),
                    layout=rng.choice(("token", "head")))
    if op == "attn":
        heads, kv_heads = rng.choice(((32, 8), (32, 8), (64, 8), (16, 16), (24, 4), (8, 1)))
        c = dict(op=op, requests=_log_int(rng, 1, 64), new=_log_int(rng, 1, 64), context=_log_int(rng, 1, 131072),
                 heads=heads, kv_heads=kv_heads, dim=rng.choice((64, 80, 96, 128, 128, 128)),
                 page=2 ** rng.randint(4, 8), dtype=rng.choice(("f16", "bf16")),
                 layout=rng.choice(("token", "head")), ragged=rng.random() < 0.7)
        # no more cached values and no more products than the largest listed case
        while (c["requests"] * c["context"] * c["kv_heads"] * c["dim"] > 4 * 131072 * 8 * 128
               or c["requests"] * c["context"] * c["heads"] * c["new"] > 4 * 131072 * 64 * 16):
            c["context"] = max(1, c["context"] * 2 // 3)
        return c
    if op == "norm":
        c = dict(op=op, tokens=_log_int(rng, 1, 4096), width=_log_int(rng, 64, 16384),
                 dtype=rng.choice(("f16", "bf16")), stream=rng.choice(("same", "f32")), post=rng.random() < 0.6,
                 gate=rng.choice(("none", "channel", "token")))
        if c["stream"] == "same":
            c["stream"] = c["dtype"]
        if rng.random() < 0.6:
            c["width"] = max(64, c["width"] // 64 * 64)
        while c["tokens"] * c["width"] > 2048 * 8192:
            c["tokens"] = max(1, c["tokens"] // 2)
        return c
    c = dict(op=op, requests=_log_int(rng, 1, 64), new=_log_int(rng, 1, 16), vocab=_log_int(rng, 1000, 131072),
             history=_log_int(rng, 1, 8000), dtype=rng.choice(("f16", "bf16", "f32")), out="f32",
             grammar=rng.choice((0.0, 0.25, 1.0)))
    while c["requests"] * c["new"] * c["vocab"] > 32 * 8 * 131072:
        c["requests"] = max(1, c["requests"] // 2)
    return c


# ---------------------------------------------------------------------------
# sizes of the requests of a batch, the same for every seed
# ---------------------------------------------------------------------------

def _contexts(case):
    """Cached tokens of each request: the first the longest, the others spread
    over the range below it where the batch is ragged."""
    R, top = case["requests"], case["context"]
    if not case.get("ragged", True):
        return [top] * R
    return [max(0, int(top * (1.0 - (0.6180339887498949 * r) % 1.0))) for r in range(R)]


def _news(case):
    """New tokens of each request: up to case["new"], at least one."""
    R, top = case["requests"], case["new"]
    if not case.get("ragged", True) or case["op"] == "logits":
        return [top] * R
    return [max(1, int(round(top * (1.0 - 0.5 * ((0.7548776662466927 * r) % 1.0))))) for r in range(R)]


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _parents(g, n, top):
    """Parents of each request's drafted tokens, within the request: the first
    is the root, a later one hangs on any earlier one, mostly a late one."""
    j = torch.arange(top, device="cuda").expand(len(n), top)
    u = torch.rand(len(n), top, generator=g, device="cuda").sqrt()
    p = torch.where(j > 0, (u * j).long().clamp(max=top - 1).minimum(j - 1), j - 1).to(torch.int32)
    return p[j < torch.tensor(n, device="cuda")[:, None]]


def _masks(parents, n, top):
    """Bits of each drafted token's ancestors, itself among them."""
    R, T = len(n), sum(n)
    count = torch.tensor(n, device="cuda")
    start = torch.zeros(R + 1, dtype=torch.long, device="cuda")
    start[1:] = count.cumsum(0)
    req = torch.repeat_interleave(torch.arange(R, device="cuda"), count, output_size=T)
    j = torch.arange(T, device="cuda") - start[req]
    return _closure(parents.long(), j, start[req])[0]


def _closure(parents, j, first):
    """(mask, depth) of each token from its parent within its request, by
    pointer doubling; the last row stands for the roots' missing parent."""
    T = parents.numel()
    up = torch.where(parents >= 0, first + parents, T)
    up = torch.cat([up, torch.full((1,), T, device="cuda")])
    mask = torch.cat([torch.ones_like(j) << j.clamp(max=63), torch.zeros(1, dtype=torch.long, device="cuda")])
    depth = (up < T).long()
    for _ in range(6):
        mask, depth, up = mask | mask[up], depth + depth[up], up[up]
    return mask[:T], depth[:T]


def _cache(g, pages, page, heads, dim, dtype, layout):
    """Key and value pages [pages][page][heads][dim]; "head": stored head by
    head within a page."""
    shape = (pages, page, heads, dim) if layout == "token" else (pages, heads, page, dim)
    kv = [torch.randn(shape, generator=g, device="cuda", dtype=DTYPES[dtype]) for _ in range(2)]
    return kv if layout == "token" else [t.transpose(1, 2) for t in kv]


def prepare(case, seed):
    g = _generator(seed)
    return _PREPARE[case["op"]](case, g)


def _prepare_plan(case, g):
    ctx, new, P = _contexts(case), _news(case), case["page"]
    R, T = len(ctx), sum(new)
    width = (case["context"] + case["new"] + P - 1) // P + 1
    have = _ints([-(-c // P) for c in ctx])
    need = sum(-(-(c + n) // P) - -(-c // P) for c, n in zip(ctx, new))
    used = int(have.sum())
    order = torch.randperm(used + need + 64, generator=g, device="cuda").to(torch.int32)
    table = torch.full((R, width), -1, dtype=torch.int32, device="cuda")
    table[torch.arange(width, device="cuda") < have[:, None]] = order[:used]
    return dict(op="plan", context=_ints(ctx), new=_ints(new), free=order[used:].contiguous(), table=table, page=P,
                tokens=T, parents=_parents(g, new, case["new"]) if case["tree"] else None)


def _prepare_write(case, g):
    T, P = case["tokens"], case["page"]
    pages = -(-T // P) + 4
    K, V = _cache(g, pages, P, case["kv_heads"], case["dim"], case["dtype"], case["layout"])
    # keys and values as a joint projection leaves them: views of one matrix's rows
    kv = torch.randn(T, 2, case["kv_heads"], case["dim"], generator=g, device="cuda", dtype=DTYPES[case["dtype"]])
    page = torch.randperm(pages, generator=g, device="cuda")
    t = torch.arange(T, device="cuda") + 5
    slots = page[t // P] * P + t % P
    if T > 4:
        slots[T // 2] = -1  # a token of a request that found no page
    return dict(op="write", K=K, V=V, k=kv[:, 0], v=kv[:, 1], slots=slots)


def _prepare_attn(case, g):
    ctx, new, P, dt = _contexts(case), _news(case), case["page"], DTYPES[case["dtype"]]
    R, T = len(ctx), sum(new)
    count = [-(-(c + n) // P) for c, n in zip(ctx, new)]
    width = max(count)
    pages = sum(count) + 2
    K, V = _cache(g, pages, P, case["kv_heads"], case["dim"], case["dtype"], case["layout"])
    table = torch.full((R, width), -1, dtype=torch.int32, device="cuda")
    at = torch.arange(width, device="cuda") < _ints(count)[:, None]
    table[at] = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)[: sum(count)]
    start = _ints([0] + new).cumsum(0).to(torch.int32)
    return dict(op="attn", K=K, V=V, table=table, context=_ints(ctx), start=start,
                q=1.5 * torch.randn(T, case["heads"], case["dim"], generator=g, device="cuda", dtype=dt),
                mask=_masks(_parents(g, new, case["new"]), new, case["new"]), max_new=case["new"],
                longest=max(c + n for c, n in zip(ctx, new)), scale=case["dim"] ** -0.5)


def _prepare_norm(case, g):
    T, H, dt, st = case["tokens"], case["width"], DTYPES[case["dtype"]], DTYPES[case["stream"]]

    def randn(*shape, dtype=dt, mean=0.0, std=1.0):
        return (mean + std * torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)).to(dtype)
    gate = {"none": None, "channel": randn(H, mean=0.5, std=0.2) if case["gate"] == "channel" else None,
            "token": randn(T, H, mean=0.5, std=0.2) if case["gate"] == "token" else None}[case["gate"]]
    return dict(op="norm", x=randn(T, H, dtype=st, std=2.0), y=randn(T, H), gate=gate,
                post=randn(H, mean=1.0, std=0.1) if case["post"] else None, pre=randn(H, mean=1.0, std=0.1),
                scale=0.7, eps=1e-5)


def _prepare_logits(case, g):
    R, N, V = case["requests"], case["new"], case["vocab"]
    T = R * N
    hist = [max(1, int(case["history"] * (1.0 - (0.6180339887498949 * r) % 1.0))) for r in range(R)]

    def uniform(n, lo, hi):
        return lo + (hi - lo) * torch.rand(n, generator=g, device="cuda")
    # text repeats its words: token ids from a distribution with a heavy head
    words = (V * torch.rand(sum(hist), generator=g, device="cuda") ** 4).long().clamp(max=V - 1).to(torch.int32)
    n_bias = [(7 * r) % 48 + 1 for r in range(R)]
    bias_start = _ints([0] + n_bias).cumsum(0).to(torch.int32)
    # distinct biased tokens within a request
    step = V // 50
    first = torch.randint(0, step, (R,), generator=g, device="cuda")
    order = torch.arange(48, device="cuda")
    bias_tokens = (first[:, None] + step * order)[order < _ints(n_bias)[:, None]].to(torch.int32)
    new = [N] * R
    M = int(round(case["grammar"] * T))
    rows = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    rows[torch.randperm(T, generator=g, device="cuda")[:M]] = torch.arange(M, dtype=torch.int32, device="cuda")
    grammar = torch.randint(-2**31, 2**31, (max(M, 1), (V + 31) // 32), dtype=torch.int64, generator=g,
                            device="cuda").to(torch.int32)
    return dict(op="logits", logits=(3 * torch.randn(T, V, generator=g, device="cuda")).to(DTYPES[case["dtype"]]),
                history=words, history_start=_ints([0] + hist).cumsum(0).to(torch.int32),
                prompt=_ints([h // 3 for h in hist]), repetition=uniform(R, 1.0, 1.3), frequency=uniform(R, 0.0, 0.5),
                presence=uniform(R, 0.0, 0.5), temperature=uniform(R, 0.5, 1.5), bias_tokens=bias_tokens,
                bias_values=uniform(int(bias_start[-1]), -5.0, 5.0), bias_start=bias_start,
                grammar=grammar if M else None, grammar_rows=rows if M else None,
                request=torch.arange(R, device="cuda").repeat_interleave(N).to(torch.int32),
                start=_ints([N * r for r in range(R + 1)]), mask=_masks(_parents(g, new, N), new, N),
                draft=(V * torch.rand(T, generator=g, device="cuda") ** 4).long().clamp(max=V - 1).to(torch.int32))


_PREPARE = {"plan": _prepare_plan, "write": _prepare_write, "attn": _prepare_attn, "norm": _prepare_norm,
            "logits": _prepare_logits}


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(s):
    return (_OWN if own else _PLAIN)[s["op"]](s)


def _own_plan(s):
    import paper_2509_18172_amd as sb
    p = sb.batch_plan(s["context"], s["new"], s["free"], s["table"], s["page"], s["tokens"], parents=s["parents"])
    return dict(table=s["table"], query_start=p.query_start, token_request=p.token_request, positions=p.positions,
                slots=p.slots, tree_mask=p.tree_mask, used=p.used)


def _own_write(s):
    import paper_2509_18172_amd as sb
    sb.cache_write(sb.KVCache(s["K"], s["V"]), s["k"], s["v"], s["slots"])
    return s["K"], s["V"]


def _own_attn(s):
    import paper_2509_18172_amd as sb
    return sb.tree_attention(s["q"], sb.KVCache(s["K"], s["V"]), s["table"], s["context"], s["start"], s["mask"],
                             max_new=s["max_new"], scale=s["scale"])


def _own_norm(s):
    import paper_2509_18172_amd as sb
    return sb.residual_norm(s["x"], s["y"], post_weight=s["post"], gate=s["gate"], scale=s["scale"],
                            pre_weight=s["pre"], eps=s["eps"])


def _own_logits(s):
    import paper_2509_18172_amd as sb
    return sb.adjust_logits(s["logits"], history=s["history"], history_start=s["history_start"],
                            prompt_lens=s["prompt"], repetition=s["repetition"], frequency=s["frequency"],
                            presence=s["presence"], temperature=s["temperature"], bias_tokens=s["bias_tokens"],
                            bias_values=s["bias_values"], bias_start=s["bias_start"], grammar=s["grammar"],
                            grammar_rows=s["grammar_rows"], token_request=s["request"], query_start=s["start"],
                            tree_mask=s["mask"], draft_tokens=s["draft"], out_dtype=torch.float32)


_OWN = {"plan": _own_plan, "write": _own_write, "attn": _own_attn, "norm": _own_norm, "logits": _own_logits}


def _plain_plan(s):
    ctx, new, free, table, P, T = s["context"].long(), s["new"].long(), s["free"], s["table"], s["page"], s["tokens"]
    R, width = table.shape
    start = torch.nn.functional.pad(new.cumsum(0), (1, 0)).clamp(max=T)
    have = (ctx + P - 1) // P
    need = (ctx + new + P - 1) // P - have
    first = need.cumsum(0) - need
    e = torch.arange(width, device="cuda")
    fresh = (e >= have[:, None]) & (e < (have + need)[:, None])
    n = first[:, None] + e - have[:, None]
    got = torch.where(n < free.numel(), free[n.clamp(0, free.numel() - 1)], -1)
    table.copy_(torch.where(fresh, got, table))
    t = torch.arange(T, device="cuda")
    real = t < start[-1]
    req = torch.searchsorted(start, t, right=True).sub(1).clamp(max=R - 1)
    j = t - start[req]
    at = ctx[req] + j
    page = torch.where(at // P < width, table[req, (at // P).clamp(max=width - 1)], -1).long()
    slots = torch.where(real & (page >= 0), page * P + at % P, -1)
    if s["parents"] is not None:
        mask, depth = _closure(s["parents"].long(), j, start[req])
    else:
        mask, depth = (torch.full_like(j, 2) << j) - 1, j
    return dict(table=table, query_start=start.int(), token_request=torch.where(real, req, -1).int(),
                positions=torch.where(real, ctx[req] + depth, 0).int(), slots=slots,
                tree_mask=torch.where(real, mask, 0), used=torch.stack([need.sum(), new.sum()]).int())


def _plain_write(s):
    P = s["K"].shape[1]
    keep = s["slots"] >= 0
    at = s["slots"][keep]
    s["K"].index_put_((at // P, at % P), s["k"][keep])
    s["V"].index_put_((at // P, at % P), s["v"][keep])
    return s["K"], s["V"]


def _plain_attn(s):
    K, V, table, ctx, start, q = s["K"], s["V"], s["table"], s["context"].long(), s["start"].long(), s["q"]
    R, P, N, L = table.shape[0], K.shape[1], s["max_new"], s["longest"]
    T, H, D = q.shape
    kvh = K.shape[2]
    new = start[1:] - start[:-1]
    pos = torch.arange(L, device="cuda")
    valid = pos < (ctx + new)[:, None]
    page = torch.where(valid, table[:, pos // P], table[:, :1]).long()
    k = K[page, pos % P].permute(0, 2, 3, 1).float().contiguous()       # R, kvh, D, L
    v = V[page, pos % P].permute(0, 2, 1, 3).float().contiguous()       # R, kvh, L, D
    i = torch.arange(N, device="cuda")
    rows = (start[:-1, None] + i).clamp(max=T - 1)
    qp = q[rows].float().view(R, N, kvh, H // kvh, D).permute(0, 2, 1, 3, 4).reshape(R, kvh, N * (H // kvh), D)
    back = pos - ctx[:, None]
    bit = (s["mask"][rows][:, :, None] >> back.clamp(0, 63)[:, None, :]) & 1
    seen = (back < 0)[:, None] | ((bit > 0) & ((back >= 0) & valid & (back < 64))[:, None])
    score = torch.matmul(qp, k).mul_(s["scale"]).view(R, kvh, N, H // kvh, L)
    score.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = score.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(R, kvh, -1, L), v).view(R, kvh, N, H // kvh, D)
    o = torch.where(total > 0, o / total, 0.0)
    o = o.permute(0, 2, 1, 3, 4).reshape(R, N, H, D)
    t = torch.arange(T, device="cuda")
    req = torch.searchsorted(start, t, right=True) - 1
    return o[req, t - start[req]].to(q.dtype)


def _plain_norm(s):
    def rms(t, w):
        return t * torch.rsqrt(t.square().mean(-1, keepdim=True) + s["eps"]) * w.float()
    z = s["y"].float()
    if s["post"] is not None:
        z = rms(z, s["post"])
    if s["gate"] is not None:
        z = z * s["gate"].float()
    x = s["x"].float() + s["scale"] * z
    return x.to(s["x"].dtype), rms(x, s["pre"]).to(s["y"].dtype)


def _plain_logits(s):
    T, V = s["logits"].shape
    R = s["prompt"].numel()
    req, start = s["request"].long(), s["history_start"].long()
    n = s["history"].numel()
    i = torch.arange(n, device="cuda")
    owner = torch.searchsorted(start, i, right=True) - 1
    generated = (i - start[owner] >= s["prompt"][owner]).float()
    word = s["history"].long()
    count = torch.zeros(R, V, device="cuda").index_put_((owner, word), generated, accumulate=True)[req]
    prompt = torch.zeros(R, V, device="cuda").index_put_((owner, word), 1 - generated, accumulate=True)[req]
    first, m = s["start"].long()[req], torch.arange(64, device="cuda")
    on = ((s["mask"][:, None] >> m) & 1).float()
    node = (first[:, None] + m).clamp(max=T - 1)
    count.scatter_add_(1, s["draft"].long()[node], on)
    l = s["logits"].float()
    rep = s["repetition"][req, None]
    l = torch.where((count > 0) | (prompt > 0), torch.where(l > 0, l / rep, l * rep), l)
    l = l - s["frequency"][req, None] * count - s["presence"][req, None] * (count > 0)
    which = torch.searchsorted(s["bias_start"].long(), torch.arange(s["bias_tokens"].numel(), device="cuda"),
                               right=True) - 1
    bias = torch.zeros(R, V, device="cuda").index_put_((which, s["bias_tokens"].long()), s["bias_values"])
    l = (l + bias[req]) / s["temperature"][req, None]
    if s["grammar"] is not None:
        v = torch.arange(V, device="cuda")
        row = s["grammar_rows"].long()
        bit = (s["grammar"][row.clamp(min=0)][:, v // 32] >> (v % 32)) & 1
        l = torch.where((bit > 0) | (row < 0)[:, None], l, -math.inf)
    return l


_PLAIN = {"plan": _plain_plan, "write": _plain_write, "attn": _plain_attn, "norm": _plain_norm,
          "logits": _plain_logits}


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    size = {"f16": 2, "bf16": 2, "f32": 4}
    op = case["op"]
    if op == "plan":
        ctx, new, P = _contexts(case), _news(case), case["page"]
        need = sum(-(-(c + n) // P) - -(-c // P) for c, n in zip(ctx, new))
        R, T = len(ctx), sum(new)
        return {"bytes": 12 * R + 4 + T * (24 + 4 * case["tree"]) + 8 * need + 8, "flops": 0}
    if op == "write":
        return {"bytes": case["tokens"] * (8 + 8 * case["kv_heads"] * case["dim"]), "flops": 0}
    if op == "attn":
        ctx, new = _contexts(case), _news(case)
        kv, row = case["kv_heads"] * case["dim"], case["heads"] * case["dim"]
        held = sum(c + n for c, n in zip(ctx, new))
        return {"bytes": 4 * kv * held + 4 * row * sum(new) + 4 * held // case["page"] + 8 * sum(new),
                "flops": 4 * row * sum(n * c + n * (n + 1) // 2 for c, n in zip(ctx, new))}
    if op == "norm":
        T, H, a, b = case["tokens"], case["width"], size[case["dtype"]], size[case["stream"]]
        per = 2 * a + 2 * b + (a if case["gate"] == "token" else 0)
        return {"bytes": T * H * per + H * a * (1 + case["post"] + (case["gate"] == "channel")),
                "flops": T * H * 10}
    T, V = case["requests"] * case["new"], case["vocab"]
    hist = sum(max(1, int(case["history"] * (1.0 - (0.6180339887498949 * r) % 1.0))) for r in range(case["requests"]))
    return {"bytes": T * V * (size[case["dtype"]] + 4) + 4 * hist + case["grammar"] * T * V / 8, "flops": T * V * 2}


# ---------------------------------------------------------------------------
# the definitions in binary64
# ---------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "plan":
        return None  # whole numbers only
    return {"write": _exact_write, "attn": _exact_attn, "norm": _exact_norm, "logits": _exact_logits}[case["op"]](s)


def _exact_write(s):
    out = []
    slots = s["slots"].cpu()
    for cache, new in ((s["K"], s["k"]), (s["V"], s["v"])):
        flat = cache.double().cpu().reshape(-1, *cache.shape[2:])
        rows = new.double().cpu()
        flat[slots[slots >= 0]] = rows[slots >= 0]
        out.append(flat.view(cache.shape))
    return tuple(out)


def _exact_attn(s):
    K, V, q = s["K"], s["V"], s["q"]
    P, kvh, D = K.shape[1:]
    H = q.shape[1]
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    start, masks = s["start"].tolist(), s["mask"].tolist()
    for r, c in enumerate(s["context"].tolist()):
        a, b = start[r], start[r + 1]
        n = b - a
        pages = s["table"][r, : -(-(c + n) // P)].long()
        k = K[pages].reshape(-1, kvh, D)[: c + n].double()
        v = V[pages].reshape(-1, kvh, D)[: c + n].double()
        seen = torch.ones(n, c + n, dtype=torch.bool, device="cuda")
        seen[:, c:] = torch.tensor([[bool((word >> j) & 1) for j in range(n)] for word in masks[a:b]], device="cuda")
        for h in range(H):
            kh, vh = k[:, h * kvh // H].contiguous(), v[:, h * kvh // H].contiguous()
            x = torch.mm(q[a:b, h].double(), kh.t().contiguous()) * s["scale"]
            w = torch.softmax(x.masked_fill(~seen, -math.inf), dim=-1)
            out[a:b, h] = torch.mm(w, vh)
    return out


def _exact_norm(s):
    x, y, eps = s["x"].double(), s["y"].double(), s["eps"]
    if s["post"] is not None:
        y = y / torch.sqrt((y * y).sum(1, keepdim=True) / y.shape[1] + eps) * s["post"].double()
    y = y if s["gate"] is None else y * s["gate"].double()
    x = x + y * s["scale"]
    return x, x / torch.sqrt((x * x).sum(1, keepdim=True) / x.shape[1] + eps) * s["pre"].double()


def _exact_logits(s):
    T, V = s["logits"].shape
    out = torch.empty(T, V, dtype=torch.float64, device="cuda")
    hs, bs, first = s["history_start"].tolist(), s["bias_start"].tolist(), s["start"].tolist()
    prompt, rows = s["prompt"].tolist(), None if s["grammar"] is None else s["grammar_rows"].tolist()
    masks = s["mask"].tolist()
    place = torch.arange(32, device="cuda", dtype=torch.int32)
    for t, r in enumerate(s["request"].tolist()):
        words = s["history"][hs[r]:hs[r + 1]].long()
        path = [first[r] + j for j in range(64) if (masks[t] >> j) & 1]
        done = torch.cat([words[prompt[r]:], s["draft"][path].long()])
        c = torch.bincount(done, minlength=V).double()
        known = c + torch.bincount(words[:prompt[r]], minlength=V)
        l = s["logits"][t].double()
        rep = float(s["repetition"][r])
        hit = known > 0
        l[hit & (l > 0)] /= rep
        l[hit & (l <= 0)] *= rep
        l -= float(s["frequency"][r]) * c
        l[c > 0] -= float(s["presence"][r])
        l[s["bias_tokens"][bs[r]:bs[r + 1]].long()] += s["bias_values"][bs[r]:bs[r + 1]].double()
        l /= float(s["temperature"][r])
        if rows is not None and rows[t] >= 0:
            allowed = ((s["grammar"][rows[t]][:, None] >> place) & 1).reshape(-1)[:V] > 0
            l[~allowed] = -math.inf
        out[t] = l
    return out
