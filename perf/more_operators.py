"""Operators of decoding with several sequences on one paged cache, as they are
timed and checked: the rotation of queries and keys by their positions (also
with the cache write in the same pass), the selection of a beam search, who uses
which page of the cache, the fork of sequences with a copy of the page that they
cannot share, and the compaction of a cache.

A case names an operator (``op``) and its sizes.  ``run`` makes one pass:
through the package's public calls where ``own`` is true, through elementary
torch operations where it is false -- in binary32, but for angles and the beams'
scores, which are binary64: at position 100000 a binary32 angle is off by 4e-3,
and which of two candidates is better may hang on the last bits of a long sum.
``exact`` gives the same outputs from the definitions in binary64.
"""
import math

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one token between the product and the cache of the 8B head layout: latency
        dict(name="rotary_1", op="rotary", tokens=1, heads=32, kv_heads=8, dim=128, pairs=64, axes=1, interleaved=False,
             dtype="f16", context=8192),
        # a prompt with images, the 70B head layout, positions in time, height and width
        dict(name="rotary_16384_3", op="rotary", tokens=16384, heads=64, kv_heads=8, dim=128, pairs=64, axes=3,
             interleaved=False, dtype="bf16", context=131072),
        # eight drafted tokens or beams: rotated, and keys and values written
        dict(name="rotary_write_8", op="rotary_write", tokens=8, heads=32, kv_heads=8, dim=128, pairs=64, axes=1,
             interleaved=False, dtype="f16", context=8192, page=16, layout="token"),
        # a prompt chunk, half of each head rotated, neighbours as pairs, pages kept head by head
        dict(name="rotary_write_8192", op="rotary_write", tokens=8192, heads=64, kv_heads=8, dim=128, pairs=32, axes=1,
             interleaved=True, dtype="bf16", context=131072, page=64, layout="head"),
        # one request with four beams on a vocabulary of odd size: latency
        dict(name="beam_1x4x50001", op="beam", requests=1, beams=4, n=4, vocab=50001, ends=1, dtype="f16"),
        # a full batch of beams on a large vocabulary, logits as their adjustment leaves them
        dict(name="beam_32x8x131072", op="beam", requests=32, beams=8, n=8, vocab=131072, ends=2, dtype="f32"),
        # a small server's pages
        dict(name="usage_8", op="usage", requests=2, beams=4, context=900, page=16, spare=512),
        # a full server's: 128 requests of eight beams
        dict(name="usage_1024_8k", op="usage", requests=128, beams=8, context=8192, page=16, spare=65536),
        # four beams of one request after a step, two layers' caches
        dict(name="fork_1x4", op="fork", requests=1, beams=4, context=1001, page=16, spare=64, layers=2, kv_heads=8,
             dim=128, dtype="f16", layout="token"),
        # a full batch of beams, larger pages, eight layers' caches
        dict(name="fork_64x8", op="fork", requests=64, beams=8, context=2048, page=64, spare=1024, layers=8, kv_heads=8,
             dim=128, dtype="bf16", layout="token"),
        # a small cache whose requests have come and gone
        dict(name="compact_8", op="compact", requests=2, beams=4, context=900, page=16, spare=512, layers=2, kv_heads=8,
             dim=128, dtype="f16", layout="head"),
        # a large one before a part of it is given back
        dict(name="compact_256_4k", op="compact", requests=256, beams=1, context=4096, page=64, spare=4096, layers=2,
             kv_heads=8, dim=128, dtype="bf16", layout="token"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("rotary", "rotary_write", "beam", "beam", "usage", "fork", "compact"))
    heads, kv_heads = rng.choice(((32, 8), (32, 8), (64, 8), (16, 16), (24, 4), (8, 1)))
    if op in ("rotary", "rotary_write"):
        dim = rng.choice((64, 80, 96, 128, 128))
        c = dict(op=op, tokens=_log_int(rng, 1, 16384 if op == "rotary" else 8192), heads=heads, kv_heads=kv_heads,
                 dim=dim, pairs=rng.choice((dim // 2, dim // 2, dim // 4, rng.randint(1, dim // 2))),
                 axes=rng.randint(1, 3), interleaved=rng.random() < 0.3, dtype=rng.choice(("f16", "bf16")),
                 context=_log_int(rng, 1, 1000000))
        if op == "rotary_write":
            c.update(page=2 ** rng.randint(4, 8), layout=rng.choice(("token", "head")))
        return c
    if op == "beam":
        B = rng.choice((1, 2, 3, 4, 5, 8, 12, 16))
        c = dict(op=op, requests=_log_int(rng, 1, 64), beams=B, n=rng.choice((B, B, 4, 2 * B)),
                 vocab=_log_int(rng, 1000, 131072), ends=rng.randint(0, 3), dtype=rng.choice(("f16", "bf16", "f32")))
        while c["requests"] * c["beams"] * c["vocab"] > 32 * 8 * 131072:
            c["requests"] = max(1, c["requests"] // 2)
        return c
    c = dict(op=op, requests=_log_int(rng, 1, 128), beams=rng.choice((1, 2, 4, 5, 8)), context=_log_int(rng, 1, 8192),
             page=2 ** rng.randint(4, 8), spare=_log_int(rng, 16, 4096))
    if op == "usage":
        return c
    c.update(layers=rng.randint(1, 6), kv_heads=kv_heads, dim=rng.choice((64, 80, 96, 128, 128)),
             dtype=rng.choice(("f16", "bf16")), layout=rng.choice(("token", "head")))
    # no more cached values than the largest listed caches, and no more to move
    while _pages(c)[1] * c["page"] * c["layers"] * c["kv_heads"] * c["dim"] > 1.5e9:
        if c["requests"] > 1:
            c["requests"] //= 2
        elif c["context"] > 64:
            c["context"] //= 2
        else:
            c["spare"], c["layers"] = max(16, c["spare"] // 2), max(1, c["layers"] - 1)
    return c


# ---------------------------------------------------------------------------
# sizes, the same for every seed
# ---------------------------------------------------------------------------

def _contexts(case):
    """Cached tokens of each request (all its beams have them): the first the
    longest, the others spread over the range below it."""
    return [max(0, int(case["context"] * (1.0 - (0.6180339887498949 * r) % 1.0))) for r in range(case["requests"])]


def _shared(case, length):
    """Full pages that a request's beams have in common: most of them."""
    return int(0.7 * length) // case["page"]


def _pages(case):
    """(pages in use, pages of the cache)"""
    P, B = case["page"], case["beams"]
    used = sum(_shared(case, c) + B * (-(-c // P) - _shared(case, c)) for c in _contexts(case))
    return used, used + B * case["requests"] + case["spare"]


def _going_on(case):
    """Beams of a request that have a continuation: about half, each the others'."""
    return (case["beams"] + 1) // 2


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    g = _generator(seed)
    return _PREPARE[case["op"]](case, g)


def _frequencies(pairs):
    return (10000.0 ** (-torch.arange(pairs, device="cuda", dtype=torch.float64) / pairs)).float()


def _prepare_rotary(case, g):
    T, H, K, D, A = case["tokens"], case["heads"], case["kv_heads"], case["dim"], case["axes"]
    # queries, keys and values as a joint product leaves them: views of one matrix's rows
    qkv = torch.randn(T, H + 2 * K, D, generator=g, device="cuda", dtype=DTYPES[case["dtype"]])
    first = torch.randint(0, case["context"], (A, 1), generator=g, device="cuda")
    t = torch.arange(T, device="cuda")
    if A == 1:
        positions = (first[0] + t).to(torch.int32)
    else:  # an image's time, row and column
        positions = (first + torch.stack([t // 1024, t // 32 % 32, t % 32])[:A]).to(torch.int32)
    axes = None
    if A > 1:  # a quarter of the pairs for time, the others shared by the rest
        i = torch.arange(case["pairs"], device="cuda")
        axes = torch.where(4 * i < case["pairs"], 0, 1 + (4 * i - case["pairs"]) * (A - 1) // (3 * case["pairs"]))
        axes = axes.clamp(max=A - 1).to(torch.int32)
    s = dict(op=case["op"], q=qkv[:, :H], k=qkv[:, H:H + K], v=qkv[:, H + K:], positions=positions, axes=axes,
             frequencies=_frequencies(case["pairs"]), interleaved=case["interleaved"])
    if case["op"] == "rotary_write":
        P = case["page"]
        pages = -(-T // P) + 4
        s["K"], s["V"] = [t[0] for t in _caches(g, 1, pages, case)]
        page = torch.randperm(pages, generator=g, device="cuda")
        at = t + 5
        s["slots"] = page[at // P] * P + at % P
        if T > 4:
            s["slots"][T // 2] = -1  # a token of a request that found no page
    return s


def _prepare_beam(case, g):
    R, B, V, E = case["requests"], case["beams"], case["vocab"], case["ends"]
    logits = (3 * torch.randn(R * B, V, generator=g, device="cuda")).to(DTYPES[case["dtype"]])
    # a grammar or a list of forbidden tokens has taken some of them out
    logits.masked_fill_(torch.rand(R * B, V, generator=g, device="cuda") < 0.1, -math.inf)
    scores = -5.0 - 3.0 * torch.rand(R, B, generator=g, device="cuda").cumsum(1)
    if B > 2:
        scores[::3, -1] = -math.inf  # a beam that has ended
    ends = None
    if E:
        ends = torch.randperm(V, generator=g, device="cuda")[:E].to(torch.int32)
        # some beams come to their end
        logits[::3, ends[0].long()] = logits[::3].amax(1)
    return dict(op="beam", logits=logits, scores=scores, n=case["n"], ends=ends)


def _prepare_pages(case, g):
    ctx, P, B = _contexts(case), case["page"], case["beams"]
    R, (used, pages) = case["requests"], _pages(case)
    width = (case["context"] + P) // P + 1
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    shared = torch.tensor([_shared(case, c) for c in ctx], device="cuda")
    count = torch.tensor([-(-c // P) for c in ctx], device="cuda")
    own_pages = count - shared
    start = shared + B * own_pages
    start = start.cumsum(0) - start
    e, b = torch.arange(width, device="cuda"), torch.arange(B, device="cuda")
    number = torch.where(e < shared[:, None, None], start[:, None, None] + e,
                         start[:, None, None] + shared[:, None, None] + b[:, None] * own_pages[:, None, None]
                         + e - shared[:, None, None])
    table = torch.where(e < count[:, None, None], order[number.clamp(max=pages - 1)], -1).view(R * B, width)
    return dict(op=case["op"], table=table.to(torch.int32), context=_ints([c for c in ctx for _ in range(B)]), page=P,
                pages=pages, beams=B, order=order, used=used)


def _caches(g, layers, pages, case):
    """Keys and values [layers][pages][page][heads][dim]; "head": stored head by
    head within a page."""
    P, H, D = case["page"], case["kv_heads"], case["dim"]
    shape = (layers, pages, P, H, D) if case["layout"] == "token" else (layers, pages, H, P, D)
    kv = [torch.randn(shape, generator=g, device="cuda", dtype=DTYPES[case["dtype"]]) for _ in range(2)]
    return kv if case["layout"] == "token" else [t.transpose(2, 3) for t in kv]


def _prepare_fork(case, g):
    s, R, B = _prepare_pages(case, g), case["requests"], case["beams"]
    s["K"], s["V"] = _caches(g, case["layers"], s["pages"], case)
    free = torch.full((s["pages"],), -1, dtype=torch.int32, device="cuda")
    free[: s["pages"] - s["used"]] = s["order"][s["used"]:].sort().values
    # the parents of a request's next beams: as many different ones for every seed
    some = torch.rand(R, B, generator=g, device="cuda").argsort(1)
    pick = torch.arange(B, device="cuda") % _going_on(case)
    pick = pick[torch.rand(R, B, generator=g, device="cuda").argsort(1)]
    return dict(s, free=free, parents=some.gather(1, pick).to(torch.int32))


def _prepare_compact(case, g):
    s = _prepare_pages(case, g)
    s["K"], s["V"] = _caches(g, case["layers"], s["pages"], case)
    return s


_PREPARE = {"rotary": _prepare_rotary, "rotary_write": _prepare_rotary, "beam": _prepare_beam, "usage": _prepare_pages,
            "fork": _prepare_fork, "compact": _prepare_compact}


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(s):
    return (_OWN if own else _PLAIN)[s["op"]](s)


def _own_rotary(s):
    import paper_2509_18172_amd as sb
    return sb.rotary(s["q"], s["k"], s["positions"], s["frequencies"], axes=s["axes"], interleaved=s["interleaved"])


def _own_rotary_write(s):
    import paper_2509_18172_amd as sb
    q = sb.rotary_write(s["q"], sb.KVCache(s["K"], s["V"]), s["k"], s["v"], s["slots"], s["positions"],
                        s["frequencies"], axes=s["axes"], interleaved=s["interleaved"])
    return q, s["K"], s["V"]


def _own_beam(s):
    import paper_2509_18172_amd as sb
    c = sb.beam_select(s["logits"], s["scores"], n=s["n"], end_tokens=s["ends"])
    return dict(tokens=c.tokens, parents=c.parents, scores=c.scores, ended=c.ended, ended_tokens=c.ended_tokens)


def _own_usage(s):
    import paper_2509_18172_amd as sb
    u = sb.page_usage(s["context"], s["table"], s["page"], s["pages"])
    return dict(refs=u.refs, free=u.free_pages, counts=u.counts)


def _own_fork(s):
    import paper_2509_18172_amd as sb
    f = sb.page_fork(s["context"], s["table"], s["parents"], s["page"], s["free"])
    sb.page_copy([sb.KVCache(k, v) for k, v in zip(s["K"], s["V"])], f.src, f.dst, f.tokens)
    return dict(table=f.page_table, context=f.context_lens, src=f.src, dst=f.dst, tokens=f.tokens, used=f.used, K=s["K"],
                V=s["V"])


def _own_compact(s):
    import paper_2509_18172_amd as sb
    c = sb.page_compact(s["context"], s["table"], s["page"], s["pages"])
    sb.page_copy([sb.KVCache(k, v) for k, v in zip(s["K"], s["V"])], c.src, c.dst)
    return dict(table=c.page_table, src=c.src, dst=c.dst, counts=c.counts, K=s["K"], V=s["V"])


_OWN = {"rotary": _own_rotary, "rotary_write": _own_rotary_write, "beam": _own_beam, "usage": _own_usage,
        "fork": _own_fork, "compact": _own_compact}


def _rotated(x, s):
    """x rounded once; cosines and sines from angles in 64 bits."""
    position = s["positions"].double() if s["axes"] is None else s["positions"].double()[s["axes"].long()].t()
    position = position if position.dim() == 2 else position[:, None]
    angle = (position * s["frequencies"].double())[:, None]
    cos, sin = angle.cos().float(), angle.sin().float()
    n = s["frequencies"].numel()
    f = x.float()
    if s["interleaved"]:
        a, b = f[..., 0:2 * n:2], f[..., 1:2 * n:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    else:
        a, b = f[..., :n], f[..., n:2 * n]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    return torch.cat([turned, f[..., 2 * n:]], dim=-1).to(x.dtype)


def _plain_rotary(s):
    return _rotated(s["q"], s), _rotated(s["k"], s)


def _plain_rotary_write(s):
    P = s["K"].shape[1]
    keep = s["slots"] >= 0
    at = s["slots"][keep]
    s["K"].index_put_((at // P, at % P), _rotated(s["k"], s)[keep])
    s["V"].index_put_((at // P, at % P), s["v"][keep])
    return _rotated(s["q"], s), s["K"], s["V"]


def _plain_beam(s):
    R, B = s["scores"].shape
    V, n, ends = s["logits"].shape[1], s["n"], s["ends"]
    x = s["logits"].double()
    top = x.amax(1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    score = x - top - (x - top).exp_().sum(1, keepdim=True).log()
    score = (score.view(R, B, V) + s["scores"].double()[:, :, None]).view(R, B * V)
    # the best of all, enough that n of them are no ends: first those above the
    # value that the last of them has, then of those that have it the lowest
    m = min(n + B * (0 if ends is None else ends.numel()), B * V)
    last = score.topk(m).values[:, -1:]
    index = torch.arange(B * V, device="cuda")
    order = torch.where(score > last, 2 * B * V, torch.where(score == last, B * V, 0)) - index
    best = order.topk(m).indices.sort(1).values
    value, by = score.gather(1, best).sort(dim=1, descending=True, stable=True)
    best = best.gather(1, by)
    real = value > -math.inf
    token, beam = best % V, best // V
    end = torch.zeros_like(real) if ends is None else (token[:, :, None] == ends).any(-1)
    # the first n that go on
    place = (real & ~end).cumsum(1) - 1
    takes = (place[:, None] == torch.arange(n, device="cuda")[:, None]) & (real & ~end)[:, None]
    pick, there = takes.long().argmax(2), takes.any(2)
    # the best end of each beam, if it is among the n best of all
    at = torch.arange(m, device="cuda")
    ends_here = (beam[:, None] == torch.arange(B, device="cuda")[:, None]) & (real & end & (at < n))[:, None]
    stop, stops = ends_here.long().argmax(2), ends_here.any(2)
    return dict(tokens=torch.where(there, token.gather(1, pick), -1).int(),
                parents=torch.where(there, beam.gather(1, pick), -1).int(),
                scores=torch.where(there, value.gather(1, pick), -math.inf).float(),
                ended=torch.where(stops, value.gather(1, stop), -math.inf).float(),
                ended_tokens=torch.where(stops, token.gather(1, stop), -1).int())


def _in_use(s):
    e = torch.arange(s["table"].shape[1], device="cuda")
    return e < ((s["context"].long() + s["page"] - 1) // s["page"])[:, None]


def _references(s):
    refs = torch.zeros(s["pages"] + 1, dtype=torch.int32, device="cuda")
    at = torch.where(_in_use(s), s["table"], s["pages"]).long().view(-1)
    return refs.index_add_(0, at, torch.ones_like(at, dtype=torch.int32))[:-1]


def _plain_usage(s):
    refs = _references(s)
    number = torch.arange(s["pages"], device="cuda")
    free = torch.where(refs == 0, number, s["pages"]).sort().values
    n = (refs == 0).sum()
    return dict(refs=refs, free=torch.where(number < n, free, -1).int(), counts=torch.stack([n, s["pages"] - n]).int())


def _copied(cache, src, dst, tokens):
    """Copies the first tokens of pages src to pages dst, in all layers."""
    real = src >= 0
    src, dst, tokens = src[real].long(), dst[real].long(), tokens[real]
    here = torch.arange(cache.shape[2], device="cuda") < tokens[:, None]
    moved = torch.where(here[None, :, :, None, None], cache[:, src], cache[:, dst])
    cache.index_put_((torch.arange(cache.shape[0], device="cuda")[:, None], dst), moved)


def _plain_fork(s):
    B, P, table = s["beams"], s["page"], s["table"]
    rows, width = table.shape
    i = torch.arange(rows, device="cuda")
    parent = i // B * B + s["parents"].view(-1)
    context = s["context"][parent]
    full, part = context.long() // P, context % P
    first = torch.full((rows,), rows, device="cuda").scatter_reduce(0, parent, i, "amin")
    takes = (part > 0) & (first[parent] != i)
    k = takes.cumsum(0) - 1
    new = torch.where(takes, s["free"][k.clamp(0, s["free"].numel() - 1)], -1)
    e = torch.arange(width, device="cuda")
    out = torch.where(_in_use(s), table, -1)[parent]
    out = torch.where((e == full[:, None]) & takes[:, None], new[:, None], out)
    src = torch.where(takes, table[parent, full.clamp(max=width - 1)], -1)
    tokens = torch.where(takes, part, 0).int()
    for cache in (s["K"], s["V"]):
        _copied(cache, src, new, tokens)
    return dict(table=out, context=context, src=src, dst=new, tokens=tokens, used=takes.sum().view(1).int(), K=s["K"],
                V=s["V"])


def _plain_compact(s):
    pages = s["pages"]
    used = _references(s) > 0
    n = used.sum()
    number = torch.arange(pages, device="cuda")
    moves = used & (number >= n)
    gaps = torch.where(~used & (number < n), number, pages).sort().values
    k = (moves.cumsum(0) - 1).clamp(min=0)
    new = torch.where(moves, gaps[k], number)
    src = torch.where(moves, number, pages).sort().values[: pages // 2]
    there = torch.arange(pages // 2, device="cuda") < moves.sum()
    src, dst = torch.where(there, src, -1).int(), torch.where(there, gaps[: pages // 2], -1).int()
    out = torch.where(_in_use(s), new[s["table"].long().clamp(min=0)], -1).int()
    for cache in (s["K"], s["V"]):
        _copied(cache, src, dst, torch.full_like(src, s["page"]))
    return dict(table=out, src=src, dst=dst, counts=torch.stack([n, moves.sum()]).int(), K=s["K"], V=s["V"])


_PLAIN = {"rotary": _plain_rotary, "rotary_write": _plain_rotary_write, "beam": _plain_beam, "usage": _plain_usage,
          "fork": _plain_fork, "compact": _plain_compact}


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    op = case["op"]
    if op in ("rotary", "rotary_write"):
        T, row = case["tokens"], case["dim"] * (case["heads"] + case["kv_heads"])
        if op == "rotary_write":
            row += case["dim"] * case["kv_heads"]
        turned = 2 * case["pairs"] * (case["heads"] + case["kv_heads"])
        return {"bytes": 4 * T * row + T * (4 * case["axes"] + 8 * (op == "rotary_write")), "flops": 3 * T * turned}
    if op == "beam":
        rows = case["requests"] * case["beams"]
        # the rows of beams that have ended need not be read
        rows -= -(-case["requests"] // 3) if case["beams"] > 2 else 0
        size = {"f16": 2, "bf16": 2, "f32": 4}[case["dtype"]]
        return {"bytes": rows * case["vocab"] * size + case["requests"] * (12 * case["n"] + 12 * case["beams"]),
                "flops": 4 * rows * case["vocab"]}
    ctx, P, B = _contexts(case), case["page"], case["beams"]
    used, pages = _pages(case)
    entries = B * sum(-(-c // P) for c in ctx)
    width = (case["context"] + P) // P + 1
    if op == "usage":
        return {"bytes": 4 * entries + 4 * B * len(ctx) + 8 * pages, "flops": 0}
    token = 8 * case["layers"] * case["kv_heads"] * case["dim"]  # of keys and values, in and out
    if op == "fork":
        moved = (B - _going_on(case)) * sum(c % P for c in ctx)
    else:
        moved = used * (pages - used) // pages * P
    return {"bytes": 4 * entries + 4 * B * len(ctx) * width + moved * token, "flops": 0}


# ---------------------------------------------------------------------------
# the definitions in binary64
# ---------------------------------------------------------------------------

def exact(case, seed):
    if case["op"] == "usage":
        return None  # whole numbers only
    s = prepare(case, seed)
    return {"rotary": _exact_rotary, "rotary_write": _exact_rotary, "beam": _exact_beam, "fork": _exact_fork,
            "compact": _exact_compact}[case["op"]](s)


def _exact_rotary(s):
    n, out = s["frequencies"].numel(), []
    axis = [0] * n if s["axes"] is None else s["axes"].tolist()
    positions = s["positions"].view(-1, s["q"].shape[0]).double()
    for x in (s["q"], s["k"]):
        y = x.double()
        for i in range(n):
            a, b = (2 * i, 2 * i + 1) if s["interleaved"] else (i, i + n)
            turn = torch.polar(torch.ones_like(positions[0]), positions[axis[i]] * float(s["frequencies"][i]))
            z = torch.complex(x[..., a].double(), x[..., b].double()) * turn[:, None]
            y[..., a], y[..., b] = z.real, z.imag
        out.append(y)
    if s["op"] == "rotary":
        return tuple(out)
    slots = s["slots"].cpu()
    caches = []
    for cache, new in ((s["K"], out[1]), (s["V"], s["v"].double())):
        flat = cache.double().cpu().reshape(-1, *cache.shape[2:])
        flat[slots[slots >= 0]] = new.cpu()[slots >= 0]
        caches.append(flat.view(cache.shape))
    return out[0], caches[0], caches[1]


def _exact_beam(s):
    R, B = s["scores"].shape
    n, ends = s["n"], [] if s["ends"] is None else s["ends"].tolist()
    scores, ended = torch.full((R, n), -math.inf, dtype=torch.float64), torch.full((R, B), -math.inf, dtype=torch.float64)
    base, keep = s["scores"].tolist(), n + len(ends)
    for r in range(R):
        found = []
        for b in range(B):
            if base[r][b] == -math.inf:
                continue
            l = torch.log_softmax(s["logits"][r * B + b].double(), dim=0)
            v, at = l.sort(dim=0, descending=True, stable=True)
            found += [(-(base[r][b] + x), b, t) for x, t in zip(v[:keep].tolist(), at[:keep].tolist()) if x > -math.inf]
        found.sort()
        on = [-x for x, b, t in found if t not in ends][:n]
        scores[r, : len(on)] = torch.tensor(on, dtype=torch.float64)
        for x, b, t in found[:n]:
            if t in ends:
                ended[r, b] = max(float(ended[r, b]), -x)
    return dict(tokens=None, parents=None, scores=scores, ended=ended, ended_tokens=None)


def _exact_fork(s):
    B, P = s["beams"], s["page"]
    table, context = s["table"].tolist(), s["context"].tolist()
    free = [p for p in s["free"].tolist() if p >= 0]
    K, V = s["K"].double(), s["V"].double()
    kept = set()
    for i, p in enumerate(s["parents"].view(-1).tolist()):
        p += i // B * B
        part = context[p] % P
        if part and p in kept:
            src, dst = table[p][context[p] // P], free.pop(0)
            for cache, old in ((K, s["K"]), (V, s["V"])):
                cache[:, dst, :part] = old[:, src, :part].double()
        kept.add(p)
    return dict(table=None, context=None, src=None, dst=None, tokens=None, used=None, K=K, V=V)


def _exact_compact(s):
    P, used = s["page"], set()
    for row, c in zip(s["table"].tolist(), s["context"].tolist()):
        used.update(row[: -(-c // P)])
    K, V = s["K"].double(), s["V"].double()
    gaps = [p for p in range(len(used)) if p not in used]
    for src, dst in zip(sorted(p for p in used if p >= len(used)), gaps):
        for cache, old in ((K, s["K"]), (V, s["V"])):
            cache[:, dst] = old[:, src].double()
    return dict(table=None, src=None, dst=None, counts=None, K=K, V=V)
