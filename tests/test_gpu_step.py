"""The operators between the products of a step against plain implementations
in 64 bits, at the sizes, masks and layouts where they can go wrong."""
import math

import numpy as np
import pytest
import torch

import paper_2509_18172_amd as sb

pytestmark = pytest.mark.gpu

DEV = "cuda"
# one rounding, relative: 2^-p for the p significant bits of the type (11, 8, 24)
HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


# ---------------------------------------------------------------------------
# the plan
# ---------------------------------------------------------------------------

def plan_reference(ctx, new, free, table, P, T, parents):
    """Straight from the definition, request by request, token by token."""
    table = [list(row) for row in table]
    width = len(table[0])
    start, request, position, slot, mask = [], [], [], [], []
    taken = tokens = 0
    for r, (c, n) in enumerate(zip(ctx, new)):
        c, n = max(c, 0), max(n, 0)
        start.append(min(tokens, T))
        have = min(-(-c // P), width)
        need = max(min(-(-(c + n) // P), width) - have, 0)
        for i in range(need):
            table[r][have + i] = free[taken + i] if taken + i < len(free) else -1
        taken += need
        seen = []
        for j in range(min(n, max(T - tokens, 0))):
            p = (parents[tokens + j] if parents is not None else j - 1) if n <= 64 else j - 1
            up = seen[p] if 0 <= p < j else set()
            seen.append(up | {j})
            request.append(r)
            position.append(c + len(seen[-1]) - 1)
            e = (c + j) // P
            page = table[r][e] if e < width else -1
            slot.append(page * P + (c + j) % P if page >= 0 else -1)
            mask.append(sum(1 << i for i in seen[-1]) if n <= 64 else 0)
        tokens += n
    start.append(min(tokens, T))
    pad = T - len(request)
    mask = [m - (1 << 64) if m >= 1 << 63 else m for m in mask]
    return dict(query_start=start, token_request=request + [-1] * pad, positions=position + [0] * pad,
                slots=slot + [-1] * pad, tree_mask=mask + [0] * pad, used=[taken, tokens]), table


def check_plan(ctx, new, free, width, P, T, parents=None, stride=None, seed=0):
    rng = np.random.default_rng(seed)
    R = len(ctx)
    table = rng.integers(-1, 1000, size=(R, width)).tolist()
    want, want_table = plan_reference(ctx, new, free, table, P, T, parents)
    full = torch.full((R, stride or width), 7777, dtype=torch.int32, device=DEV)
    full[:, :width] = i32(table)
    p = sb.batch_plan(i32(ctx), i32(new), i32(free), full[:, :width], P, T,
                      parents=None if parents is None else i32(parents))
    for name, value in want.items():
        assert getattr(p, name).tolist() == value, name
    assert full[:, :width].tolist() == want_table
    assert bool((full[:, width:] == 7777).all())


PLANS = {
    "one_token": ([900], [1], 3, 60, 16, 1),
    "first_token": ([0], [1], 3, 4, 16, 1),
    "page_filled": ([16, 32, 15], [1, 16, 2], 9, 8, 16, 19),
    "nothing_new": ([5, 0, 40], [0, 0, 0], 4, 8, 16, 0),
    "some_empty": ([5, 0, 40, 7, 0], [0, 3, 0, 9, 0], 4, 8, 16, 12),
    "padded": ([31, 64], [4, 5], 6, 8, 32, 300),
    "cut": ([31, 64, 3], [40, 50, 9], 12, 8, 32, 63),
    "free_list_short": ([0, 0, 0], [40, 40, 40], 5, 8, 16, 120),
    "free_list_empty": ([10, 16], [3, 4], 0, 8, 16, 7),
    "table_short": ([50, 200, 3], [40, 9, 100], 20, 4, 16, 149),
    "long_prompt": ([0, 70], [1000, 64], 90, 70, 16, 1064),
    "negative": ([-5, 7], [3, -2], 4, 8, 16, 5),
    "long_context": ([2 ** 31 - 100], [20], 4, 1 << 19, 4096, 20),
}


@pytest.mark.parametrize("name", PLANS)
@pytest.mark.parametrize("tree", [False, True])
def test_plan(name, tree):
    ctx, new, n_free, width, P, T = PLANS[name]
    rng = np.random.default_rng(3)
    free = rng.permutation(5000)[:n_free].tolist()
    parents = None
    if tree:
        # any earlier token of the request, roots, and indices that name no earlier token
        parents = [int(v) for n in new for j in range(max(n, 0)) for v in [rng.integers(-2, j + 3)]][:T]
        parents += [0] * (T - len(parents))
    check_plan(ctx, new, free, width, P, T, parents, stride=width + 3)


@pytest.mark.parametrize("seed", range(6))
def test_plan_random(seed):
    rng = np.random.default_rng(100 + seed)
    R = [1, 63, 64, 257, 1000, 4096][seed]
    P = int(2 ** rng.integers(4, 9))
    ctx = rng.integers(0, 700, R).tolist()
    new = rng.integers(0, 66 if R < 1000 else 5, R).tolist()
    T = sum(new) + int(rng.integers(-3, 4)) if sum(new) > 3 else sum(new)
    total = sum(-(-(c + n) // P) - -(-c // P) for c, n in zip(ctx, new))
    parents = [int(rng.integers(-1, max(j, 1))) for n in new for j in range(n)][:T]
    parents += [0] * (T - len(parents))
    check_plan(ctx, new, rng.permutation(total + 5).tolist(), (700 + 66) // P + 2, P, T, parents, seed=seed)


# ---------------------------------------------------------------------------
# the cache write
# ---------------------------------------------------------------------------

def make_cache(pages, P, heads, dim, dtype, layout, fill=None, gen=None):
    shape = {"token": (pages, P, heads, dim), "head": (pages, heads, P, dim), "pair": (pages, 2, P, heads, dim)}[layout]
    t = [torch.empty(shape, dtype=dtype, device=DEV) for _ in range(1 if layout == "pair" else 2)]
    for x in t:
        if fill is None:
            x.normal_(generator=gen)
        else:
            x.fill_(fill)
    if layout == "pair":
        return sb.KVCache(t[0][:, 0], t[0][:, 1])
    return sb.KVCache(*[x.transpose(1, 2) if layout == "head" else x for x in t])


@pytest.mark.parametrize("T", [1, 2, 17, 300])
@pytest.mark.parametrize("heads,dim,P,dtype,layout", [(8, 128, 16, torch.float16, "token"), (1, 8, 16, torch.bfloat16, "head"),
                                                      (3, 80, 64, torch.float16, "pair"), (40, 128, 32, torch.bfloat16, "head")])
def test_cache_write(T, heads, dim, P, dtype, layout):
    gen = torch.Generator(device=DEV).manual_seed(T)
    pages = -(-T // P) + 3
    cache = make_cache(pages, P, heads, dim, dtype, layout, gen=gen)
    joint = torch.randn(T, 3 * heads * dim, generator=gen, device=DEV).to(dtype)
    k = joint[:, :heads * dim].view(T, heads, dim)
    v = joint[:, 2 * heads * dim:].view(T, heads, dim)
    slots = torch.randperm(pages * P, generator=gen, device=DEV)[:T]
    if T > 2:
        slots[1] = -1
        slots[2] = pages * P  # one past the cache
        slots[T // 2] = -(1 << 40)
    want_k, want_v = cache.k.clone(), cache.v.clone()
    for t, s in enumerate(slots.tolist()):
        if 0 <= s < pages * P:
            want_k[s // P, s % P] = k[t]
            want_v[s // P, s % P] = v[t]
    sb.cache_write(cache, k, v, slots)
    assert torch.equal(cache.k, want_k) and torch.equal(cache.v, want_v)


def test_cache_write_nothing():
    cache = make_cache(2, 16, 2, 64, torch.float16, "token", fill=3.0)
    none = torch.empty(0, 2, 64, dtype=torch.float16, device=DEV)
    sb.cache_write(cache, none, none, torch.empty(0, dtype=torch.int64, device=DEV))
    assert bool((cache.k == 3).all())


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------

def attention_reference(q, cache, table, ctx, start, mask, max_new, scale):
    """(output, sum of weights times magnitudes) in binary64 on the CPU; only
    what a row sees is looked at."""
    T, H, D = q.shape
    pages, P, KH, _ = cache.k.shape
    out, size = np.zeros((T, H, D)), np.zeros((T, H, D))
    qd = q.double().cpu().numpy()
    table = table.cpu().numpy()
    for r in range(len(ctx)):
        n = min(start[r + 1] - start[r], max_new)
        span = np.arange(ctx[r] + n)
        page = table[r][span // P] if len(span) else np.zeros(0, dtype=np.int64)
        ok = (page >= 0) & (page < pages)
        index = torch.from_numpy(np.where(ok, page, 0).astype(np.int64)).to(DEV), torch.from_numpy(span % P).to(DEV)
        k, v = (t[index].double().cpu().numpy() for t in (cache.k, cache.v))
        for j in range(n):
            t = start[r] + j
            bits = int(mask[t])
            seen = ok & ((span < ctx[r]) | np.array([p >= ctx[r] and (bits >> int(p - ctx[r])) & 1 for p in span], dtype=bool))
            if not seen.any():
                continue
            for h in range(H):
                kh = h // (H // KH)
                s = k[seen][:, kh] @ qd[t, h] * scale
                w = np.exp(s - s.max())
                w /= w.sum()
                out[t, h] = w @ v[seen][:, kh]
                size[t, h] = w @ np.abs(v[seen][:, kh])
    return out, size


def attention_bound(want, size, dtype, longest, vmax):
    """Rounding of the weights and of the output, the binary32 exponentials
    and sums, and weights that become subnormal in binary16."""
    u = HALF[dtype]
    return 1.01 * u * (size + np.abs(want)) + 2.0 ** -15 * size + (longest * 2.0 ** -25 * vmax if dtype == torch.float16 else 0) + 1e-30


def tree_batch(news, gen_seed, kind="tree"):
    rng = np.random.default_rng(gen_seed)
    masks = []
    for n in news:
        rows = []
        for j in range(n):
            p = j - 1 if kind == "chain" else int(rng.integers(-1, j)) if j else -1
            rows.append((1 << j) | (rows[p] if p >= 0 else 0))
        masks += rows
    if kind == "any":  # not a tree: arbitrary bits, some rows with none
        masks = [int(rng.integers(0, 1 << 62)) & int(rng.integers(0, 1 << 62)) if i % 3 else 0 for i in range(len(masks))]
    return [m - (1 << 64) if m >= 1 << 63 else m for m in masks]


def run_attention(news, ctx, heads, kv_heads, dim, P, dtype, layout="token", kind="tree", garbage=False, extra=0, seed=0,
                  scale=None, q_view=False, edit=None):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    R, T = len(ctx), sum(news)
    count = [-(-(c + n) // P) for c, n in zip(ctx, news)]
    width = max(max(count), 1) + 1
    pages = sum(count) + 2
    cache = make_cache(pages, P, kv_heads, dim, dtype, layout, fill=float("nan") if garbage else None, gen=gen)
    table = torch.full((R, width), -1, dtype=torch.int32)
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    at = 0
    for r in range(R):
        table[r, :count[r]] = order[at:at + count[r]]
        at += count[r]
    if garbage:  # NaN everywhere but in the requests' own positions
        for r in range(R):
            for p in range(ctx[r] + news[r]):
                for t in (cache.k, cache.v):
                    t[int(table[r, p // P]), p % P] = torch.randn(kv_heads, dim, generator=gen, device=DEV).to(dtype)
    table = table.to(DEV)
    start = [sum(news[:r]) for r in range(R + 1)]
    mask = tree_batch(news, seed, kind)
    if edit:
        edit(cache, table, mask)
    wide = torch.randn(T + extra, heads + 2 * q_view, dim + 8 * q_view, generator=gen, device=DEV).to(dtype)
    q = wide[:, 1:-1, :dim] if q_view else wide
    scale = dim ** -0.5 if scale is None else scale
    out = torch.full((T + extra, heads, dim), 5.0, dtype=dtype, device=DEV)
    masks = torch.tensor(mask + [0] * extra, dtype=torch.int64, device=DEV)
    got = sb.tree_attention(q, cache, table, i32(ctx), i32(start), masks, max(max(news), 1), scale=scale, out=out)
    want, size = attention_reference(q, cache, table, ctx, start, mask, max(max(news), 1), scale)
    return got, want, size, cache


def compare_attention(got, want, size, dtype, longest, T):
    g = got.double().cpu().numpy()
    bound = attention_bound(want[:T], size[:T], dtype, longest, 8.0)
    assert np.isfinite(g[:T]).all()
    err = np.abs(g[:T] - want[:T])
    assert (err <= bound).all(), (err / bound).max()
    assert (g[T:] == 5.0).all()


ATTN = [
    # news, contexts, heads, kv heads, dim, page, dtype, layout
    ([1], [0], 1, 1, 64, 16, torch.float16, "token"),
    ([1], [1], 4, 1, 128, 16, torch.bfloat16, "head"),
    ([1], [1000], 32, 8, 128, 16, torch.float16, "token"),
    ([8], [333], 32, 8, 128, 64, torch.float16, "pair"),
    ([8, 3, 1, 5], [500, 0, 47, 128], 8, 2, 128, 16, torch.bfloat16, "token"),
    ([64], [130], 8, 1, 128, 32, torch.float16, "head"),
    ([64, 1, 33], [0, 700, 63], 16, 4, 64, 16, torch.bfloat16, "token"),
    ([5, 16], [100, 31], 6, 2, 80, 16, torch.float16, "token"),
    ([7], [260], 3, 3, 96, 128, torch.bfloat16, "head"),
    ([2, 2], [15, 16], 12, 1, 72, 16, torch.float16, "token"),
    ([4], [90], 2, 2, 8, 16, torch.float16, "token"),
    ([9], [77], 5, 1, 40, 32, torch.bfloat16, "head"),
    ([1] * 20, list(range(0, 400, 20)), 8, 8, 64, 16, torch.float16, "token"),
    ([0, 6, 0, 1], [50, 70, 0, 9], 8, 2, 128, 16, torch.float16, "token"),
    ([3], [4096 + 17], 4, 2, 128, 4096, torch.bfloat16, "token"),
    ([17, 1], [3000, 2999], 64, 8, 128, 64, torch.bfloat16, "token"),
]


@pytest.mark.parametrize("case", range(len(ATTN)))
@pytest.mark.parametrize("kind", ["tree", "chain"])
def test_attention(case, kind):
    news, ctx, H, KH, D, P, dtype, layout = ATTN[case]
    got, want, size, _ = run_attention(news, ctx, H, KH, D, P, dtype, layout, kind, seed=case, extra=case % 3)
    compare_attention(got, want, size, dtype, max(ctx) + max(news), sum(news))


@pytest.mark.parametrize("case", [0, 2, 4, 6, 7, 10, 13])
def test_attention_unseen_slots_hold_nan(case):
    news, ctx, H, KH, D, P, dtype, layout = ATTN[case]
    got, want, size, _ = run_attention(news, ctx, H, KH, D, P, dtype, layout, seed=case, garbage=True)
    compare_attention(got, want, size, dtype, max(ctx) + max(news), sum(news))


@pytest.mark.parametrize("news,ctx", [([12], [0]), ([40, 12], [0, 75]), ([64], [40])])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_attention_any_mask_and_empty_rows(news, ctx, dtype):
    """Masks that are no trees; a row that sees nothing gives 0."""
    got, want, size, _ = run_attention(news, ctx, 8, 2, 128, 16, dtype, kind="any", seed=5)
    compare_attention(got, want, size, dtype, max(ctx) + max(news), sum(news))
    if ctx[0] == 0:
        assert bool((got[0] == 0).all())


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("where", ["k", "v", "kv"])
@pytest.mark.parametrize("n,c,dim", [(9, 50, 128), (40, 0, 64), (9, 21, 80)])
def test_attention_bad_values_in_masked_tokens(bad, dtype, where, n, c, dim):
    """A drafted token with NaN or infinities reaches the rows that see it
    and no others."""
    def edit(cache, table, mask):
        P = cache.k.shape[1]
        for name in where:
            for j in (2, n - 3):
                p = c + j
                getattr(cache, name)[int(table[0, p // P]), p % P, :, 3:7] = bad
    got, want, size, _ = run_attention([n], [c], 8, 2, dim, 16, dtype, seed=9, edit=edit)
    mask = tree_batch([n], 9)
    with np.errstate(all="ignore"):
        g = got.double().cpu().numpy()
        clean = [t for t in range(n) if not (mask[t] >> 2) & 1 and not (mask[t] >> (n - 3)) & 1]
        dirty = [t for t in range(n) if t not in clean]
        assert clean and dirty
        bound = attention_bound(want[clean], size[clean], dtype, c + n, 8.0)
        assert (np.abs(g[clean] - want[clean]) <= bound).all()
        if where == "v":
            # the spoilt elements as binary64 has them, the others intact
            rest = [d for d in range(dim) if not 3 <= d < 7]
            b = attention_bound(want[dirty], size[dirty], dtype, c + n, 8.0)
            assert (np.abs(g[dirty] - want[dirty]) <= b)[:, :, rest].all()
            a, w = g[dirty][:, :, 3:7], want[dirty][:, :, 3:7]
            assert (np.isnan(a) == np.isnan(w)).all() and (a[np.isinf(w)] == w[np.isinf(w)]).all()
        elif where == "k" and math.isnan(bad):
            assert np.isnan(g[dirty]).all()


def test_attention_bad_values_in_the_context_reach_every_row():
    def edit(cache, table, mask):
        cache.v[int(table[0, 0]), 5, 1, 7] = float("inf")
    got, want, _, _ = run_attention([6], [200], 8, 2, 128, 16, torch.float16, seed=2, edit=edit)
    g = got.double().cpu().numpy()
    assert (g[:, 4:, 7] == np.inf).all() and np.isfinite(g[:, :4]).all() and np.isfinite(g[:, 4:, 8:]).all()


def test_attention_pages_outside_the_cache_are_not_seen():
    def edit(cache, table, mask):
        table[0, 2] = -1
        table[0, 4] = cache.k.shape[0]
        table[1, 0] = -7
    got, want, size, _ = run_attention([5, 3], [110, 20], 8, 2, 128, 16, torch.float16, seed=3, edit=edit)
    compare_attention(got, want, size, torch.float16, 120, 8)


@pytest.mark.parametrize("scale", [0.0, -0.2, 1.0, 30.0])
def test_attention_scales(scale):
    """No scale, a negative one, and one that leaves a single weight."""
    got, want, size, _ = run_attention([9], [150], 4, 1, 64, 16, torch.float16, seed=4, scale=scale)
    g = got.double().cpu().numpy()
    # the exponent's own error: 64 products and sums in binary32 of scores up to |scale| * 64 * 16
    slack = min(1.0, abs(scale) * 64 * 16 * 2.0 ** -22)
    bound = attention_bound(want, size, torch.float16, 160, 8.0) + slack * size
    assert (np.abs(g - want) <= bound).all()


def test_attention_rising_scores():
    """Scores that grow along the context, so that the running maximum moves
    in every tile, and then fall."""
    def edit(cache, table, mask):
        P = cache.k.shape[1]
        for p in range(300):
            cache.k[int(table[0, p // P]), p % P] *= 0.02 * (p if p < 200 else 300 - p)
    got, want, size, _ = run_attention([4], [296], 4, 1, 128, 16, torch.bfloat16, seed=6, edit=edit, scale=0.5)
    g = got.double().cpu().numpy()
    bound = attention_bound(want, size, torch.bfloat16, 300, 8.0) + 2.0 ** -9 * size
    assert (np.abs(g - want) <= bound).all()


def test_attention_query_view():
    got, want, size, _ = run_attention([6], [90], 8, 2, 72, 16, torch.float16, seed=8, q_view=True)
    compare_attention(got, want, size, torch.float16, 100, 6)


def test_attention_cuts_what_max_new_and_the_table_leave_out():
    """More new tokens than max_new: the rest is neither seen nor written; a
    context longer than the table ends with it."""
    gen = torch.Generator(device=DEV).manual_seed(1)
    cache = make_cache(6, 16, 2, 64, torch.float16, "token", gen=gen)
    table = torch.arange(6, dtype=torch.int32, device=DEV).view(2, 3)
    q = torch.randn(12, 4, 64, generator=gen, device=DEV).half()
    mask = tree_batch([8, 4], 1, "chain")
    out = torch.full((12, 4, 64), 5.0, dtype=torch.float16, device=DEV)
    got = sb.tree_attention(q, cache, table, i32([20, 1000]), i32([0, 8, 12]), torch.tensor(mask, device=DEV), 5, out=out)
    assert bool((got[5:8] == 5).all())
    # request 1: its 48 cached tokens fill the table, its new ones have no room
    assert bool((got[8:] == 5).all())
    want, size = attention_reference(q[:8], cache, table[:1], [20], [0, 8], mask[:8], 5, 0.125)
    err = np.abs(got[:5].double().cpu().numpy() - want[:5])
    assert (err <= attention_bound(want[:5], size[:5], torch.float16, 30, 8.0)).all()


def test_attention_offsets_past_32_bits():
    """Pages whose element offset passes 2^32 (8 GiB of keys and of values)."""
    P, KH, D = 64, 8, 128
    pages = (1 << 32) // (P * KH * D) + 9
    gen = torch.Generator(device=DEV).manual_seed(3)
    k, v = (torch.empty(pages, P, KH, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    use = [pages - 1, 2, pages - 5, (pages - 9) // 2 + 1]
    for p in use:
        k[p].normal_(generator=gen)
        v[p].normal_(generator=gen)
    cache = sb.KVCache(k, v)
    q = torch.randn(3, 16, D, generator=gen, device=DEV).bfloat16()
    mask = tree_batch([3], 3)
    new_k, new_v = (torch.randn(3, KH, D, generator=gen, device=DEV).bfloat16() for _ in range(2))
    ctx = 3 * P + 20
    slots = torch.tensor([use[3] * P + 20 + j for j in range(3)], device=DEV)
    sb.cache_write(cache, new_k, new_v, slots)
    assert torch.equal(k[use[3], 20:23], new_k) and torch.equal(v[use[3], 20:23], new_v)
    got = sb.tree_attention(q, cache, i32([use]), i32([ctx]), i32([0, 3]), torch.tensor(mask, device=DEV), 3)
    want, size = attention_reference(q, cache, i32([use]), [ctx], [0, 3], mask, 3, D ** -0.5)
    assert (np.abs(got.double().cpu().numpy() - want) <= attention_bound(want, size, torch.bfloat16, ctx, 8.0)).all()


def test_attention_repeats_its_bits():
    a = [run_attention([8, 5], [2000, 777], 32, 8, 128, 16, torch.float16, seed=1)[0] for _ in range(3)]
    assert torch.equal(a[0], a[1]) and torch.equal(a[0], a[2])


MANY = [
    # news, contexts, heads, kv heads, dim, dtype: items short and long, two units of work and more a workgroup
    ([1, 1, 0, 1, 2] * 60, [(37 * r) % 311 for r in range(300)], 8, 8, 64, torch.bfloat16),
    ([1, 3, 1, 0] * 33, [(53 * r) % 509 for r in range(132)], 16, 8, 128, torch.float16),
    ([9, 1, 16, 0, 2, 12] * 5, [900, 3, 0, 700, 1700, 64] * 5, 16, 8, 128, torch.bfloat16),
    ([33, 3, 17, 40] * 6, [2500, 10, 40, 1300] * 6, 16, 8, 80, torch.float16),
    ([33, 64, 3, 33] * 6, [2450, 0, 140, 1400] * 6, 16, 8, 64, torch.bfloat16),
]


@pytest.mark.parametrize("case", range(len(MANY)))
def test_attention_many_items(case):
    news, ctx, H, KH, D, dtype = MANY[case]
    got, want, size, _ = run_attention(news, ctx, H, KH, D, 16, dtype, seed=case, extra=1)
    compare_attention(got, want, size, dtype, max(ctx) + max(news), sum(news))


# ---------------------------------------------------------------------------
# the norms
# ---------------------------------------------------------------------------

def norm_reference(x, y, post, gate, scale, pre, eps):
    d = [None if t is None else t.double() for t in (x, y, post, gate, pre)]
    x, y, post, gate, pre = d
    size = x.abs()
    if y is not None:
        if post is not None:
            y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + eps) * post
        if gate is not None:
            y = y * gate
        x = x + scale * y
        size = size + (scale * y).abs()
    h = None
    if pre is not None:
        inv = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
        h = (x * inv * pre, size * inv * pre.abs())
    return x, size, h


WIDTHS = [1, 7, 64, 128, 1000, 1001, 2048, 4096, 5003, 8192, 12288, 16384, 32761, 32768]


@pytest.mark.parametrize("H", WIDTHS)
@pytest.mark.parametrize("dtype,xt", [(torch.float16, torch.float16), (torch.float16, torch.float32),
                                      (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32)])
@pytest.mark.parametrize("parts", ["pre", "y", "post+pre", "post+token+pre", "channel+pre", "post"])
def test_norm(H, dtype, xt, parts):
    gen = torch.Generator(device=DEV).manual_seed(H)
    T = 5 if H < 10000 else 2

    def rand(*shape, dt=dtype):
        return torch.randn(*shape, generator=gen, device=DEV).to(dt)
    x = 3 * rand(T, H, dt=xt)
    y = None if parts == "pre" else rand(T, H)
    post = rand(H) if "post" in parts else None
    gate = rand(T, H) if "token" in parts else rand(H) if "channel" in parts else None
    pre = rand(H) if "pre" in parts else None
    xo, h = sb.residual_norm(x, y, post_weight=post, gate=gate, scale=-0.6, pre_weight=pre, eps=1e-5)
    want, size, wh = norm_reference(x, y, post, gate, -0.6, pre, 1e-5)
    # a sum of up to 32768 squares, a root and a handful of products in binary32
    f32 = 2.0 ** -18
    assert xo.dtype == xt
    assert bool(((xo.double() - want).abs() <= HALF[xt] * want.abs() * 1.01 + f32 * size + 1e-7).all())
    if pre is None:
        assert h is None
    else:
        assert h.dtype == dtype
        assert bool(((h.double() - wh[0]).abs() <= HALF[dtype] * wh[0].abs() * 1.01 + f32 * wh[1] + 1e-7).all())


def test_norm_in_place_and_strides():
    gen = torch.Generator(device=DEV).manual_seed(1)
    for H in (4096, 1000, 1001):
        wide = torch.randn(6, 3 * H + 9, generator=gen, device=DEV).half()
        x, y, g = wide[:, 1:H + 1], wide[:, H + 2:2 * H + 2], wide[:, 2 * H + 5:3 * H + 5]
        before, untouched = x.clone(), wide[:, H + 1:].clone()
        w = torch.randn(H, generator=gen, device=DEV).half()
        h = torch.full((6, H + 8), 9.0, dtype=torch.float16, device=DEV)
        xo, hh = sb.residual_norm(x, y, post_weight=w, gate=g, scale=0.5, pre_weight=w, x_out=x, h_out=h[:, :H])
        assert xo is x
        want, size, wh = norm_reference(before, y, w, g, 0.5, w, 1e-5)
        assert bool(((x.double() - want).abs() <= 2.0 ** -11 * want.abs() * 1.01 + 2.0 ** -18 * size + 1e-7).all())
        assert bool(((hh.double() - wh[0]).abs() <= 2.0 ** -11 * wh[0].abs() * 1.01 + 2.0 ** -18 * wh[1] + 1e-7).all())
        assert torch.equal(wide[:, H + 1:], untouched) and bool((h[:, H:] == 9).all())


def test_norm_zeros_large_and_bad_values():
    """A row of zeros (only eps under the root), rows near the largest
    binary16, and NaN or infinities kept to their own row."""
    H = 4096
    x = torch.zeros(5, H, dtype=torch.float32, device=DEV)
    y = torch.zeros(5, H, dtype=torch.float16, device=DEV)
    w = torch.ones(H, dtype=torch.float16, device=DEV)
    x[1], y[1] = 60000.0, 60000.0
    y[2, 5] = float("nan")
    x[3, 7] = float("inf")
    x[4] = 1.0
    xo, h = sb.residual_norm(x, y, post_weight=w, pre_weight=w)
    assert bool((xo[0] == 0).all()) and bool((h[0] == 0).all())
    assert bool((h[1] == 1).all()) and abs(float(xo[1, 0]) - 60001) < 0.02
    assert bool(torch.isnan(h[2]).all()) and bool(torch.isnan(h[3]).any()) and bool((h[4] == 1).all())


def test_norm_many_tokens():
    gen = torch.Generator(device=DEV).manual_seed(2)
    x = torch.randn(3000, 512, generator=gen, device=DEV).bfloat16()
    y = torch.randn(3000, 512, generator=gen, device=DEV).bfloat16()
    w = torch.randn(512, generator=gen, device=DEV).bfloat16()
    xo, h = sb.residual_norm(x, y, post_weight=w, pre_weight=w)
    want, size, wh = norm_reference(x, y, w, None, 1.0, w, 1e-5)
    assert bool(((xo.double() - want).abs() <= 2.0 ** -8 * want.abs() * 1.01 + 2.0 ** -18 * size).all())
    assert bool(((h.double() - wh[0]).abs() <= 2.0 ** -8 * wh[0].abs() * 1.01 + 2.0 ** -18 * wh[1]).all())


# ---------------------------------------------------------------------------
# logits
# ---------------------------------------------------------------------------

def logits_reference(c):
    """Row by row in binary64; and the sum of the terms' magnitudes."""
    l0 = c["logits"].double().cpu().numpy()
    T, V = l0.shape
    out, size = l0.copy(), np.abs(l0)
    get = lambda n: None if c.get(n) is None else c[n].cpu().numpy()  # noqa: E731
    for t in range(T):
        r = int(get("token_request")[t]) if c.get("token_request") is not None else t
        if not 0 <= r < c["R"]:
            continue
        count, known = np.zeros(V), np.zeros(V, dtype=bool)
        if c.get("history") is not None:
            h0, h1 = get("history_start")[r:r + 2]
            prompt = get("prompt_lens")[r] if c.get("prompt_lens") is not None else 0
            for i in range(h0, h1):
                v = get("history")[i]
                if 0 <= v < V:
                    known[v] = True
                    count[v] += i - h0 >= prompt
        if c.get("draft_tokens") is not None:
            for j in range(64):
                if (int(get("tree_mask")[t]) >> j) & 1:
                    v = get("draft_tokens")[get("query_start")[r] + j]
                    if 0 <= v < V:
                        known[v] = True
                        count[v] += 1
        rep, freq, pres, temp = (float(get(n)[r]) if c.get(n) is not None else d for n, d in
                                 (("repetition", 1.0), ("frequency", 0.0), ("presence", 0.0), ("temperature", 1.0)))
        l = out[t]
        l[known] = np.where(l[known] > 0, l[known] / rep, l[known] * rep)
        l -= freq * count + pres * (count > 0)
        size[t] = np.abs(l0[t]) * max(rep, 1 / rep) + abs(freq) * count + abs(pres)
        if c.get("bias_tokens") is not None:
            b0, b1 = get("bias_start")[r:r + 2]
            last = {int(get("bias_tokens")[i]): float(get("bias_values")[i]) for i in range(b0, b1)}
            for v, b in last.items():
                if 0 <= v < V:
                    l[v] += b
                    size[t, v] += abs(b)
        if temp > 0:
            l /= temp
            size[t] /= temp
        if c.get("grammar") is not None:
            g = int(get("grammar_rows")[t]) if c.get("grammar_rows") is not None else t
            if 0 <= g < c["grammar"].shape[0]:
                words = get("grammar")[g].view(np.uint32)
                allowed = (words[np.arange(V) // 32] >> (np.arange(V) % 32).astype(np.uint32)) & 1
                l[allowed == 0] = -np.inf
    return out, size


def logits_case(R, N, V, dtype, history, seed, parts):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    rng = np.random.default_rng(seed)
    T = R * N
    c = dict(R=R, logits=(4 * torch.randn(T, V, generator=gen, device=DEV)).to(dtype))
    if "history" in parts:
        lens = rng.integers(0, history + 1, R)
        c["history"] = i32(rng.integers(-2, min(V, 40) + 2, int(lens.sum())).tolist())
        c["history_start"] = i32([0] + np.cumsum(lens).tolist())
        c["prompt_lens"] = i32((lens // 2).tolist())
    if "params" in parts:
        for n, lo, hi in (("repetition", 0.8, 1.5), ("frequency", -0.5, 0.5), ("presence", -0.5, 0.5), ("temperature", -0.2, 2.0)):
            c[n] = torch.tensor(rng.uniform(lo, hi, R), dtype=torch.float32, device=DEV)
    if "bias" in parts:
        lens = rng.integers(0, 30, R)
        c["bias_tokens"] = i32(rng.integers(-1, V + 1, int(lens.sum())).tolist())
        c["bias_values"] = torch.tensor(rng.normal(0, 4, int(lens.sum())), dtype=torch.float32, device=DEV)
        c["bias_start"] = i32([0] + np.cumsum(lens).tolist())
    if "grammar" in parts:
        M = max(1, T // 2)
        c["grammar"] = torch.from_numpy(rng.integers(0, 2 ** 32, (M, (V + 31) // 32), dtype=np.uint32).view(np.int32)).to(DEV)
        c["grammar"][0] = 0  # allows nothing
        c["grammar_rows"] = i32([(i % (M + 2)) - 1 for i in range(T)])
    if "tree" in parts:
        c["token_request"] = i32([t // N for t in range(T)])
        c["query_start"] = i32([N * r for r in range(R + 1)])
        c["draft_tokens"] = i32(rng.integers(-1, V + 1, T).tolist())
        c["tree_mask"] = torch.tensor(tree_batch([N] * R, seed), device=DEV)
    return c


def check_logits(c, out_dtype=None, **more):
    got = sb.adjust_logits(**{k: v for k, v in c.items() if k != "R"}, n_requests=c["R"], out_dtype=out_dtype, **more)
    return got


def compare_logits(got, want, size, dtype):
    g = got.double().cpu().numpy()
    hidden = np.isneginf(want)
    assert (np.isneginf(g) == hidden).all()
    err = np.abs(np.where(hidden, 0, g) - np.where(hidden, 0, want))
    # binary32: up to six roundings of terms of this size; then the output's own
    bound = 2.0 ** -21 * size + 1.01 * HALF[dtype] * np.where(hidden, 0, np.abs(want)) + 1e-7
    assert (err <= bound).all(), (err / bound).max()


@pytest.mark.parametrize("R,N,V", [(1, 1, 1), (1, 1, 7), (2, 3, 33), (3, 2, 1000), (1, 1, 50001), (2, 8, 4096),
                                   (1, 64, 4097), (5, 1, 12289)])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("parts", ["history+params+bias+grammar+tree", "params", "history+params", "bias", "grammar",
                                   "params+tree"])
def test_logits(R, N, V, dtype, parts):
    if N > 1 and "tree" not in parts:
        R, N = R * N, 1
    c = logits_case(R, N, V, dtype, 300, V + R, parts)
    want, size = logits_reference(c)
    compare_logits(check_logits(c, torch.float32), want, size, torch.float32)
    compare_logits(check_logits(c), want, size, dtype)


def test_logits_in_place_and_strides():
    c = logits_case(3, 4, 1001, torch.float16, 50, 1, "history+params+bias+grammar+tree")
    want, size = logits_reference(c)
    wide = torch.full((12, 1024), 3.0, dtype=torch.float16, device=DEV)
    wide[:, :1001] = c["logits"]
    c["logits"] = wide[:, :1001]
    got = check_logits(c, out=c["logits"])
    assert got.data_ptr() == wide.data_ptr()
    compare_logits(got, want, size, torch.float16)
    assert bool((wide[:, 1001:] == 3).all())


def test_logits_rows_of_no_request_and_special_values():
    c = logits_case(2, 3, 500, torch.float32, 60, 2, "history+params+bias+grammar+tree")
    c["token_request"][1] = -1
    c["token_request"][4] = 2
    c["logits"][0, 3] = float("nan")
    c["logits"][0, 4:8] = float("-inf")
    c["logits"][3, 4] = float("inf")
    got = check_logits(c)
    want, _ = logits_reference(c)
    g = got.double().cpu().numpy()
    assert torch.equal(got[1], c["logits"][1]) and torch.equal(got[4], c["logits"][4])
    assert (np.isnan(g) == np.isnan(want)).all() and (np.isposinf(g) == np.isposinf(want)).all()
    assert (np.isneginf(g) == np.isneginf(want)).all()


def test_logits_long_history():
    """A token more often than 16 bits count, and ids across all tiles."""
    V, n = 30000, 200000
    rng = np.random.default_rng(3)
    h = np.where(rng.random(n) < 0.5, 777, rng.integers(0, V, n))
    c = dict(R=1, logits=torch.zeros(1, V, device=DEV), history=i32(h.tolist()), history_start=i32([0, n]),
             prompt_lens=i32([1000]), frequency=torch.tensor([0.25], device=DEV))
    got = check_logits(c)
    want = -0.25 * np.bincount(h[1000:], minlength=V)
    assert (got[0].cpu().numpy() == want).all()


@pytest.mark.parametrize("V", [65536, 65543])
@pytest.mark.parametrize("parts", ["history+params+bias+grammar+tree", "params"])
def test_logits_many_tiles(V, parts):
    c = logits_case(20, 5, V, torch.float16, 300, V, parts) if "tree" in parts else logits_case(100, 1, V, torch.float16, 300, V, parts)
    want, size = logits_reference(c)
    compare_logits(check_logits(c, torch.float32), want, size, torch.float32)
    in_place = c["logits"].clone()
    compare_logits(check_logits(dict(c, logits=in_place), out=in_place), want, size, torch.float16)


# ---------------------------------------------------------------------------
# streams and graphs
# ---------------------------------------------------------------------------

def step_inputs(seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    R, N, P, H, KH, D, V, W = 3, 4, 16, 8, 2, 128, 1000, 512
    T = R * N
    s = dict(ctx=i32([40, 7, 130]), new=i32([N] * R), free=torch.randperm(64, generator=gen, device=DEV).to(torch.int32)[:20] + 16,
             table=torch.arange(R * 10, device=DEV, dtype=torch.int32).view(R, 10) % 16,
             parents=i32([-1, 0, 0, 1] * R), cache=make_cache(80, P, KH, D, torch.float16, "token", gen=gen),
             k=torch.randn(T, KH, D, generator=gen, device=DEV).half(), v=torch.randn(T, KH, D, generator=gen, device=DEV).half(),
             q=torch.randn(T, H, D, generator=gen, device=DEV).half(), x=torch.randn(T, W, generator=gen, device=DEV),
             y=torch.randn(T, W, generator=gen, device=DEV).half(), w=torch.randn(W, generator=gen, device=DEV).half(),
             logits=torch.randn(T, V, generator=gen, device=DEV).half(), draft=torch.randint(0, V, (T,), generator=gen, device=DEV, dtype=torch.int32),
             freq=torch.full((R,), 0.5, device=DEV), P=P, T=T, N=N)
    return s


def step_run(s, stream=None):
    p = sb.batch_plan(s["ctx"], s["new"], s["free"], s["table"], s["P"], s["T"], parents=s["parents"], stream=stream)
    sb.cache_write(s["cache"], s["k"], s["v"], p.slots, stream=stream)
    o = sb.tree_attention(s["q"], s["cache"], s["table"], s["ctx"], p.query_start, p.tree_mask, s["N"], stream=stream)
    x, h = sb.residual_norm(s["x"], s["y"], post_weight=s["w"], pre_weight=s["w"], stream=stream)
    l = sb.adjust_logits(s["logits"], frequency=s["freq"], token_request=p.token_request, query_start=p.query_start,
                         tree_mask=p.tree_mask, draft_tokens=s["draft"], stream=stream)
    return [p.slots, p.positions, p.tree_mask, s["cache"].k, s["cache"].v, o, x, h, l]


def test_step_on_another_stream():
    want = [t.clone() for t in step_run(step_inputs(1))]
    s = step_inputs(1)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = step_run(s, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_step_in_a_graph():
    """Captured once, replayed with new inputs between eager work."""
    s = step_inputs(1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step_run(s)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step_run(s)
    for seed in (2, 3, 4):
        fresh = step_inputs(seed)
        for name, t in fresh.items():
            if isinstance(t, torch.Tensor):
                s[name].copy_(t)
        s["cache"].k.copy_(fresh["cache"].k)
        s["cache"].v.copy_(fresh["cache"].v)
        g.replay()
        want = step_run(fresh)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), seed


@pytest.mark.parametrize("T", [0])
def test_step_of_no_tokens(T):
    s = step_inputs(1)
    z = i32([0, 0, 0])
    p = sb.batch_plan(s["ctx"], z, s["free"], s["table"], s["P"], 0)
    assert p.query_start.tolist() == [0, 0, 0, 0] and p.used.tolist() == [0, 0]
    o = sb.tree_attention(s["q"][:0], s["cache"], s["table"], s["ctx"], p.query_start, p.tree_mask, 1)
    assert tuple(o.shape) == (0, 8, 128)
    x, h = sb.residual_norm(s["x"][:0], s["y"][:0], pre_weight=s["w"])
    assert x.shape == (0, 512) and h.shape == (0, 512)
    assert sb.adjust_logits(s["logits"][:0], n_requests=3).shape == (0, 1000)


# ---------------------------------------------------------------------------
# refusals of the tensor helpers
# ---------------------------------------------------------------------------

def test_helpers_refuse_what_does_not_fit():
    s = step_inputs(1)
    T = s["T"]
    p = sb.batch_plan(s["ctx"], s["new"], s["free"], s["table"], s["P"], T, parents=s["parents"])

    def attend(q=s["q"], cache=s["cache"], table=s["table"], ctx=s["ctx"], start=p.query_start, mask=p.tree_mask, n=s["N"], **more):
        return sb.tree_attention(q, cache, table, ctx, start, mask, n, **more)
    bad = [
        lambda: sb.batch_plan(s["ctx"].long(), s["new"], s["free"], s["table"], s["P"], T),
        lambda: sb.batch_plan(s["ctx"], s["new"][:2], s["free"], s["table"], s["P"], T),
        lambda: sb.batch_plan(s["ctx"], s["new"], s["free"], s["table"][:2], s["P"], T),
        lambda: sb.batch_plan(s["ctx"], s["new"], s["free"], s["table"].t().contiguous().t(), s["P"], T),
        lambda: sb.batch_plan(s["ctx"], s["new"], s["free"], s["table"], s["P"], T, parents=s["parents"][:-1]),
        lambda: sb.cache_write(s["cache"], s["k"].bfloat16(), s["v"], p.slots),
        lambda: sb.cache_write(s["cache"], s["k"], s["v"][:-1], p.slots),
        lambda: sb.cache_write(s["cache"], s["k"][..., :64], s["v"], p.slots),
        lambda: sb.cache_write(s["cache"], s["k"], s["v"], p.slots.int()),
        lambda: attend(q=s["q"].bfloat16()),
        lambda: attend(q=s["q"].transpose(0, 2).contiguous().transpose(0, 2)),
        lambda: attend(ctx=s["ctx"][:2]),
        lambda: attend(start=p.query_start[:-1]),
        lambda: attend(mask=p.tree_mask[:-1]),
        lambda: attend(out=torch.empty(T, 8, 128, device=DEV)),
        lambda: attend(table=s["table"].cpu()),
        lambda: sb.residual_norm(s["x"], s["y"].float()[:, :5]),
        lambda: sb.residual_norm(s["x"], s["y"], post_weight=s["w"][:-1]),
        lambda: sb.residual_norm(s["x"], post_weight=s["w"]),
        lambda: sb.residual_norm(s["x"]),
        lambda: sb.residual_norm(s["x"], s["y"], h_out=s["y"]),
        lambda: sb.residual_norm(s["x"], s["y"], x_out=s["y"]),
        lambda: sb.adjust_logits(s["logits"], frequency=s["freq"].double()),
        lambda: sb.adjust_logits(s["logits"], history=s["draft"]),
        lambda: sb.adjust_logits(s["logits"], bias_tokens=s["draft"]),
        lambda: sb.adjust_logits(s["logits"], grammar=torch.zeros(2, 31, dtype=torch.int32, device=DEV)),
        lambda: sb.adjust_logits(s["logits"], out=s["logits"], out_dtype=torch.float32),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(AssertionError):
            call()
            print("accepted:", i)
    refused = [
        lambda: sb.batch_plan(s["ctx"], s["new"], s["free"], s["table"], 24, T),
        lambda: attend(n=65), lambda: attend(n=0), lambda: attend(scale=float("nan")),
        lambda: attend(workspace=torch.empty(64, dtype=torch.uint8, device=DEV)),
        lambda: sb.residual_norm(s["x"], s["y"], eps=-1.0),
        lambda: sb.adjust_logits(s["logits"], draft_tokens=s["draft"]),
        lambda: sb.adjust_logits(s["logits"].float(), out=torch.empty_like(s["logits"])),
    ]
    for call in refused:
        with pytest.raises(sb.SBVRError):
            call()


def test_helpers_fill_what_they_are_given():
    s = step_inputs(4)
    p = sb.batch_plan(s["ctx"], s["new"], s["free"], s["table"].clone(), s["P"], s["T"], parents=s["parents"])
    q = sb.BatchPlan(*[torch.full_like(getattr(p, n), -9) for n in sb.BatchPlan.__slots__])
    assert sb.batch_plan(s["ctx"], s["new"], s["free"], s["table"].clone(), s["P"], s["T"], parents=s["parents"], out=q) is q
    assert all(torch.equal(getattr(p, n), getattr(q, n)) for n in sb.BatchPlan.__slots__)
    need = sb.sbvr_tree_attention_workspace_bytes(3, s["N"], 8, 2, 128)
    ws = torch.empty(need + 16, dtype=torch.uint8, device=DEV)
    out = torch.empty_like(s["q"])
    sb.cache_write(s["cache"], s["k"], s["v"], p.slots)
    got = sb.tree_attention(s["q"], s["cache"], s["table"], s["ctx"], p.query_start, p.tree_mask, s["N"], out=out, workspace=ws)
    assert got.data_ptr() == out.data_ptr()
    assert torch.equal(out, sb.tree_attention(s["q"], s["cache"], s["table"], s["ctx"], p.query_start, p.tree_mask, s["N"]))


# ---------------------------------------------------------------------------
# attention: many small weights beside a large one
# ---------------------------------------------------------------------------

SHAPES = [  # new tokens, heads, kv heads: up to 16, 64 and 128 rows a key/value head
    (1, 8, 8), (8, 16, 4), (16, 16, 2)]


@pytest.mark.parametrize("new,heads,kv_heads", SHAPES)
@pytest.mark.parametrize("dim", [64, 128])
def test_attention_many_small_weights(new, heads, kv_heads, dim):
    """Every 32nd position has the weight 1, all others e^-17.5 (2^-25.2, less
    than half of the smallest binary16 number) and values 60000 times as large,
    so that together they are a few percent of the result."""
    N, P, gap, large = 4096, 16, 17.5, 60000.0
    pages = N // P + 5
    cache = make_cache(pages, P, kv_heads, dim, torch.float16, "token", fill=0.0)
    k, v = cache.k.view(-1, kv_heads, dim), cache.v.view(-1, kv_heads, dim)
    v.fill_(large)
    k[:N:32, :, 0], v[:N:32] = gap, 1.0
    table = torch.arange(pages, device=DEV, dtype=torch.int32).view(1, -1)
    q = torch.zeros(new, heads, dim, dtype=torch.float16, device=DEV)
    q[..., 0] = 1.0
    mask = tree_batch([new], 1, "chain")
    got = sb.tree_attention(q, cache, table, i32([N]), i32([0, new]), torch.tensor(mask, device=DEV), new, scale=1.0)
    want, size = attention_reference(q, cache, table, [N], [0, new], mask, new, 1.0)
    # A weight is rounded to a multiple of 2^-24 at the most, where the largest of its tile stands for 2^7 or
    # more: 2^-32 of it, times 31 of 32 positions and their values.  Then the binary32 exponentials and the
    # rounding of the result (attention_bound's terms without its allowance for vanished weights).
    bound = 31 * 2.0 ** -32 * large + 1.01 * 2.0 ** -11 * (size + np.abs(want)) + 2.0 ** -15 * size
    assert want.min() > 1.04
    err = np.abs(got.double().cpu().numpy() - want)
    assert (err <= bound).all(), (err / bound).max()


# ---------------------------------------------------------------------------
# attention: infinite keys, every head size
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("new,heads,kv_heads", SHAPES)
@pytest.mark.parametrize("dim", [8, 32, 40, 64, 72, 80, 96, 104, 128])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("element", [0, 7])
def test_attention_scores_of_minus_infinity(new, heads, kv_heads, dim, dtype, element):
    """A key that gives every row the score -infinity has the weight 0, in the
    context and among the step's own tokens, whatever the head's size."""
    gen = torch.Generator(device=DEV).manual_seed(dim + element)
    N, P = 150, 16
    pages = (N + new + P - 1) // P
    cache = make_cache(pages, P, kv_heads, dim, dtype, "token", gen=gen)
    flat = cache.k.view(-1, kv_heads, dim)
    for p in (3, 40, 149, N):  # (the first own token: the others see themselves)
        flat[p, :, element] = float("-inf")
    table = torch.arange(pages, device=DEV, dtype=torch.int32).view(1, -1)
    q = torch.randn(new, heads, dim, generator=gen, device=DEV).to(dtype)
    q[..., element] = q[..., element].abs() + 0.25
    mask = tree_batch([new], 1, "chain")
    got = sb.tree_attention(q, cache, table, i32([N]), i32([0, new]), torch.tensor(mask, device=DEV), new)
    want, size = attention_reference(q, cache, table, [N], [0, new], mask, new, dim ** -0.5)
    assert np.isfinite(want).all()
    compare_attention(got, want, size, dtype, N + new, new)


def test_helpers_refuse_rows_that_overlap():
    """An expanded page table or grammar, and rows closer than they are wide:
    the rows past the first would be looked for behind it."""
    s = step_inputs(1)
    p = sb.batch_plan(s["ctx"], s["new"], s["free"], s["table"], s["P"], s["T"], parents=s["parents"])
    table, words = s["table"][0].clone(), torch.zeros(32, dtype=torch.int32, device=DEV)
    for rows in (lambda t, n: t.expand(n, -1), lambda t, n: t.as_strided((n, t.numel() - n + 1), (1, 1))):
        with pytest.raises(sb.SBVRError):
            sb.batch_plan(s["ctx"], s["new"], s["free"], rows(table, 3), s["P"], s["T"])
        with pytest.raises(sb.SBVRError):
            sb.tree_attention(s["q"], s["cache"], rows(table, 3), s["ctx"], p.query_start, p.tree_mask, s["N"])
        with pytest.raises(sb.SBVRError):
            grammar = rows(words, s["T"])
            V = 32 * grammar.shape[1] - 24
            sb.adjust_logits(torch.zeros(s["T"], V, device=DEV), grammar=grammar)
    # one row for all is a row number for all
    l = torch.zeros(s["T"], 1000, device=DEV)
    got = sb.adjust_logits(l, grammar=words.view(1, 32), grammar_rows=torch.zeros(s["T"], dtype=torch.int32, device=DEV))
    assert bool(torch.isneginf(got).all())


def test_memory_of_a_call_belongs_to_its_stream():
    """What a call on a given stream allocates is no block that the current
    stream has just freed (its kernels may still use it), and is not handed to the
    current stream when it is freed."""
    s = step_inputs(1)
    side = torch.cuda.Stream()
    kept = step_run(s)  # (the current stream's own results, of the same sizes)
    sizes = sorted({t.numel() * t.element_size() for t in kept} | {
        sb.sbvr_tree_attention_workspace_bytes(3, s["N"], 8, 2, 128), 4 * 4, 2 * 4})
    freed = [torch.empty(n, dtype=torch.uint8, device=DEV) for n in sizes for _ in range(3)]
    blocks = {t.data_ptr() for t in freed}
    del freed
    torch.cuda.synchronize()
    before = torch.cuda.current_stream(), torch.cuda.current_device()
    p = sb.batch_plan(s["ctx"], s["new"], s["free"], s["table"], s["P"], s["T"], parents=s["parents"], stream=side)
    got = [getattr(p, n) for n in sb.BatchPlan.__slots__]
    got += step_run(s, stream=side)
    assert (torch.cuda.current_stream(), torch.cuda.current_device()) == before
    own = [t for t in got if all(t is not u for u in (s["cache"].k, s["cache"].v))]
    side.synchronize()
    assert not blocks & {t.data_ptr() for t in own}
    mine = {t.data_ptr() for t in own}
    del got, own, p
    again = [torch.empty(n, dtype=torch.uint8, device=DEV) for n in sizes for _ in range(3)]
    assert not mine & {t.data_ptr() for t in again}


# ---------------------------------------------------------------------------
# attention: rows of no request, and requests that do not fit
# ---------------------------------------------------------------------------

def poison(shape, dtype):
    """Leaves memory of this size full of 7s to the next allocation."""
    t = torch.full(shape, 7.0, dtype=dtype, device=DEV)
    del t


@pytest.mark.parametrize("new,heads,kv_heads", SHAPES)
@pytest.mark.parametrize("room", [0, 1, 70])
@pytest.mark.parametrize("requests", [1, 3, 200])
def test_attention_of_a_padded_plan(new, heads, kv_heads, room, requests):
    """Rows past the plan's last token are 0, the others what they are without
    them."""
    gen = torch.Generator(device=DEV).manual_seed(requests)
    P, D, R = 16, 64, requests
    news = [new if r % 2 == 0 else new // 2 for r in range(R)]  # (an empty request among them)
    ctx = [(37 * r) % 100 for r in range(R)]
    T, width = sum(news), 8
    cache = make_cache(R * width, P, kv_heads, D, torch.float16, "token", gen=gen)
    table = torch.arange(R * width, dtype=torch.int32, device=DEV).view(R, width)
    q = torch.randn(T + room, heads, D, generator=gen, device=DEV).half()
    start = i32([sum(news[:r]) for r in range(R + 1)])
    mask = torch.tensor(tree_batch(news, 3) + [0] * room, device=DEV)
    given = torch.full((T + room, heads, D), 5.0, dtype=torch.float16, device=DEV)
    sb.tree_attention(q, cache, table, i32(ctx), start, mask, new, out=given)
    poison(given.shape, torch.float16)
    got = sb.tree_attention(q, cache, table, i32(ctx), start, mask, new)
    assert torch.equal(got[:T], given[:T])
    assert bool((got[T:] == 0).all()) and bool((given[T:] == 5).all())


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("long", [9, 65, 300])
def test_attention_of_a_prompt_too_long_for_it(dtype, long):
    """A request of more new tokens than max_new (beyond 64 the plan has no
    masks for it), or than its pages hold, is NaN in every row; the requests beside
    it are not touched."""
    gen = torch.Generator(device=DEV).manual_seed(long)
    P, KH, H, D, most = 16, 2, 8, 128, min(long - 1, 64)
    news, ctx = [3, long, 2, 5], [40, 7, 30, 60]
    T, pages = sum(news), 25
    free = torch.arange(200, dtype=torch.int32, device=DEV)
    table = torch.full((4, pages), -1, dtype=torch.int32, device=DEV)
    table[:, :4] = torch.arange(200, 216, dtype=torch.int32, device=DEV).view(4, 4)
    cache = make_cache(216, P, KH, D, dtype, "token", gen=gen)
    p = sb.batch_plan(i32(ctx), i32(news), free, table, P, T + 4)
    q = torch.randn(T + 4, H, D, generator=gen, device=DEV).to(dtype)
    # request 3's table ends inside its new tokens: 60 cached ones and 4 of 5 fit
    short = table.clone()[:, :4].contiguous() if long < 50 else table
    cut = [1, 3] if long < 50 else [1]
    poison(q.shape, dtype)
    got = sb.tree_attention(q, cache, short, i32(ctx), p.query_start, p.tree_mask, most)
    start = p.query_start.tolist()
    want, size = attention_reference(q, cache, short, [c if r not in cut else 0 for r, c in enumerate(ctx)], start,
                                     [0 if t >= T else m for t, m in enumerate(p.tree_mask.tolist())], 5, D ** -0.5)
    for r in range(4):
        rows = got[start[r]:start[r + 1]].double().cpu().numpy()
        if r in cut:
            assert np.isnan(rows).all()
        else:
            bound = attention_bound(want[start[r]:start[r + 1]], size[start[r]:start[r + 1]], dtype, 80, 8.0)
            assert (np.abs(rows - want[start[r]:start[r + 1]]) <= bound).all()
    assert bool((got[T:] == 0).all())


def test_a_whole_step_of_no_tokens():
    """What an empty plan hands on is taken by every operator of the step."""
    s = step_inputs(1)
    p = sb.batch_plan(s["ctx"], i32([0, 0, 0]), s["free"], s["table"], s["P"], 0)
    before = s["cache"].k.clone()
    sb.cache_write(s["cache"], s["k"][:0], s["v"][:0], p.slots)
    assert torch.equal(s["cache"].k, before)
    assert sb.tree_attention(s["q"][:0], s["cache"], s["table"], s["ctx"], p.query_start, p.tree_mask, s["N"]).shape[0] == 0
    l = s["logits"][:0]
    assert sb.adjust_logits(l).shape == (0, 1000)
    got = sb.adjust_logits(l, frequency=s["freq"], token_request=p.token_request, query_start=p.query_start,
                           tree_mask=p.tree_mask, draft_tokens=s["draft"][:0], history=s["draft"],
                           history_start=i32([0, 4, 8, 12]), bias_tokens=s["draft"][:0], bias_values=s["freq"][:0],
                           bias_start=i32([0, 0, 0, 0]), grammar=torch.empty(0, 32, dtype=torch.int32, device=DEV),
                           grammar_rows=p.token_request, out_dtype=torch.float32)
    assert got.shape == (0, 1000) and got.dtype == torch.float32
