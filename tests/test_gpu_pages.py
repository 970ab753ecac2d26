"""The operators on pages that sequences share against plain implementations."""
import numpy as np
import pytest
import torch

import paper_2509_18172_amd as sb

pytestmark = pytest.mark.gpu

DEV = "cuda"


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def in_use(lens, table, P):
    """Per row the entries in use."""
    return [row[:min(-(-max(c, 0) // P), len(row))] for c, row in zip(lens, table)]


def put(table, stride):
    """A table with rows `stride` apart, and 7777 between them."""
    R, width = len(table), len(table[0])
    full = torch.full((R, stride), 7777, dtype=torch.int32, device=DEV)
    full[:, :width] = i32(table)
    return full, full[:, :width]


# name: (lengths, width of the table, page size, pages of the cache)
SIZES = {
    "one": ([900], 60, 16, 100), "empty": ([0], 4, 16, 7), "none_left": ([64], 4, 16, 4), "one_page": ([3], 1, 16, 1),
    "no_entry": ([0, 0], 3, 32, 1), "some_empty": ([5, 0, 40, 7, 0], 8, 16, 33), "negative": ([-5, 20], 4, 16, 31),
    "full_pages": ([32, 64, 0, 96], 6, 32, 64), "cut": ([1000, 70], 3, 16, 65), "huge_length": ([2 ** 31 - 1, 1], 5, 16, 40),
    "wide": ([700, 16 * 1000, 3], 1025, 16, 3000), "large_pages": ([4096 * 3 + 1, 4095], 5, 4096, 20),
}


def make(name, seed=0, invalid=True):
    lens, width, P, pages = SIZES[name]
    rng = np.random.default_rng(seed)
    table = rng.integers(-2 if invalid else 0, pages + 3 if invalid else pages, (len(lens), width)).tolist()
    return lens, table, P, pages


def usage_reference(lens, table, P, pages):
    refs = [0] * pages
    for row in in_use(lens, table, P):
        for page in row:
            if 0 <= page < pages:
                refs[page] += 1
    free = [p for p in range(pages) if refs[p] == 0]
    return refs, free + [-1] * (pages - len(free)), [len(free), pages - len(free)]


def check_usage(lens, table, P, pages, stride=0):
    full, view = put(table, max(stride, len(table[0])))
    u = sb.page_usage(i32(lens), view, P, pages)
    assert [u.refs.tolist(), u.free_pages.tolist(), u.counts.tolist()] == list(usage_reference(lens, table, P, pages))
    return u


@pytest.mark.parametrize("name", SIZES)
def test_usage(name):
    lens, table, P, pages = make(name)
    check_usage(lens, table, P, pages)
    check_usage(lens, table, P, pages, stride=len(table[0]) + 5)


@pytest.mark.parametrize("pages", [1, 2, 31, 32, 33, 1023, 1024, 1025, 16384, 16385, 32768, 32769, 70000, 300001])
def test_usage_of_many_pages(pages):
    rng = np.random.default_rng(pages)
    R, width = 40, 300
    table = rng.integers(0, pages, (R, width)).tolist()
    check_usage(rng.integers(0, width * 16, R).tolist(), table, 16, pages)


def test_usage_of_most_rows():
    rng = np.random.default_rng(0)
    table = rng.integers(0, 9000, (4096, 70)).tolist()
    check_usage(rng.integers(0, 70 * 16, 4096).tolist(), table, 16, 9000)


@pytest.mark.parametrize("R,width,pages", [(1000, 300, 30000), (130, 513, 12289), (4096, 150, 9000), (2000, 100, 4), (700, 50, 400001)])
def test_usage_of_many_rows_and_pages(R, width, pages):
    """Rows that are split over workgroups, with one owner of pages and several."""
    rng = np.random.default_rng(R)
    table = rng.integers(-1, pages + 1, (R, width)).tolist()
    lens = rng.integers(0, width * 16 + 40, R)
    lens[::3] //= 10
    check_usage(lens.tolist(), table, 16, pages, stride=width + 1)


@pytest.mark.parametrize("pages", [703, 704, 705, 11263, 11264, 11265, 11264 + 704, 11264 + 705, 2 * 11264, 2 * 11264 + 1])
@pytest.mark.parametrize("R,width", [(20, 300), (600, 65)])
def test_usage_at_the_edges_of_owners_and_shares(pages, R, width):
    """A workgroup owns 11264 pages, a wavefront or a later launch's workgroup has 704
    of them; the entries whole and split."""
    rng = np.random.default_rng(pages)
    table = rng.integers(0, pages, (R, width))
    table[0, :4] = [0, pages - 1, pages, -1]
    check_usage(rng.integers(64, width * 16, R).tolist(), table.tolist(), 16, pages)


@pytest.mark.parametrize("R,width,pages", [
    (511, 64, 300), (512, 64, 300), (4095, 64, 5000), (4096, 64, 5000),        # chunks of 64 entries: two and sixteen splits
    (2000, 100, 400001), (4096, 65, 17 * 11264), (600, 64, 129 * 11264)])     # as many as 256 workgroups leave: 7, 15 and 1
def test_usage_at_the_edges_of_splits(R, width, pages):
    rng = np.random.default_rng(R)
    lens = rng.integers(0, width * 16 + 40, R)
    lens[-1] = width * 16
    table = rng.integers(0, pages, (R, width))
    table[-1, -1] = pages - 1
    check_usage(lens.tolist(), table.tolist(), 16, pages)


def test_usage_of_one_page_by_all():
    check_usage([160] * 500, [[5] * 10] * 500, 16, 9)


def test_usage_without_rows():
    u = sb.page_usage(i32([]), torch.empty(0, 4, dtype=torch.int32, device=DEV), 16, 50)
    assert u.refs.tolist() == [0] * 50 and u.free_pages.tolist() == list(range(50)) and u.counts.tolist() == [50, 0]


# ---------------------------------------------------------------------------
# fork
# ---------------------------------------------------------------------------

def fork_reference(lens, table, parents, P, free, taken):
    G, N = len(parents), len(parents[0]) if parents else 0
    per, width = len(lens) // G, len(table[0])
    out, out_lens, copies, used, seen = [], [], [], 0, set()
    for g in range(G):
        for p in parents[g]:
            if not 0 <= p < per:
                out.append([-1] * width)
                out_lens.append(0)
                copies.append((-1, -1, 0))
                continue
            p += g * per
            length = max(lens[p], 0)
            row = in_use([length], [table[p]], P)[0]
            copy, full = (-1, -1, 0), length // P
            if length % P and full < width and p in seen and row[full] >= 0:
                at = max(taken, 0) + used
                page = max(free[at], -1) if at < len(free) else -1
                if page >= 0:
                    copy = (row[full], page, length % P)
                row = row[:full] + [page]
                used += 1
            seen.add(p)
            out.append(row + [-1] * (width - len(row)))
            out_lens.append(length)
            copies.append(copy)
    return out, out_lens, [c[0] for c in copies], [c[1] for c in copies], [c[2] for c in copies], [used]


def check_fork(lens, table, parents, P, free, taken=None, stride=0):
    width = len(table[0])
    full, view = put(table, max(stride, width))
    want = fork_reference(lens, table, parents, P, free, taken or 0)
    f = sb.page_fork(i32(lens), view, i32(parents), P, i32(free), taken=None if taken is None else i32([taken, 99]))
    got = [getattr(f, name).tolist() for name in sb.PageFork.__slots__]
    assert got == list(want)
    # into rows of a wider table, what lies behind stays
    room = torch.full((len(want[0]), width + 3), 555, dtype=torch.int32, device=DEV)
    out = sb.PageFork(room[:, :width], *[torch.empty_like(getattr(f, n)) for n in sb.PageFork.__slots__[1:]])
    assert sb.page_fork(i32(lens), view, i32(parents), P, i32(free), taken=None if taken is None else i32([taken]),
                        out=out) is out
    assert room[:, :width].tolist() == want[0] and bool((room[:, width:] == 555).all())
    return f


FORKS = {
    # lengths, width, page size, parents, free pages, taken
    "one": ([20], 3, 16, [[0]], 4, None), "expand": ([21], 3, 16, [[0, 0, 0, 0]], 4, None),
    "full_page": ([32], 3, 16, [[0, 0, 0]], 4, None), "short": ([5, 5, 5, 5], 2, 16, [[3, 3, 3, 0]], 9, None),
    "groups": ([20, 21, 22, 40, 41, 42], 4, 16, [[1, 1, 0], [2, 2, 2]], 9, 2),
    "shrink": ([20, 21, 22, 40, 41, 42], 4, 16, [[1], [2]], 9, None), "grow": ([20, 33], 4, 16, [[0, 0, 0, 0], [0, 0, 0, 0]], 9, 1),
    "no_parent": ([20, 20], 3, 16, [[-1, 1, 2, 1, 7, -9]], 4, None), "all_gone": ([20, 20], 3, 16, [[-1, -1]], 4, None),
    "no_free": ([20], 3, 16, [[0, 0, 0]], 0, None), "few_free": ([20], 3, 16, [[0, 0, 0, 0]], 2, None),
    "taken_all": ([20], 3, 16, [[0, 0, 0, 0]], 5, 4), "taken_more": ([20], 3, 16, [[0, 0]], 5, 2 ** 31 - 1),
    "taken_negative": ([20], 3, 16, [[0, 0]], 5, -3), "cut": ([1000, 50], 3, 16, [[0, 0, 1, 1]], 5, None),
    "empty_rows": ([0, -4, 16], 3, 16, [[0, 0, 1, 1, 2, 2]], 5, None), "large_page": ([4097, 4095], 2, 4096, [[0, 0, 1, 1]], 5, 1),
    "huge": ([2 ** 31 - 1], 4, 16, [[0, 0]], 3, None),
}


@pytest.mark.parametrize("name", FORKS)
def test_fork(name):
    lens, width, P, parents, n_free, taken = FORKS[name]
    rng = np.random.default_rng(1)
    table = rng.integers(0, 1000, (len(lens), width)).tolist()
    check_fork(lens, table, parents, P, rng.permutation(500)[:n_free].tolist(), taken, stride=width + 2)


def test_fork_of_rows_without_pages():
    """A partly filled page that the parent does not have is no page of the child."""
    check_fork([20, 20], [[4, -1, 9], [3, 8, 9]], [[0, 0, 1, 1]], 16, [70, 71, 72])
    check_fork([20], [[4, 6, 9]], [[0, 0, 0]], 16, [-1, 71, -5])


@pytest.mark.parametrize("seed", range(10))
def test_fork_random(seed):
    rng = np.random.default_rng(seed)
    G = int(rng.choice([1, 2, 31, 128, 500]))
    per, n = (int(rng.integers(1, min(4096 // G, 40) + 1)) for _ in range(2))
    P, width = int(2 ** rng.integers(4, 8)), int(rng.integers(1, 60) if seed else 2000)
    lens = rng.integers(0, width * P + 20, G * per).tolist()
    table = rng.integers(0, 9999, (G * per, width)).tolist()
    parents = rng.integers(-1, per + (seed % 2), (G, n)).tolist()
    check_fork(lens, table, parents, P, rng.permutation(9000)[:int(rng.integers(0, G * n + 1))].tolist(),
               int(rng.integers(0, 9)))


def test_fork_of_most_rows():
    rng = np.random.default_rng(0)
    lens = rng.integers(0, 300, 4096).tolist()
    check_fork(lens, rng.integers(0, 9999, (4096, 20)).tolist(), rng.integers(0, 8, (512, 8)).tolist(), 16, list(range(5000)))


@pytest.mark.parametrize("rows", [255, 256, 257, 1023, 1024, 1025])
def test_fork_rows_of_a_kernel(rows):
    """Up to the rows that a kernel takes, and one more, old and new."""
    rng = np.random.default_rng(rows)
    lens, table = rng.integers(0, 70, rows).tolist(), rng.integers(0, 9999, (rows, 5)).tolist()
    check_fork(lens, table, rng.integers(0, rows, (1, rows)).tolist(), 16, list(range(2000)))
    check_fork(lens[:3], table[:3], rng.integers(0, 3, (1, rows)).tolist(), 16, list(range(2000)))
    check_fork(lens, table, rng.integers(0, rows, (1, 3)).tolist(), 16, list(range(2000)))


def test_fork_from_no_rows():
    f = sb.page_fork(i32([]), torch.empty(0, 4, dtype=torch.int32, device=DEV), i32([[0, 1]]), 16, i32([3]))
    assert f.page_table.tolist() == [[-1] * 4] * 2 and f.context_lens.tolist() == [0, 0] and f.used.tolist() == [0]
    f = sb.page_fork(i32([20]), i32([[1, 2]]), torch.empty(1, 0, dtype=torch.int32, device=DEV), 16, i32([3]))
    assert f.page_table.shape == (0, 2) and f.used.tolist() == [0]


def test_no_requests():
    """What a selection of no requests gives is forked and moved too."""
    lens, table, made = i32([]), torch.empty(0, 4, dtype=torch.int32, device=DEV), caches(1, 10, 16, 2, 64)
    usage = sb.page_usage(lens, table, 16, 10)
    choice = sb.beam_select(torch.empty(0, 100, device=DEV), torch.empty(0, 3, device=DEV))
    assert choice.parents.shape == (0, 3)
    fork = sb.page_fork(lens, table, choice.parents, 16, usage.free_pages, taken=usage.counts)
    assert fork.page_table.shape == (0, 4) and fork.context_lens.shape == fork.src.shape == (0,) and fork.used.tolist() == [0]
    sb.page_copy(made, fork.src, fork.dst, fork.tokens)
    assert sb.page_compact(fork.context_lens, fork.page_table, 16, 10).counts.tolist() == [0, 0]
    with pytest.raises(sb.SBVRError):  # rows of no group
        sb.page_fork(i32([20]), i32([[1, 2]]), choice.parents, 16, usage.free_pages)


# ---------------------------------------------------------------------------
# compaction
# ---------------------------------------------------------------------------

def compact_reference(lens, table, P, pages):
    rows = in_use(lens, table, P)
    used = sorted({p for row in rows for p in row if 0 <= p < pages})
    src = [p for p in used if p >= len(used)]
    dst = sorted(set(range(len(used))) - set(used))
    new = dict(zip(src, dst))
    out = [[new.get(p, p) if 0 <= p < pages else -1 for p in row] + [-1] * (len(old) - len(row)) for row, old in zip(rows, table)]
    pad = [-1] * (pages // 2 - len(src))
    return out, src + pad, dst + pad, [len(used), len(src)]


def check_compact(lens, table, P, pages, stride=0):
    full, view = put(table, max(stride, len(table[0])))
    want = compact_reference(lens, table, P, pages)
    c = sb.page_compact(i32(lens), view, P, pages)
    assert [getattr(c, name).tolist() for name in sb.PageCompaction.__slots__] == list(want)
    # in place
    out = sb.PageCompaction(view, c.src.clone(), c.dst.clone(), c.counts.clone())
    sb.page_compact(i32(lens), view, P, pages, out=out)
    assert [getattr(out, name).tolist() for name in sb.PageCompaction.__slots__] == list(want)
    assert bool((full[:, len(table[0]):] == 7777).all())
    # again: nothing is left to move
    again = sb.page_compact(i32(lens), view, P, pages)
    assert again.page_table.tolist() == want[0] and again.counts.tolist() == [want[3][0], 0]


@pytest.mark.parametrize("name", SIZES)
def test_compact(name):
    lens, table, P, pages = make(name, seed=1)
    check_compact(lens, table, P, pages, stride=len(table[0]) + 3)


@pytest.mark.parametrize("pages", [1, 2, 3, 32, 33, 64, 1024, 5000, 16385, 32768, 32769, 70000, 300001])
def test_compact_many_pages(pages):
    rng = np.random.default_rng(pages)
    R, width = 30, 400
    check_compact(rng.integers(0, width * 16, R).tolist(), rng.integers(0, pages, (R, width)).tolist(), 16, pages)


def test_compact_of_the_highest_pages():
    check_compact([64], [[99, 98, 97, 96]], 16, 100)
    check_compact([64], [[0, 1, 2, 3]], 16, 100)
    check_compact([32], [[1, 1]], 16, 2)


def test_compact_of_most_rows():
    rng = np.random.default_rng(0)
    check_compact(rng.integers(0, 300, 4096).tolist(), rng.integers(0, 40000, (4096, 20)).tolist(), 16, 40000)


@pytest.mark.parametrize("R,width,pages", [(4096, 70, 5000), (4096, 65, 131072), (10, 5, 131073), (300, 1000, 70000)])
def test_compact_many_entries(R, width, pages):
    rng = np.random.default_rng(R)
    lens = rng.integers(0, width * 16 + 30, R)
    lens[rng.random(R) < 0.7] //= 20
    check_compact(lens.tolist(), rng.integers(-1, pages + 1, (R, width)).tolist(), 16, pages, stride=width + 2)


@pytest.mark.parametrize("R,width,pages", [
    (2, 1024, 2500), (1, 2047, 3000), (1, 2048, 3000), (1, 2049, 3000), (2049, 1, 4100),  # with the tables, and without
    (2048, 64, 70000), (2048, 64, 131073), (1, 131073, 131072), (131, 1001, 131072)])     # one workgroup, and many
def test_compact_at_the_edges_of_its_forms(R, width, pages):
    rng = np.random.default_rng(R + width)
    lens = rng.integers(0, width * 16 + 40, R)
    lens[-1] = width * 16
    table = rng.integers(0, pages, (R, width))
    table[-1, -1], table[0, 0] = pages - 1, -1
    check_compact(lens.tolist(), table.tolist(), 16, pages, stride=width + 1)


def test_compact_without_rows():
    c = sb.page_compact(i32([]), torch.empty(0, 4, dtype=torch.int32, device=DEV), 16, 10)
    assert c.src.tolist() == [-1] * 5 and c.dst.tolist() == [-1] * 5 and c.counts.tolist() == [0, 0]


# ---------------------------------------------------------------------------
# copies
# ---------------------------------------------------------------------------

def caches(layers, pages, P, heads, dim, dtype=torch.float16, layout="token", seed=0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    made = []
    for _ in range(layers):
        shape = {"token": (pages, P, heads, dim), "head": (pages, heads, P, dim), "pair": (pages, 2, P, heads, dim)}[layout]
        t = [torch.randn(shape, generator=gen, device=DEV, dtype=dtype) for _ in range(1 if layout == "pair" else 2)]
        kv = (t[0][:, 0], t[0][:, 1]) if layout == "pair" else [x.transpose(1, 2) if layout == "head" else x for x in t]
        made.append(sb.KVCache(*kv))
    return made


def check_copy(made, src, dst, tokens):
    want = [[t.clone() for t in (c.k, c.v)] for c in made]
    pages, P = made[0].k.shape[:2]
    for i, (s, d) in enumerate(zip(src, dst)):
        if 0 <= s < pages and 0 <= d < pages:
            n = P if tokens is None else min(max(tokens[i], 0), P)
            for kv in want:
                for t in kv:
                    t[d, :n] = t[s, :n]
    sb.page_copy(made, i32(src), i32(dst), None if tokens is None else i32(tokens))
    for c, (k, v) in zip(made, want):
        assert torch.equal(c.k, k) and torch.equal(c.v, v)


@pytest.mark.parametrize("layers,P,heads,dim,dtype,layout", [
    (1, 16, 8, 128, torch.float16, "token"), (3, 64, 8, 128, torch.bfloat16, "head"), (2, 32, 3, 80, torch.float16, "pair"),
    (2, 16, 1, 8, torch.bfloat16, "token"), (1, 128, 40, 128, torch.float16, "token"), (65, 16, 2, 64, torch.float16, "token"),
    (1, 4096, 1, 64, torch.float16, "head")])
def test_copy(layers, P, heads, dim, dtype, layout):
    pages = 12
    rng = np.random.default_rng(P)
    order = rng.permutation(pages).tolist()
    src, dst = order[:4] + [order[0], 3, -1, order[1], pages], order[4:8] + [order[8], -1, 5, pages, order[9]]
    for tokens in (None, [P, 1, P - 1, P // 2, 0, 5, 5, 5, 5], [-3, P + 1, 2 ** 31 - 1, 3, P, 1, 1, 1, 1]):
        check_copy(caches(layers, pages, P, heads, dim, dtype, layout), src, dst, tokens)


def test_copy_of_one_cache_and_of_nothing():
    made = caches(1, 4, 16, 2, 64)
    check_copy(made, [], [], None)
    want = made[0].k.clone()
    want[3] = want[1]
    sb.page_copy(made[0], i32([1]), i32([3]))
    assert torch.equal(made[0].k, want)


def test_copy_between_layouts():
    """Keys head by head, values token by token."""
    made = caches(2, 9, 32, 4, 64, layout="head")
    other = caches(2, 9, 32, 4, 64, layout="token", seed=1)
    check_copy([sb.KVCache(a.k, b.v) for a, b in zip(made, other)], [0, 5], [3, 1], [32, 7])
    check_copy([sb.KVCache(b.k, a.v) for a, b in zip(made, other)], [0, 5], [3, 1], [9, 32])


def test_copy_past_32_bits():
    """Pages whose elements' numbers pass 2^31."""
    P, heads, dim, pages = 64, 8, 128, 2 ** 31 // (64 * 8 * 128) + 3
    cache = sb.KVCache.alloc(pages, P, heads, dim)
    for t in (cache.k, cache.v):
        t[pages - 2:].normal_()
        t[:2].normal_()
    want = [(t[pages - 1].clone(), t[1].clone()) for t in (cache.k, cache.v)]
    sb.page_copy(cache, i32([pages - 1, 1]), i32([0, pages - 2]))
    for t, (high, low) in zip((cache.k, cache.v), want):
        assert torch.equal(t[0], high) and torch.equal(t[pages - 2], low) and torch.equal(t[pages - 1], high)


def test_copy_of_many():
    n = 3000
    made = caches(2, 2 * n, 16, 2, 64)
    order = np.random.default_rng(0).permutation(2 * n).tolist()
    check = [t.clone() for t in (made[1].k, made[1].v)]
    sb.page_copy(made, i32(order[:n]), i32(order[n:]))
    for t, w in zip((made[1].k, made[1].v), check):
        w[order[n:]] = w[order[:n]]
        assert torch.equal(t, w)


# ---------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------

def content(cache, lens, table, P):
    """Each row's tokens, keys and values."""
    rows = []
    for c, row in zip(lens, table):
        pages = row[:-(-c // P)]
        rows.append((cache.k[pages].reshape(-1, *cache.k.shape[2:])[:c], cache.v[pages].reshape(-1, *cache.v.shape[2:])[:c]))
    return rows


@pytest.mark.parametrize("layout", ["token", "head"])
def test_rows_live_through_steps(layout):
    """Rows that are written, forked, dropped and moved together keep their
    content: every step's tokens are followed on the side."""
    R, B, P, pages, width, H, D = 2, 3, 16, 160, 12, 2, 64
    made = caches(2, pages, P, H, D, layout=layout)
    rng = np.random.default_rng(0)
    rows = R * B
    lens, table = i32([0] * rows), torch.full((rows, width), -1, dtype=torch.int32, device=DEV)
    follow = [[] for _ in range(rows)]
    for step in range(14):
        usage = sb.page_usage(lens, table, P, pages)
        new = i32(rng.integers(0, 20, rows).tolist())
        T = int(new.sum())
        plan = sb.batch_plan(lens, new, usage.free_pages, table, P, T)
        for cache in made:
            k, v = (torch.randn(T, H, D, device=DEV).half() for _ in range(2))
            sb.cache_write(cache, k, v, plan.slots)
            if cache is made[1]:
                start = plan.query_start.tolist()
                for r in range(rows):
                    follow[r] = follow[r] + [(k[t], v[t]) for t in range(start[r], start[r + 1])]
        lens += new
        parents = rng.integers(-1 if step % 5 == 4 else 0, B, (R, B)).tolist()
        fork = sb.page_fork(lens, table, i32(parents), P, usage.free_pages, taken=plan.used)
        assert int(fork.used) + int(plan.used[0]) <= int(usage.counts[0])
        sb.page_copy(made, fork.src, fork.dst, fork.tokens)
        lens, table = fork.context_lens, fork.page_table
        follow = [follow[i // B * B + p] if p >= 0 else [] for i, p in enumerate(sum(parents, []))]
        if step % 3 == 2:
            moved = sb.page_compact(lens, table, P, pages)
            sb.page_copy(made, moved.src, moved.dst)
            table = moved.page_table
            assert int(table.max()) < int(moved.counts[0])
        # rows that have grown too long start anew
        full = (lens > (width - 2) * P - 20).tolist()
        lens = i32([0 if f else n for f, n in zip(full, lens.tolist())])
        follow = [[] if f else x for f, x in zip(full, follow)]
        assert lens.tolist() == [len(x) for x in follow]
        for (k, v), tokens in zip(content(made[1], lens.tolist(), table.tolist(), P), follow):
            if tokens:
                assert torch.equal(k, torch.stack([t[0] for t in tokens]))
                assert torch.equal(v, torch.stack([t[1] for t in tokens]))


def test_in_a_graph():
    """Usage, fork, copy and compaction captured together and replayed on other
    lengths, tables and parents."""
    R, P, pages, width = 8, 16, 200, 10
    made = caches(2, pages, P, 2, 64)
    rng = np.random.default_rng(0)
    lens, table, parents = i32([0] * R), torch.zeros(R, width, dtype=torch.int32, device=DEV), i32([[0] * 4] * 2)

    def step():
        u = sb.page_usage(lens, table, P, pages)
        f = sb.page_fork(lens, table, parents, P, u.free_pages)
        sb.page_copy(made, f.src, f.dst, f.tokens)
        c = sb.page_compact(f.context_lens, f.page_table, P, pages)
        sb.page_copy(made, c.src, c.dst)
        return u, f, c
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        u, f, c = step()
    for _ in range(4):
        order = rng.permutation(pages)[:R * width].reshape(R, width)
        lens.copy_(i32(rng.integers(0, width * P, R).tolist()))
        table.copy_(i32(order.tolist()))
        parents.copy_(i32(rng.integers(0, 4, (2, 4)).tolist()))
        before = content(made[1], lens.tolist(), table.tolist(), P)
        graph.replay()
        torch.cuda.synchronize()
        want = usage_reference(lens.tolist(), table.tolist(), P, pages)
        assert [u.refs.tolist(), u.free_pages.tolist(), u.counts.tolist()] == list(want)
        forked = fork_reference(lens.tolist(), table.tolist(), parents.tolist(), P, want[1], 0)
        assert [getattr(f, n).tolist() for n in sb.PageFork.__slots__] == list(forked)
        moved = compact_reference(forked[1], forked[0], P, pages)
        assert [getattr(c, n).tolist() for n in sb.PageCompaction.__slots__] == list(moved)
        after = content(made[1], forked[1], moved[0], P)
        for i, p in enumerate(sum(parents.tolist(), [])):
            a, b = after[i], before[i // 4 * 4 + p]
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_on_another_stream():
    lens, table, P, pages = make("wide", invalid=False)
    args = i32(lens), i32(table), P, pages
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    u, c = sb.page_usage(*args, stream=other), sb.page_compact(*args, stream=other)
    other.synchronize()
    assert [u.refs.tolist(), u.free_pages.tolist(), u.counts.tolist()] == list(usage_reference(lens, table, P, pages))
    assert c.page_table.tolist() == compact_reference(lens, table, P, pages)[0]


def test_refusals():
    lens, table = i32([20, 20]), i32([[1, 2], [3, 4]])
    free, parents = i32([7, 8]), i32([[0, 1]])
    for bad in (dict(context_lens=lens.long()), dict(context_lens=lens[:1]), dict(page_table=table.t()), dict(page_table=table[0]),
                dict(n_pages=-1), dict(workspace=torch.empty(4, device=DEV)), dict(out=sb.PageUsage(lens, lens, lens))):
        with pytest.raises(AssertionError):
            sb.page_usage(**{**dict(context_lens=lens, page_table=table, page_size=16, n_pages=50), **bad})
    for bad in (dict(page_size=17), dict(page_size=8), dict(n_pages=0), dict(n_pages=(1 << 22) + 1),
                dict(page_table=table[:1].expand(2, 2)), dict(workspace=torch.empty(0, dtype=torch.uint8, device=DEV))):
        a = {**dict(context_lens=lens, page_table=table, page_size=16, n_pages=50), **bad}
        with pytest.raises(sb.SBVRError):
            sb.page_usage(**a)
        with pytest.raises(sb.SBVRError):
            sb.page_compact(**a)
    with pytest.raises(sb.SBVRError):  # in place at another stride
        room = i32([[1, 2, 0, 0], [3, 4, 0, 0]])
        view = room.as_strided((2, 2), (2, 1))
        sb.page_compact(lens, room[:, :2], 16, 50, out=sb.PageCompaction(view, *[torch.empty(25, dtype=torch.int32, device=DEV)] * 2,
                                                                         i32([0, 0])))
    for bad in (dict(parents=parents[0]), dict(parents=parents.long()), dict(free_pages=free.long()), dict(taken=free[:0]),
                dict(taken=free.long()), dict(out=sb.PageFork(*[lens] * 6))):
        with pytest.raises(AssertionError):
            sb.page_fork(**{**dict(context_lens=lens, page_table=table, parents=parents, page_size=16, free_pages=free), **bad})
    six = [torch.empty(2, dtype=torch.int32, device=DEV) for _ in range(5)]
    for bad in (dict(parents=i32([[0], [0], [0]])), dict(page_size=0), dict(out=sb.PageFork(table, *six[:4], six[4][:1])),
                dict(parents=torch.empty(0, 3, dtype=torch.int32, device=DEV))):
        with pytest.raises(sb.SBVRError):
            sb.page_fork(**{**dict(context_lens=lens, page_table=table, parents=parents, page_size=16, free_pages=free), **bad})
    a, b = caches(1, 4, 16, 2, 64)[0], caches(1, 5, 16, 2, 64)[0]
    with pytest.raises(sb.SBVRError):
        sb.page_copy([a, b], lens, lens)
    for bad in ((a, lens, lens[:1]), (a, lens.long(), lens), (a, lens, lens, lens[:1]), ([], lens, lens), (a, table, table)):
        with pytest.raises(AssertionError):
            sb.page_copy(*bad)
