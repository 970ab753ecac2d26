"""The selection of a beam search against the definition in 64 bits, at the
sizes, masks and ties where it can go wrong."""
import math

import numpy as np
import pytest
import torch

import paper_2509_18172_amd as sb

pytestmark = pytest.mark.gpu

DEV = "cuda"
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
INF = math.inf

# How far a score may be off before its own rounding: a lane sums at most 32
# exponentials in binary32 (31 roundings of 2^-24), each of them within |d| 2^-24 + 2^-23
# for the exponent's roundings (d = logit - top; beyond |d| = 20 a term adds less than
# 2^-28 of the sum a piece) and the function's own 2^-23: together below 2^-18.
OFF = 2.0 ** -18


def close(score):
    return OFF + abs(score) * 2.0 ** -24 if math.isfinite(score) else 0.0


def cleaned(row):
    """Logits as they count: NaN is -infinity, +infinity the largest number."""
    row = row.astype(np.float64)
    row[np.isnan(row)] = -INF
    return np.minimum(row, float(np.finfo(np.float32).max))


def candidates(logits, scores, request, beams, most):
    """(score, beam, token) of each beam's `most` best continuations, best first,
    and the scores of all [beam][token]."""
    found, every = [], np.full((beams, logits.shape[1]), -INF)
    for b in range(beams):
        base = float(scores[request][b])
        row = cleaned(logits[request * beams + b])
        if not math.isfinite(base) or row.max() == -INF:
            continue
        # (the largest number and a logarithm do not add up: it is subtracted first)
        every[b] = base + ((row - row.max()) - math.log(np.exp(row - row.max()).sum()))
        for v in np.argsort(-row, kind="stable")[:most]:
            if row[v] > -INF:
                found.append((-every[b, v], b, int(v)))
    found.sort()
    return [(-s, b, v) for s, b, v in found], every


def check(logits, scores, n, ends=(), got=None, exact=False):
    """got (or the operator's choice) against the definition.  Where two scores
    are nearer than their errors either may be first; exact: none are but equal ones."""
    R, B = scores.shape
    if got is None:
        e = torch.tensor(list(ends), dtype=torch.int32, device=DEV) if ends is not None else None
        got = sb.beam_select(logits, scores, n=n, end_tokens=e)
    host = logits.float().cpu().numpy() if logits.dtype != F32 else logits.cpu().numpy()
    base, ends = scores.cpu().numpy(), set(ends or ())
    tokens, parents, chosen = got.tokens.tolist(), got.parents.tolist(), got.scores.tolist()
    ended, ended_tokens = got.ended.tolist(), got.ended_tokens.tolist()
    for r in range(R):
        every, value = candidates(host, base, r, B, n + len(ends) + 1)
        going = [c for c in every if c[2] not in ends]
        real = min(n, len(going))
        assert tokens[r][real:] == [-1] * (n - real) and parents[r][real:] == [-1] * (n - real)
        assert chosen[r][real:] == [-INF] * (n - real)
        pairs = list(zip(parents[r], tokens[r]))[:real]
        assert len(set(pairs)) == real and all(value[p] > -INF and p[1] not in ends for p in pairs)
        for i, p in enumerate(pairs):
            assert abs(chosen[r][i] - value[p]) <= close(value[p]), (r, i)
            assert value[p] >= going[i][0] - 2 * OFF, (r, i)  # no better one was passed over
            if exact:
                assert p == going[i][1:], (r, i, p, going[i])
        for i in range(1, real):  # order, and equal logits of a beam by token
            (b0, v0), (b1, v1) = pairs[i - 1], pairs[i]
            assert chosen[r][i - 1] >= chosen[r][i]
            if b0 == b1 and host[r * B + b0][v0] == host[r * B + b1][v1]:
                assert v0 < v1
        last = every[min(n, len(every)) - 1][0] if every else -INF
        for b in range(B):
            mine = [c for c in every[:n] if c[1] == b and c[2] in ends]
            if mine and (exact or mine[0][0] > every[n][0] + 2 * OFF if len(every) > n else mine):
                assert ended_tokens[r][b] == mine[0][2] or abs(value[(b, ended_tokens[r][b])] - mine[0][0]) <= 2 * OFF
                assert abs(ended[r][b] - mine[0][0]) <= close(mine[0][0])
            elif ended_tokens[r][b] == -1:
                assert ended[r][b] == -INF
            else:  # an end that is as good as the n-th best
                s = value[(b, ended_tokens[r][b])]
                assert ended_tokens[r][b] in ends and s >= last - 2 * OFF and abs(ended[r][b] - s) <= close(s)
                assert not exact
    return got


def make(R, B, V, dtype, seed=0, masked=0.0, scale=3.0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    logits = (scale * torch.randn(R * B, V, generator=gen, device=DEV)).to(dtype)
    if masked:
        logits.masked_fill_(torch.rand(R * B, V, generator=gen, device=DEV) < masked, -INF)
    scores = -3.0 * torch.rand(R, B, generator=gen, device=DEV).cumsum(1)
    return logits, scores


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("R,B,V,n", [(1, 1, 1000, 1), (1, 4, 5003, 4), (3, 2, 2048, 5), (2, 5, 8191, 10), (1, 32, 777, 32),
                                     (9, 8, 3001, 16), (2, 3, 20000, 3), (1, 1, 50001, 64)])
def test_beam(dtype, R, B, V, n):
    check(*make(R, B, V, dtype), n)


@pytest.mark.parametrize("V", [1, 2, 3, 7, 8, 9, 15, 63, 64, 65, 255, 256, 257, 2047, 2049, 4097])
@pytest.mark.parametrize("n", [1, 3, 16])
def test_small_vocabularies(V, n):
    for dtype in (F16, F32):
        check(*make(2, 3, V, dtype, seed=V), n, ends=(0, V - 1) if V > 2 else ())


@pytest.mark.parametrize("R,B,V,n,ends", [(64, 8, 16385, 8, 1), (128, 4, 9000, 8, 3), (40, 16, 8192, 16, 0), (600, 1, 8193, 5, 2)])
def test_large_tiles(R, B, V, n, ends):
    """Enough rows for tiles of 8192 logits."""
    logits, scores = make(R, B, V, F16, seed=R, masked=0.05)
    rng = np.random.default_rng(R)
    check(logits, scores, n, ends=rng.permutation(V)[:ends].tolist())


@pytest.mark.parametrize("B,n,V", [(32, 32, 70001), (32, 64, 40000), (16, 64, 100003), (1, 64, 300007)])
def test_parts_of_several_tiles(B, n, V):
    """More tiles than a request may have parts."""
    check(*make(1, B, V, BF16, seed=n), n)


def test_large_tiles_in_turn():
    """Parts of several large tiles: 640 rows that 32 beams and 32 entries leave
    four parts each."""
    logits, scores = make(20, 32, 70000, F16, seed=4)
    check(logits, scores, 30, ends=(5, 69999))


@pytest.mark.parametrize("B,n,V", [(2, 33, 900), (2, 62, 900), (1, 60, 8192 + 300), (3, 40, 2048 + 100), (2, 64, 200)])
def test_hardly_filled_tiles(B, n, V):
    """Tiles with fewer groups than there are entries to keep."""
    for R in (1, 300):
        logits, scores = make(R, B, V, F32, seed=n)
        check(logits[:4 * B], scores[:4], n)
        got, few = sb.beam_select(logits, scores, n=n), sb.beam_select(logits[:4 * B], scores[:4], n=n)
        assert torch.equal(got.tokens[:4], few.tokens) and torch.equal(got.parents[:4], few.parents)


@pytest.mark.parametrize("allowed", [0, 1, 5, 30])
def test_finite_masks(allowed):
    """Rows in which all but a few tokens have one low, finite logit, as some masks
    leave them: the lowest tokens among equal ones follow."""
    for R, B, V in ((1, 2, 3000), (150, 4, 9000)):
        logits, scores = make(R, B, V, F32, seed=allowed)
        keep = torch.randperm(V, device=DEV)[:allowed]
        masked = torch.full_like(logits, -10000.0)
        masked[:, keep] = logits[:, keep]
        scores[:] = -1.0
        masked[:] = masked[:1].clone()  # (the beams alike: equal scores are equal in every form)
        check(masked[:2 * B], scores[:2], 20, ends=(0, 7), exact=True)
        got = sb.beam_select(masked, scores, n=20)
        assert bool((got.tokens == got.tokens[:1]).all()) and bool((got.parents == got.parents[:1]).all())


@pytest.mark.parametrize("order", ["rising", "falling", "equal", "two"])
@pytest.mark.parametrize("V", [300, 9000])
@pytest.mark.parametrize("n", [1, 8, 60])
def test_ordered_and_equal_logits(order, V, n):
    """Logits of which many lanes, or one, have all the best: multiples of 1/8, so
    that equal scores are equal in every form."""
    row = {"rising": np.arange(V) // 4 / 8.0, "falling": -(np.arange(V) // 4) / 8.0, "equal": np.zeros(V),
           "two": (np.arange(V) % 2) / 8.0}[order]
    row = torch.tensor(row, dtype=F32, device=DEV)
    for B in (1, 3):
        logits = row.expand(2 * B, V).contiguous()
        check(logits, torch.full((2, B), -1.0, device=DEV), n, ends=(0, V // 2, V - 1), exact=True)


def test_many_rows_of_equal_logits():
    """The same with large tiles, where a list is longest."""
    V = 8192 * 2 + 5
    logits = torch.zeros(260 * 2, V, dtype=F16, device=DEV)
    logits[::2, 100:2000] = 1.0
    check(logits, torch.zeros(260, 2, device=DEV), 30, ends=(101, 500), exact=True)
    rising = (torch.arange(V, device=DEV) // 32 / 8.0).to(F32).expand(520, V).contiguous()
    check(rising[:6], torch.zeros(3, 2, device=DEV), 30, exact=True)
    got = sb.beam_select(rising, torch.zeros(260, 2, device=DEV), n=30)
    few = sb.beam_select(rising[:2], torch.zeros(1, 2, device=DEV), n=30)
    assert torch.equal(got.tokens, few.tokens.expand(260, 30)) and torch.equal(got.parents, few.parents.expand(260, 30))


@pytest.mark.parametrize("kind", ["equal", "beams", "near", "few"])
@pytest.mark.parametrize("n", [1, 4, 16, 50])
def test_equal_lists_of_many_parts(kind, n):
    """A request whose parts' entries are all as good, or nearly: the join thins them out
    too.  Score differences are exact in binary64, rows are the same for all beams."""
    B, V = 8, 70001
    row = torch.zeros(V, device=DEV)
    if kind == "near":
        row += torch.randint(0, 1000, (V,), generator=torch.Generator(device=DEV).manual_seed(n), device=DEV) * 2.0 ** -30
    if kind == "few":
        row[[5, 30000, 70000]] = 0.125
    scores = torch.full((2, B), -1.0, device=DEV)
    if kind == "beams":
        scores[0, [2, 7]] = -0.75
        scores[1, 3] = -INF
    check(row.expand(2 * B, V).contiguous(), scores, n, ends=(0, 3, 30000, V - 1), exact=True)


@pytest.mark.parametrize("V", [100, 2500, 9000])
def test_masked_rows(V):
    """Rows and beams that leave nothing, or less than is asked for."""
    logits, scores = make(4, 3, V, F32, seed=1)
    logits[0:3] = -INF                      # a request without continuations
    logits[3] = -INF                        # one beam of three
    logits[4, 5:] = -INF                    # five tokens
    logits[5] = -INF
    logits[5, V - 1] = 2.0                  # one
    scores[2, 0] = -INF                     # beams that have ended
    scores[3] = -INF
    got = check(logits, scores, 8, ends=(4,))
    assert got.tokens[0].tolist() == [-1] * 8 and got.ended_tokens[3].tolist() == [-1] * 3
    scores[1, 1], scores[1, 2], scores[2, 1] = math.nan, INF, -INF
    check(logits, scores, 8, ends=(4,))


def test_logits_of_dead_beams_are_not_read():
    logits, scores = make(2, 2, 3000, F16, seed=2)
    scores[0, 1] = -INF
    want = sb.beam_select(logits, scores)
    logits[1] = math.nan
    got = sb.beam_select(logits, scores)
    assert torch.equal(got.tokens, want.tokens) and torch.equal(got.scores, want.scores)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_nan_and_infinite_logits(dtype):
    logits, scores = make(3, 2, 4000, dtype, seed=3)
    logits[0, 10] = math.nan
    logits[1] = math.nan
    logits[2, 7], logits[2, 3000] = INF, INF
    logits[3, ::2] = math.nan
    logits[4, 100] = INF
    logits[5, 3999] = -INF
    check(logits, scores, 4)


def test_extreme_logits():
    """Far apart, all far from 0, and so small that they are denormal."""
    V = 3000
    logits = torch.full((4, V), -1e30, dtype=F32, device=DEV)
    logits[0, 17] = 3e38
    logits[1] = torch.linspace(-3e38, 3e38, V, device=DEV)
    logits[2] = 1e30
    logits[3] = torch.linspace(0, 1e-40, V, device=DEV)
    check(logits, torch.tensor([[-1.0], [-2.0], [-3.0], [-4.0]], device=DEV), 4)
    for first, second, third in ((-1e38, 5.0, 7.0), (5.0, 1e38, -3e38), (3e38, 1.0, 3.2e38), (-3e38, -2e38, 3.0), (30.0, 2e37, 2.0)):
        logits = torch.full((1, 3 * 2048), first, dtype=F32, device=DEV)  # by tiles of a part, where there are many rows
        logits[:, 2048:4096], logits[:, 4096:] = second, third
        logits += torch.arange(3 * 2048, device=DEV) % 5
        check(logits, torch.zeros(1, 1, device=DEV), 3)
        wide = logits.repeat_interleave(4, dim=1).expand(32, -1).contiguous()
        check(wide, torch.zeros(1, 32, device=DEV), 3)


def parts_of(R, B, V, n, ends=0):
    """Parts that the operator cuts a row into: its workspace is a sum of 16 bytes
    and n + ends entries of 8 for each."""
    need, each = sb.sbvr_beam_select_workspace_bytes(R, B, V, n, ends), R * B * (16 + 8 * (n + ends))
    assert need % each == 0
    return need // each


# Rows of three tiles of 2048 or 8192 logits in one part: one request of 32 beams has too
# few rows for the large ones, and 64 entries a row leave no more parts (a part has a
# tile at least, so this stays what it is when a rule for tiles or parts moves).
IN_TURN = [(1, 2048), (2, 8192)]


def in_turn(R, tile, rows, n, ends=()):
    """check() of R requests of 32 beams, every row [three tiles]."""
    V = len(rows)
    assert parts_of(R, 32, V, n, len(ends)) == 1 and V > 2 * tile
    logits = torch.from_numpy(np.asarray(rows, np.float32)).to(DEV).expand(32 * R, V).contiguous()
    return check(logits, torch.zeros(R, 32, device=DEV), n, ends=ends, exact=True)


@pytest.mark.parametrize("R,tile", IN_TURN)
@pytest.mark.parametrize("levels", [
    (-1e38, 5.0, 7.0), (5.0, 1e38, -3e38), (3e38, 1.0, 3.2e38), (-3e38, -2e38, 3.0), (30.0, 2e37, 2.0), (-1e9, 111.3, 110.0),
    (2e6, -2e6, 1.9e6), (-INF, 3e38, 3e38), (INF, -INF, 1.0), (1e6, 1000001.0, 999999.0), (-1e9, -1e9, 0.0), (0.0, -1e9, -1e9)])
def test_extreme_tiles_in_turn(R, tile, levels):
    """The sum follows a largest logit that rises, or does not, by more than binary32
    can tell apart."""
    row = np.concatenate([np.float32(v) + np.arange(tile, dtype=np.float32) % 5 for v in levels])
    in_turn(R, tile, row, 64)


@pytest.mark.parametrize("R,tile", IN_TURN)
@pytest.mark.parametrize("kind", ["equal", "rising", "falling", "two", "steps", "stairs", "some", "plateau"])
def test_ordered_tiles_in_turn(R, tile, kind):
    """Equal logits, and lists that are too long, beside what earlier tiles have left
    (multiples of 1/8, so that equal scores are equal in every form)."""
    v = np.arange(3 * tile - 5)  # (the last piece is moved back)
    row = {"equal": 0 * v, "rising": v // 16, "falling": -(v // 16), "two": v % 2, "steps": v // tile, "stairs": -(v // tile),
           # 30 of the first tile are better than the next one's equal ones, 34 are not
           "some": np.where(v < tile, 2.0 * (v % 61 == 7) * (v < 61 * 30), 1.0),
           # the best are of the last tile, as many as are kept, behind as good ones of the first
           "plateau": 3.0 * ((v < 40) | (v > 3 * tile - 70)) + (v // tile == 1)}[kind] / 8.0
    in_turn(R, tile, row, 60, ends=(1, 7, tile, 2 * tile + 3))


def first_of(row, n, without=()):
    """The n best tokens of a beam whose scores are all the same number: by logit, and
    equal ones by number."""
    row = cleaned(row)
    order = np.argsort(-row, kind="stable")[:n + len(without)].tolist()
    return [v for v in order if v not in without and row[v] > -INF][:n]


@pytest.mark.parametrize("dtype", [F16, F32])
@pytest.mark.parametrize("V", [40, 5000, 70001, 300007])
@pytest.mark.parametrize("n,ends", [(1, 0), (4, 0), (8, 3), (40, 2), (64, 0)])
@pytest.mark.parametrize("low", [-1e30, float(np.finfo(np.float32).min)])
def test_logits_decide_where_a_score_hides_them(dtype, V, n, ends, low):
    """Beams as good as dead, whose score has no room for a logit: of one beam the
    higher logit is the better, in whatever parts of the row the two lie."""
    B = 3
    logits, _ = make(2, B, V, dtype, seed=V + n)
    logits[:, ::3] = logits[:, :1]  # many alike, too
    scores = torch.tensor([[low, low, low], [-INF, low, 0.0]], device=DEV)
    logits[5, 2:] = -INF  # two continuations of the one that lives
    host = logits.float().cpu().numpy()
    end = [int(host[b].argmax()) for b in (0, 1, 4)][:ends]
    got = sb.beam_select(logits, scores, n=n, end_tokens=torch.tensor(end, dtype=torch.int32, device=DEV))
    want = [(0, v) for v in first_of(host[0], n, end)]
    want = (want + [(1, v) for v in first_of(host[1], n, end)] + [(2, v) for v in first_of(host[2], n, end)])[:n]
    pairs = list(zip(got.parents[0].tolist(), got.tokens[0].tolist()))
    assert pairs[:len(want)] == want and pairs[len(want):] == [(-1, -1)] * (n - len(want))
    best = first_of(host[0], n)
    assert got.ended_tokens[0, 0].item() == next((v for v in best if v in end), -1)
    alive = sorted([0, 1], key=lambda v: (-host[5][v], v))
    want = ([(2, v) for v in alive if v not in end] + [(1, v) for v in first_of(host[4], n, end)])[:n]
    pairs = list(zip(got.parents[1].tolist(), got.tokens[1].tolist()))
    assert pairs[:len(want)] == want and pairs[len(want):] == [(-1, -1)] * (n - len(want))


@pytest.mark.parametrize("V", [300, 70001])
@pytest.mark.parametrize("n", [1, 5, 64])
def test_logits_decide_where_they_are_small_beside_the_sum(V, n):
    """Logits around 1e-25: exp(logit) is 1, and every score the sum's logarithm."""
    rng = np.random.default_rng(V + n)
    rows = (rng.integers(-V, V, (4, V)) * 1e-25).astype(np.float32)
    got = sb.beam_select(torch.from_numpy(rows).to(DEV), torch.full((2, 2), -2.0, device=DEV), n=n)
    for r in range(2):
        assert got.parents[r].tolist() == [0] * n and got.tokens[r].tolist() == first_of(rows[2 * r], n)


def test_zeros_of_either_sign_are_equal():
    for V in (300, 9000, 70000):
        logits = torch.zeros(2, V, dtype=F32, device=DEV)
        logits[:, ::2] = -0.0
        logits[:, V // 2:] -= 1
        check(logits, torch.zeros(1, 2, device=DEV), 10, exact=True)
        logits[:, V // 3] = 0.25
        check(logits, torch.zeros(1, 2, device=DEV), 10, exact=True)


def test_ends_among_the_best():
    """Ends inside and behind the n best, several of one beam, all of a beam."""
    V = 1000
    logits = torch.zeros(4, V, dtype=F32, device=DEV)
    logits[0, [3, 4, 5]] = torch.tensor([9.0, 8.0, 7.0], device=DEV)
    logits[1, [3, 4, 900]] = torch.tensor([7.5, 10.0, 9.5], device=DEV)
    logits[2, :] = -INF
    logits[2, [3, 4]] = 1.0
    logits[3, 5] = 5.0
    scores = torch.tensor([[0.0, -0.25], [-1.0, -2.0]], device=DEV)
    for n in (1, 2, 3, 4, 6):
        check(logits, scores, n, ends=(4, 3), exact=True)
    check(logits, scores, 2, ends=(4, 4, 3, -1, V, 2 ** 31 - 1), exact=True)  # twice, and no tokens


@pytest.mark.parametrize("n", [1, 2, 30])
def test_only_ends(n):
    V = 50
    logits, scores = make(2, 2, V, F32, seed=5)
    check(logits, scores, n, ends=range(0, 34))


def test_rows_of_a_larger_matrix():
    logits, scores = make(3, 2, 4001, F16, seed=6)
    want = sb.beam_select(logits, scores)
    room = torch.full((6, 4100), 60000.0, dtype=F16, device=DEV)
    room[:, 3:4004] = logits
    got = sb.beam_select(room[:, 3:4004], scores)
    for name in sb.BeamChoice.__slots__:
        assert torch.equal(getattr(got, name), getattr(want, name))


def test_one_row_for_all_beams():
    """An expanded prompt's logits (row stride 0): equal beams are told apart by
    their scores, and then by their number."""
    logits, _ = make(1, 1, 6000, F32, seed=7)
    rows = logits.expand(4, 6000)
    check(rows, torch.tensor([[-1.0, -1.0], [-1.0, -INF]], device=DEV), 4, exact=True)


@pytest.mark.parametrize("seed", range(8))
def test_random(seed):
    rng = np.random.default_rng(seed)
    R, B = int(rng.integers(1, 20)), int(rng.integers(1, 17))
    V, n = int(rng.integers(1, 12000)), int(rng.integers(1, 40))
    logits, scores = make(R, B, V, [F16, BF16, F32][seed % 3], seed=seed, masked=float(rng.random()) * 0.9)
    check(logits, scores, n, ends=rng.integers(0, V, int(rng.integers(0, 5))).tolist())


def test_equal_best_among_many_close_ones():
    """Each tile better than those before, its four best equal, all others so close that
    they are listed first: of equal ones the lower token is the better."""
    V, B = 8192 * 15, 32
    rng = np.random.default_rng(0)
    scores = torch.full((1, B), -100.0, device=DEV)
    scores[0, 5] = 0
    for trial in range(100):
        # tile t from 1 + 1000 t 2^-23 on: all of them 1 to 7 bits behind the point
        base = np.arange(V) // 2048 * 1000 + rng.integers(0, 999, V)
        best = V - 2048 + rng.permutation(2048)[:4]
        base[best] = 60 * 1000
        row = torch.from_numpy((1 + base * 2.0 ** -23).astype(np.float32))
        got = sb.beam_select(row.to(DEV).expand(B, V).contiguous(), scores, n=4)
        assert got.tokens[0].tolist() == sorted(best.tolist()), trial
        assert got.parents[0].tolist() == [5] * 4


@pytest.mark.parametrize("R,tile", IN_TURN)
@pytest.mark.parametrize("low", [-1e9, float(np.finfo(np.float32).min), -2e6, 1.0])
@pytest.mark.parametrize("near", [111.0, 1000.0, 30000.0, 900000.0])
def test_a_sum_of_several_tiles_refers_to_one_number(R, tile, low, near):
    """A tile of masked logits, one that has the largest, one that has most of the sum:
    the last two are of one part, and what rounding the largest's exponent (up to half
    a unit of its last place: 5e-6 of the sum near 111, 1e-3 near 30000) does to one
    it has to do to the other."""
    B, n, V = 32, 64, 3 * tile
    assert parts_of(R, B, V, n) == 1  # three tiles, or twelve
    some = np.float32(near) + np.arange(1000, dtype=np.float32) * np.spacing(np.float32(near))
    exponent = some.astype(np.float64) * float(np.float32(1.44269502))
    top = some[np.abs(exponent.astype(np.float32) - exponent).argmax()]
    row = np.full(V, low, np.float32)
    row[tile:2 * tile] = top - np.float32(20)
    row[tile + 77] = top
    row[2 * tile:] = top - np.arange(tile, dtype=np.float32) % 64 / np.float32(16)
    row[2 * tile::64] = top - np.float32(1 / 16)  # (the largest is in the tile before)
    logits = torch.from_numpy(row).to(DEV).expand(R * B, V).contiguous()
    check(logits, torch.zeros(R, B, device=DEV), n)


def test_equal_best_in_a_thinned_list():
    """A tile's four best are equal and alone above some hundred that are listed with
    them, behind tiles that have filled the list of the kept: where they lie in four
    wavefronts' shares of the list (3 of 32 times, by the order of the additions to
    it), thinning leaves exactly them, and they have to be put in order all the same."""
    B, n, tile, V = 32, 4, 8192, 8192 * 45
    assert V >= 3 * tile * parts_of(1, B, V, n)
    rng = np.random.default_rng(0)
    scores = torch.full((1, B), -100.0, device=DEV)
    scores[0, 5] = 0
    for trial in range(100):
        row = np.full(V, -3.0, np.float32)
        for t in range(V // tile):  # a thousand that share their upper 16 bits, each tile's above the last one's
            at = t * tile + rng.permutation(tile)[:1000]
            row[at] = 1 + (t * 1000 + rng.integers(0, 999, 1000)) * 2.0 ** -23
        best = V - tile + rng.permutation(tile)[:4]
        row[best] = 1 + 60 * 1000 * 2.0 ** -23
        got = sb.beam_select(torch.from_numpy(row).to(DEV).expand(B, V).contiguous(), scores, n=n)
        assert got.tokens[0].tolist() == sorted(best.tolist()), trial
        assert got.parents[0].tolist() == [5] * 4


@pytest.mark.parametrize("R,B,V", [(1, 4, 1000), (40, 8, 5001), (2047, 32, 100), (3, 32, 60000)])
def test_scores_in_place(R, B, V):
    logits = torch.randn(R * B, V, device=DEV, generator=torch.Generator(device=DEV).manual_seed(R))
    scores = torch.randn(R, B, device=DEV, generator=torch.Generator(device=DEV).manual_seed(V))
    want = sb.beam_select(logits, scores)
    out = sb.BeamChoice(*(torch.empty_like(getattr(want, n)) for n in sb.BeamChoice.__slots__))
    out.scores = scores
    sb.beam_select(logits, scores, out=out)
    for n in sb.BeamChoice.__slots__:
        assert torch.equal(getattr(out, n), getattr(want, n)), n


def test_offsets_past_32_bits():
    """More than 2^31 logits: the last rows are as if they were alone."""
    V, rows = 60_000_001, 37
    logits = torch.empty(rows, V, dtype=F16, device=DEV).normal_(generator=torch.Generator(device=DEV).manual_seed(0))
    logits[-1, [3, V - 1, 77]] = torch.tensor([20.0, 19.0, 18.0], dtype=F16, device=DEV)
    scores = torch.zeros(rows, 1, device=DEV)
    got, alone = sb.beam_select(logits, scores, n=5), sb.beam_select(logits[-2:].contiguous(), scores[-2:], n=5)
    assert got.tokens[-1, :3].tolist() == [3, V - 1, 77]
    assert torch.equal(got.tokens[-2:], alone.tokens)
    assert float((got.scores[-2:] - alone.scores).abs().max()) <= 2 * close(20.0)


def test_the_same_call_gives_the_same_bits():
    logits, scores = make(16, 8, 30000, F16, seed=8)
    a = sb.beam_select(logits, scores, n=16)
    for _ in range(3):
        b = sb.beam_select(logits, scores, n=16)
        for name in sb.BeamChoice.__slots__:
            assert torch.equal(getattr(a, name), getattr(b, name))


def test_steps_of_a_search():
    """Three steps, each on the scores of the one before, as one search: the sums
    of the steps' exact scores."""
    R, B, V = 2, 4, 500
    scores = torch.full((R, B), -INF, device=DEV)
    scores[:, 0] = 0
    for step in range(3):
        logits, _ = make(R, B, V, F32, seed=20 + step)
        scores = check(logits, scores, B, ends=(1,)).scores


def test_in_a_graph():
    logits, scores = make(2, 4, 9000, F16, seed=9)
    out, ws = sb.beam_select(logits, scores, n=6, end_tokens=torch.tensor([7], dtype=torch.int32, device=DEV)), None
    ws = torch.empty(sb.sbvr_beam_select_workspace_bytes(2, 4, 9000, 6, 1), dtype=torch.uint8, device=DEV)
    ends = torch.tensor([7], dtype=torch.int32, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sb.beam_select(logits, scores, n=6, end_tokens=ends, out=out, workspace=ws)
    for step in range(4):
        l, s = make(2, 4, 9000, F16, seed=30 + step)
        logits.copy_(l)
        scores.copy_(s)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        eager = check(l, s, 6, ends=(7,))
        for name in sb.BeamChoice.__slots__:
            assert torch.equal(getattr(out, name), getattr(eager, name))


def test_two_at_once():
    """Two calls on two streams, each with a workspace of its own."""
    a, b = make(8, 4, 30000, F16, seed=10), make(8, 4, 30000, F16, seed=11)
    want = [sb.beam_select(*x) for x in (a, b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [sb.beam_select(*x, stream=s) for x, s in zip((a, b), streams)]
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert torch.equal(g.tokens, w.tokens) and torch.equal(g.scores, w.scores)


def test_no_requests():
    got = sb.beam_select(torch.empty(0, 100, dtype=F16, device=DEV), torch.empty(0, 4, device=DEV))
    assert got.tokens.shape == (0, 4) and got.ended.shape == (0, 4)


def test_refusals():
    logits, scores = make(2, 4, 100, F16)
    ends = torch.tensor([1], dtype=torch.int32, device=DEV)
    for bad in (dict(logits=logits[:7]), dict(logits=logits.double()), dict(logits=logits.t()), dict(scores=scores.double()),
                dict(scores=scores[0]), dict(scores=scores.t()), dict(end_tokens=ends.long()), dict(end_tokens=ends[None]),
                dict(workspace=torch.empty(4, device=DEV)), dict(n=-1),
                dict(out=sb.BeamChoice(*[torch.empty(2, 3, device=DEV)] * 5))):
        with pytest.raises(AssertionError):
            sb.beam_select(**{**dict(logits=logits, scores=scores, end_tokens=ends), **bad})
    small = torch.empty(64, dtype=torch.uint8, device=DEV)
    for bad in (dict(n=0), dict(n=65), dict(n=64, end_tokens=ends), dict(workspace=small),
                dict(logits=logits.expand(2, 8, 100).reshape(16, 100)[:0], scores=scores[:, :0])):
        with pytest.raises(sb.SBVRError):
            sb.beam_select(**{**dict(logits=logits, scores=scores), **bad})
    with pytest.raises(sb.SBVRError):
        sb.beam_select(torch.zeros(33, 50, device=DEV), torch.zeros(1, 33, device=DEV))
