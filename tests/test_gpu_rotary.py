"""The rotation of queries and keys by their positions against the definition in
64 bits, at the sizes, layouts and positions where it can go wrong."""
import numpy as np
import pytest
import torch

import paper_2509_18172_amd as sb

pytestmark = pytest.mark.gpu

DEV = "cuda"
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
HALF = {F16: 2.0 ** -11, BF16: 2.0 ** -8, F32: 2.0 ** -24}  # one rounding, relative
INF, NAN = float("inf"), float("nan")
LEAST = {F16: 2.0 ** -25, BF16: 2.0 ** -134, F32: 2.0 ** -150}  # and below the normal numbers


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def frequencies(n):
    return torch.tensor([10000.0 ** (-i / n) for i in range(n)], dtype=F32, device=DEV)


def reference(x, positions, freq, axes=None, interleaved=False, inverse=False):
    """The turned x in binary64 and how far a result may be off before its own
    rounding: sines and cosines are within 2^-22 (the turn is rounded to 24 bits:
    2^-24 of at most pi; the function adds at most 2 units of 2^-24), the two
    products and the sum add 2^-23, so (|a| + |b|) 2^-21 covers them; the angle in
    64 bits is off by three roundings of 2^-53, and the reference's by one."""
    x, freq = x.double().cpu(), freq.double().cpu()
    pos = positions.cpu().view(-1, x.shape[0]).double()
    y, off = x.clone(), torch.zeros_like(x)
    for i in range(freq.numel()):
        axis = 0 if axes is None else int(axes[i])
        if not 0 <= axis < pos.shape[0]:
            continue
        angle = pos[axis] * freq[i] * (-1 if inverse else 1)
        c, s = angle.cos()[:, None], angle.sin()[:, None]
        ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + freq.numel())
        a, b = x[..., ia], x[..., ib]
        y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
        off[..., ia] = off[..., ib] = (a.abs() + b.abs()) * (2.0 ** -21 + angle.abs()[:, None] * 2.0 ** -51)
    return y, off


def check(got, want, x_dtype):
    y, off = want
    got = got.double().cpu()
    bound = off + (y.abs() + off) * HALF[x_dtype] + LEAST[x_dtype]
    worst = ((got - y).abs() - bound).max().item() if got.numel() else 0
    assert worst <= 0, worst


def qkv(T, H, K, D, dtype, seed=0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn(T, H + 2 * K, D, generator=gen, device=DEV, dtype=dtype)
    return x[:, :H], x[:, H:H + K], x[:, H + K:]


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("T,H,K", [(1, 32, 8), (1, 1, 1), (7, 24, 4), (300, 8, 1), (33, 64, 8)])
@pytest.mark.parametrize("D,n", [(128, 64), (128, 32), (64, 32), (80, 40), (96, 24)])
def test_rotary(dtype, T, H, K, D, n):
    q, k, _ = qkv(T, H, K, D, dtype)
    pos = i32(np.random.default_rng(T).integers(0, 200000, T))
    for interleaved in (False, True):
        got = sb.rotary(q, k, pos, frequencies(n), interleaved=interleaved)
        for g, x in zip(got, (q, k)):
            assert g.shape == x.shape and g.is_contiguous()
            check(g, reference(x, pos, frequencies(n), interleaved=interleaved), dtype)


@pytest.mark.parametrize("D,n", [(8, 1), (8, 4), (16, 7), (64, 1), (64, 9), (128, 37), (72, 36), (512, 256), (512, 100)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("in_place", [False, True])
def test_odd_pairs(D, n, interleaved, in_place):
    q, k, _ = qkv(19, 5, 3, D, F16)
    pos = i32(list(range(19)))
    want = [reference(x, pos, frequencies(n), interleaved=interleaved) for x in (q, k)]
    got = sb.rotary(q, k, pos, frequencies(n), interleaved=interleaved, **(dict(q_out=q, k_out=k) if in_place else {}))
    for g, w in zip(got, want):
        check(g, w, F16)


@pytest.mark.parametrize("position", [0, 1, -1, 131071, 10 ** 6 + 1, 2 ** 31 - 1, -2 ** 31])
def test_far_positions(position):
    q, k, _ = qkv(3, 2, 1, 64, F32)
    pos = i32([position] * 3)
    freq = frequencies(32)
    for g, x in zip(sb.rotary(q, k, pos, freq), (q, k)):
        check(g, reference(x, pos, freq), F32)


@pytest.mark.parametrize("axes", [1, 2, 3])
def test_several_axes(axes):
    T, n = 50, 64
    q, k, _ = qkv(T, 4, 2, 128, BF16)
    pos = i32(np.random.default_rng(0).integers(0, 5000, (axes, T)))
    which = [i % axes for i in range(n)]
    which[3], which[10], which[63] = -1, axes, 2 ** 31 - 1  # of no axis: not turned
    for g, x in zip(sb.rotary(q, k, pos, frequencies(n), axes=i32(which)), (q, k)):
        check(g, reference(x, pos, frequencies(n), which), BF16)
    # rows of a longer list, as a padded batch has them
    long = torch.full((axes, T + 14), 99999, dtype=torch.int32, device=DEV)
    long[:, :T] = pos
    a = sb.rotary(q, None, long[:, :T], frequencies(n), axes=i32(which))[0]
    b = sb.rotary(q, None, pos, frequencies(n), axes=i32(which))[0]
    assert torch.equal(a, b)


@pytest.mark.parametrize("T", [1, 50])
def test_expanded_positions(T):
    """A text's positions are the same on all axes: one row, expanded."""
    n = 32
    q, k, v = qkv(T, 4, 2, 64, F16)
    pos, which = i32(list(range(7, 7 + T))), i32([i % 3 for i in range(n)])
    want = sb.rotary(q, k, pos, frequencies(n))
    for g, w in zip(sb.rotary(q, k, pos.expand(3, T), frequencies(n), axes=which), want):
        assert torch.equal(g, w)
    cache, slots = caches(-(-T // 16), 16, 2, 64, F16, "token"), torch.arange(T, device=DEV)
    assert torch.equal(sb.rotary_write(q, cache, k, v, slots, pos.expand(3, T), frequencies(n), axes=which), want[0])
    assert torch.equal(cache.k.reshape(-1, 2, 64)[:T], want[1])


def test_one_of_the_two():
    q, k, _ = qkv(5, 4, 2, 64, F16)
    pos, freq = i32([3, 1, 4, 1, 5]), frequencies(32)
    both = sb.rotary(q, k, pos, freq)
    a, none = sb.rotary(q, None, pos, freq)
    assert none is None and torch.equal(a, both[0])
    none, b = sb.rotary(None, k, pos, freq)
    assert none is None and torch.equal(b, both[1])


def test_inverse_is_the_gradient():
    """d(y . g)/dx of the definition is the inverse rotation of g, also against
    differences of the operator itself."""
    T, D, n = 6, 64, 24
    q, _, _ = qkv(T, 2, 1, D, F32)
    g = torch.randn(q.shape, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1))
    pos, freq = i32([0, 5, 77, 1000, 30000, 131071]), frequencies(n)
    x = q.double().cpu().requires_grad_()
    angle = pos.cpu().double()[:, None] * freq.cpu().double()
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    a, b = x[..., :n], x[..., n:2 * n]
    y = torch.cat([a * c - b * s, b * c + a * s, x[..., 2 * n:]], dim=-1)
    (y * g.double().cpu()).sum().backward()
    grad = sb.rotary(g, None, pos, freq, inverse=True)[0]
    check(grad, (x.grad, reference(g, pos, freq, inverse=True)[1]), F32)
    # the operator is linear: a step of 1 has no error but rounding's, 16 elements
    # of up to 4 each within 2^-20
    for t, h, d in ((0, 0, 0), (3, 1, 10), (5, 0, 47), (5, 1, 50)):
        step = torch.zeros_like(q)
        step[t, h, d] = 1
        y1, y0 = (sb.rotary(v.contiguous(), None, pos, freq)[0].double() for v in (q + step, q - step))
        slope = ((y1 - y0) / 2 * g.double()).sum().item()
        assert abs(slope - grad[t, h, d].item()) <= 2.0 ** -20 * 2 * 4 * 4


def test_turned_back():
    q, k, _ = qkv(40, 4, 2, 128, F32)
    pos, freq = i32(list(range(0, 40000, 1000))), frequencies(64)
    back = sb.rotary(*sb.rotary(q, k, pos, freq), pos, freq, inverse=True)
    for b, x in zip(back, (q, k)):  # two turns of at most 2^-20 (|a| + |b|) each
        assert (b - x).abs().max().item() <= 2 * 2.0 ** -20 * 2 * x.abs().max().item()


def test_outputs_given():
    """Outputs with strides of their own; what lies between their rows stays."""
    T, H, D = 9, 3, 64
    q, _, _ = qkv(T, H, 1, D, F16)
    pos, freq = i32(list(range(T))), frequencies(32)
    want = sb.rotary(q, None, pos, freq)[0]
    room = torch.full((T, H + 2, D + 8), 7.0, dtype=F16, device=DEV)
    view = room[:, 1:H + 1, :D]
    assert sb.rotary(q, None, pos, freq, q_out=view)[0] is not None
    assert torch.equal(view, want)
    keep = torch.ones_like(room, dtype=torch.bool)
    keep[:, 1:H + 1, :D] = False
    assert bool((room[keep] == 7).all())
    # heads first, as another layout of the batch
    other = torch.empty(H, T, D, dtype=F16, device=DEV)
    sb.rotary(q, None, pos, freq, q_out=other.transpose(0, 1))
    assert torch.equal(other.transpose(0, 1), want)


def test_infinite_and_nan_elements_stay_theirs():
    """An element that is not finite reaches its pair and nothing else."""
    q, _, _ = qkv(2, 2, 1, 64, F16)
    q = q.contiguous()
    pos, freq = i32([3, 4]), frequencies(16)
    want = sb.rotary(q, None, pos, freq)[0]
    q[1, 0, 5], q[1, 1, 40] = float("nan"), float("inf")
    got = sb.rotary(q, None, pos, freq)[0]
    bad = torch.zeros_like(want, dtype=torch.bool)
    bad[1, 0, 5] = bad[1, 0, 21] = bad[1, 1, 40] = True
    assert torch.equal(got[~bad], want[~bad]) and not bool(got[bad].isfinite().any())


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("D,n", [(64, 32), (64, 27), (8, 3)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("in_place", [False, True])
def test_pairs_of_no_axis_keep_their_bits(dtype, D, n, interleaved, in_place):
    """Each of a pair that is not turned stays what it is, whatever the other one is:
    infinite, no number, a zero of either sign."""
    T = 4 * 36
    odd = torch.tensor([INF, -INF, NAN, 0.0, -0.0, 1.5], device=DEV)
    x = torch.randn(T, 3, D, device=DEV, generator=torch.Generator(device=DEV).manual_seed(0)).to(dtype)
    still = [i for i in range(n) if i % 3 == 1 or i == n - 1]
    at = [(2 * i, 2 * i + 1) if interleaved else (i, i + n) for i in still]
    for t in range(T):
        for a, b in at:
            x[t, :, a], x[t, :, b] = odd[t % 36 // 6], odd[t % 6]
    pos, axes = i32(list(range(T))), i32([[-1, 1, 7][i % 3] if i in still else 0 for i in range(n)])
    x0 = x.clone()
    got = sb.rotary(x, None, pos, frequencies(n), axes=axes, interleaved=interleaved, q_out=x if in_place else None)[0]
    keep = sum(at, ())
    bits = torch.int32 if dtype == F32 else torch.int16
    assert torch.equal(got[..., keep].view(bits), x0[..., keep].view(bits))
    turned = [e for e in range(D) if e not in keep]
    want = sb.rotary(torch.where(x0.isfinite(), x0, 0), None, pos, frequencies(n), axes=axes, interleaved=interleaved)[0]
    assert torch.equal(got[..., turned], want[..., turned])


@pytest.mark.parametrize("T", [1, 8, 300, 5000])
def test_large(T):
    q, k, _ = qkv(T, 64, 8, 128, BF16)
    pos = torch.arange(T, dtype=torch.int32, device=DEV) + 100000
    got = sb.rotary(q, k, pos, frequencies(64))
    rows = [0, T // 3, T - 1]
    for g, x in zip(got, (q, k)):
        check(g[rows], reference(x[rows], pos[rows], frequencies(64)), BF16)
    again = sb.rotary(q, k, pos, frequencies(64))
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


# ---------------------------------------------------------------------------
# with the cache write
# ---------------------------------------------------------------------------

def caches(pages, P, heads, dim, dtype, layout):
    shape = (pages, P, heads, dim) if layout == "token" else (pages, heads, P, dim)
    t = [torch.full(shape, 5.0, dtype=dtype, device=DEV) for _ in range(2)]
    return sb.KVCache(*[x.transpose(1, 2) if layout == "head" else x for x in t])


@pytest.mark.parametrize("T", [1, 3, 40, 700])
@pytest.mark.parametrize("H,K,D,n,P,dtype,layout,interleaved", [
    (32, 8, 128, 64, 16, F16, "token", False), (4, 1, 64, 32, 32, BF16, "head", True), (16, 16, 80, 37, 64, F16, "head", False),
    (24, 4, 96, 3, 16, BF16, "token", False), (8, 8, 8, 4, 16, F16, "token", True)])
def test_rotary_write(T, H, K, D, n, P, dtype, layout, interleaved):
    q, k, v = qkv(T, H, K, D, dtype)
    rng = np.random.default_rng(T)
    pages = -(-T // P) + 3
    slots = rng.permutation(pages * P)[:T].astype(np.int64)
    if T > 2:
        slots[1], slots[2] = -1, pages * P  # no page, and past the cache
    pos, freq = i32(rng.integers(0, 100000, T)), frequencies(n)
    want_q, want_k = sb.rotary(q, k, pos, freq, interleaved=interleaved)
    want, got = caches(pages, P, K, D, dtype, layout), caches(pages, P, K, D, dtype, layout)
    slots = torch.tensor(slots, device=DEV)
    sb.cache_write(want, want_k, v, slots)
    got_q = sb.rotary_write(q, got, k, v, slots, pos, freq, interleaved=interleaved)
    assert torch.equal(got_q, want_q) and torch.equal(got.k, want.k) and torch.equal(got.v, want.v)
    check(got_q, reference(q, pos, freq, interleaved=interleaved), dtype)
    # keys and values alone, and queries in place
    alone = caches(pages, P, K, D, dtype, layout)
    assert sb.rotary_write(None, alone, k, v, slots, pos, freq, interleaved=interleaved) is None
    assert torch.equal(alone.k, want.k) and torch.equal(alone.v, want.v)
    sb.rotary_write(q, alone, k, v, slots, pos, freq, interleaved=interleaved, q_out=q)
    assert torch.equal(q, want_q)


def test_rotary_write_past_32_bits():
    """Slots whose elements' numbers pass 2^31."""
    P, K, D = 64, 8, 128
    pages = 2 ** 31 // (P * K * D) + 3
    q, k, v = qkv(3, 8, K, D, F16)
    cache = sb.KVCache.alloc(pages, P, K, D)
    slots, pos = torch.tensor([pages * P - 1, 5, (pages - 1) * P], device=DEV), i32([9, 100, 70000])
    _, want = sb.rotary(q, k, pos, frequencies(64))
    sb.rotary_write(q, cache, k, v, slots, pos, frequencies(64))
    for t, w in ((cache.k, want), (cache.v, v)):
        assert torch.equal(torch.stack([t[s // P, s % P] for s in slots.tolist()]), w)


def test_rotary_write_axes_and_inverse():
    T, K, D, n, P = 20, 2, 64, 32, 16
    q, k, v = qkv(T, 4, K, D, F16)
    pos, which = i32(np.random.default_rng(0).integers(0, 999, (3, T))), i32([i % 3 for i in range(n)])
    cache, slots = caches(4, P, K, D, F16, "token"), torch.arange(T, device=DEV)
    got = sb.rotary_write(q, cache, k, v, slots, pos, frequencies(n), axes=which, inverse=True)
    a, b = sb.rotary(q, k, pos, frequencies(n), axes=which, inverse=True)
    assert torch.equal(got, a) and torch.equal(cache.k.reshape(-1, K, D)[:T], b)


# ---------------------------------------------------------------------------
# graphs, streams, refusals
# ---------------------------------------------------------------------------

def test_in_a_graph():
    T = 8
    q, k, v = qkv(T, 8, 2, 64, F16)
    pos, freq, slots = i32([0] * T), frequencies(32), torch.arange(T, device=DEV)
    cache, out = caches(2, 16, 2, 64, F16, "token"), torch.empty(T, 8, 64, dtype=F16, device=DEV)
    sb.rotary_write(q, cache, k, v, slots, pos, freq, q_out=out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sb.rotary_write(q, cache, k, v, slots, pos, freq, q_out=out)
    for step in range(4):
        pos.copy_(i32(list(range(step * 100, step * 100 + T))))
        graph.replay()
        torch.cuda.synchronize()
        a, b = sb.rotary(q, k, pos, freq)
        assert torch.equal(out, a) and torch.equal(cache.k.view(-1, 2, 64)[:T], b)


def test_on_another_stream():
    q, k, _ = qkv(100, 8, 2, 64, F16)
    pos, freq = i32(list(range(100))), frequencies(32)
    want = sb.rotary(q, k, pos, freq)
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    got = sb.rotary(q, k, pos, freq, stream=other)
    other.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_no_tokens():
    q, k, v = qkv(0, 4, 2, 64, F16)
    pos, freq = i32([]), frequencies(32)
    a, b = sb.rotary(q, k, pos, freq)
    assert a.shape == q.shape and b.shape == k.shape
    cache = caches(2, 16, 2, 64, F16, "token")
    assert sb.rotary_write(q, cache, k, v, torch.empty(0, dtype=torch.int64, device=DEV), pos, freq).shape == q.shape


def test_refusals():
    q, k, v = qkv(4, 4, 2, 64, F16)
    pos, freq = i32([0, 1, 2, 3]), frequencies(32)

    def refused(error, *args, **more):
        with pytest.raises(error):
            sb.rotary(*args, **more)
    refused(AssertionError, None, None, pos, freq)
    refused(AssertionError, q.cpu(), None, pos, freq)
    refused(AssertionError, q, k.float(), pos, freq)
    refused(AssertionError, q, k[:3], pos, freq)
    refused(AssertionError, q.double(), None, pos, freq)
    refused(AssertionError, q, k, pos.long(), freq)
    refused(AssertionError, q, k, pos[:3], freq)
    refused(AssertionError, q, k, pos, freq.double())
    refused(AssertionError, q, k, pos, freq, axes=i32([0] * 31))
    refused(AssertionError, q, None, pos, freq, k_out=k)
    refused(AssertionError, q.transpose(1, 2), None, pos, freq)
    refused(sb.SBVRError, q, k, pos, frequencies(33))                             # more than half of a head
    refused(sb.SBVRError, q, k, pos, freq[:0])
    refused(sb.SBVRError, q[..., :60], None, pos, frequencies(30))                # head_dim
    refused(sb.SBVRError, q, k, i32([[0, 1, 2, 3]] * 2).as_strided((2, 4), (1, 1)), freq)  # axes that overlap
    refused(sb.SBVRError, q, None, pos, freq, q_out=q[:1].expand(4, 4, 64))       # rows that overlap
    refused(sb.SBVRError, q, None, pos, freq, q_out=torch.empty(4 * 4 * 72 + 4, dtype=F16, device=DEV)[4:].as_strided(
        (4, 4, 64), (288, 72, 1)))                                                # 8 bytes off
    cache = caches(2, 16, 2, 64, F16, "token")
    slots = torch.arange(4, device=DEV)
    for bad in (dict(k=k[:, :1]), dict(v=v[:3]), dict(slots=slots.int()), dict(k=k.to(BF16)), dict(q=q.to(BF16)),
                dict(q=q[:3]), dict(q_out=q[:3])):
        a = dict(q=q, cache=cache, k=k, v=v, slots=slots, positions=pos, frequencies=freq)
        with pytest.raises(AssertionError):
            sb.rotary_write(**{**a, **bad})
    with pytest.raises(AssertionError):
        sb.rotary_write(None, cache, k, v, slots, pos, freq, q_out=q)
