"""Refusals of the rotation, the beam selection and the operators on pages, on
the host: a bad argument returns its status before any HIP call, so the pointers
here are never dereferenced.  And what their tensor helpers hand to the library."""
import ctypes as C

import pytest
import torch

import paper_2509_18172_amd as sb
from paper_2509_18172_amd import step
from test_step_binding import Calls, Shell

FAKE = 1 << 20  # 16-byte-aligned
INVALID, UNSUPPORTED, WORKSPACE, ALIGNMENT = (sb.SBVR_E_INVALID_ARG, sb.SBVR_E_UNSUPPORTED, sb.SBVR_E_WORKSPACE,
                                              sb.SBVR_E_ALIGNMENT)


def cache(**more):
    c = dict(k=FAKE, v=FAKE, k_page_stride=16384, k_token_stride=1024, k_head_stride=128, v_page_stride=16384,
             v_token_stride=1024, v_head_stride=128, n_pages=4, page_size=16, kv_heads=8, head_dim=128,
             dtype=sb.SBVR_F16)
    c.update(more)
    return sb.CacheStruct(**c)


def rotation(**more):
    a = dict(T=4, heads=32, kv_heads=8, head_dim=128, dtype=sb.SBVR_F16, pairs=64, axes=1, positions=FAKE, position_stride=4,
             frequencies=FAKE)
    for n, heads in (("q", 32), ("k", 8), ("q_out", 32), ("k_out", 8)):
        a.update({n: FAKE + (1 << 16) * ("out" in n), n + "_token_stride": heads * 128, n + "_head_stride": 128})
    a.update(more)
    return sb.RotaryStruct(**a)


BAD_ROTATION = [
    (dict(T=-1), INVALID), (dict(heads=0, kv_heads=0), INVALID), (dict(heads=-1), INVALID), (dict(kv_heads=-1), INVALID),
    (dict(head_dim=0), INVALID), (dict(head_dim=124), INVALID), (dict(pairs=0), INVALID), (dict(pairs=65), INVALID),
    (dict(axes=0), INVALID), (dict(dtype=3), INVALID), (dict(dtype=-1), INVALID), (dict(interleaved=2), INVALID),
    (dict(inverse=-1), INVALID), (dict(position_stride=-1), INVALID), (dict(axes=2, position_stride=3), INVALID),
    (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(q_out=None), INVALID), (dict(positions=None), INVALID),
    (dict(frequencies=None), INVALID), (dict(q_token_stride=-8), INVALID), (dict(k_head_stride=4), INVALID),
    (dict(q_out_token_stride=4088), INVALID), (dict(q_out_token_stride=0), INVALID), (dict(q_out_head_stride=0), INVALID),
    (dict(q_out_head_stride=120), INVALID), (dict(q_out=FAKE, q_out_token_stride=8192), INVALID),
    (dict(heads=4097), UNSUPPORTED), (dict(kv_heads=4097), UNSUPPORTED), (dict(head_dim=520), UNSUPPORTED),
    (dict(q=FAKE + 8), ALIGNMENT), (dict(q_out=FAKE + 2), ALIGNMENT), (dict(k=FAKE + 4), ALIGNMENT),
    (dict(positions=FAKE + 2), ALIGNMENT), (dict(pair_axis=FAKE + 1), ALIGNMENT), (dict(frequencies=FAKE + 2), ALIGNMENT)]


@pytest.mark.parametrize("bad,status", BAD_ROTATION + [
    (dict(k_out=None), INVALID), (dict(k_out_token_stride=8), INVALID), (dict(k_out=FAKE + 2), ALIGNMENT),
    (dict(k_out=FAKE, k_out_head_stride=256, k_out_token_stride=2048), INVALID)])
def test_rotary_refusals(bad, status):
    assert sb.sbvr_rotary(rotation(**bad)) == status


def write(a=None, c=None, v=FAKE, vt=1024, vh=128, slots=FAKE, **more):
    return sb.sbvr_rotary_write(a or rotation(**{"k_out": None, **more}), c or cache(), v, vt, vh, slots)


@pytest.mark.parametrize("bad,status", [b for b in BAD_ROTATION if not {"head_dim", "kv_heads", "dtype"} & set(b[0])] + [
    (dict(k_out=FAKE), INVALID), (dict(kv_heads=4), INVALID), (dict(head_dim=64, pairs=32), INVALID),
    (dict(dtype=sb.SBVR_BF16), INVALID), (dict(dtype=sb.SBVR_F32), INVALID), (dict(v=None), INVALID), (dict(vt=-8), INVALID),
    (dict(vh=4), INVALID), (dict(slots=None), INVALID), (dict(v=FAKE + 8), ALIGNMENT), (dict(slots=FAKE + 4), ALIGNMENT),
    (dict(c=cache(page_size=15)), INVALID), (dict(c=cache(k=None)), INVALID),
    (dict(c=cache(head_dim=256, k_head_stride=256, v_head_stride=256)), UNSUPPORTED)])
def test_rotary_write_refusals(bad, status):
    assert write(**bad) == status


def test_rotation_strides_in_int64():
    """The check that rows do not overlap holds for the largest strides."""
    wide = dict(q_out_token_stride=1 << 40, q_out_head_stride=1 << 40, T=2 ** 31 - 1, heads=4096)
    assert sb.sbvr_rotary(rotation(**wide)) == INVALID


def beams(ws=FAKE, ws_bytes=1 << 30, **more):
    a = dict(R=2, B=4, V=1000, n=4, n_end=1, dtype=sb.SBVR_F16, logits=FAKE, logits_stride=1000, scores=FAKE,
             end_tokens=FAKE, tokens=FAKE, parents=FAKE, scores_out=FAKE, ended=FAKE, ended_tokens=FAKE)
    a.update(more)
    return sb.sbvr_beam_select(sb.BeamStruct(**a), ws, ws_bytes)


@pytest.mark.parametrize("bad,status", [
    (dict(R=-1), INVALID), (dict(B=0), INVALID), (dict(V=0), INVALID), (dict(n=0), INVALID), (dict(n_end=-1), INVALID),
    (dict(dtype=3), INVALID), (dict(logits_stride=-1), INVALID), (dict(logits=None), INVALID), (dict(scores=None), INVALID),
    (dict(end_tokens=None), INVALID), (dict(tokens=None), INVALID), (dict(parents=None), INVALID),
    (dict(scores_out=None), INVALID), (dict(ended=None), INVALID), (dict(ended_tokens=None), INVALID),
    (dict(B=33), UNSUPPORTED), (dict(n=64), UNSUPPORTED), (dict(n=2 ** 31 - 1, n_end=2 ** 31 - 1), UNSUPPORTED),
    (dict(V=(1 << 30) + 1), UNSUPPORTED), (dict(R=16384), UNSUPPORTED), (dict(R=2 ** 31 - 1), UNSUPPORTED),
    (dict(ws=None), WORKSPACE), (dict(ws_bytes=0), WORKSPACE), (dict(ws_bytes=100), WORKSPACE),
    (dict(logits=FAKE + 1), ALIGNMENT), (dict(logits=FAKE + 2, dtype=sb.SBVR_F32), ALIGNMENT), (dict(ws=FAKE + 8), ALIGNMENT),
    (dict(scores=FAKE + 2), ALIGNMENT), (dict(ended=FAKE + 1), ALIGNMENT)])
def test_beam_refusals(bad, status):
    assert beams(**bad) == status


@pytest.mark.parametrize("B,n", [(4, 3), (4, 5), (1, 2)])
def test_beam_scores_in_place_of_another_width_are_refused(B, n):
    """Request r's new scores lie where another request's old ones are read."""
    outs = dict(zip(("tokens", "parents", "ended", "ended_tokens"), range(FAKE + 4096, FAKE + 5 * 4096, 4096)))
    assert beams(B=B, n=n, **outs) == INVALID
    assert beams(R=1, B=B, n=n, **outs) == INVALID


@pytest.mark.parametrize("R,B,V,n,ends", [(1, 1, 1, 1, 0), (1, 32, 1 << 30, 64, 0), (2047, 32, 1 << 30, 1, 63), (65535, 1, 50000, 8, 2),
                                          (32, 8, 131072, 8, 2)])
def test_beam_workspace(R, B, V, n, ends):
    """Sums and entries of a row's parts, of which a request has at most 4096
    entries: enough is accepted (no HIP call is made for a null logits pointer),
    a byte less is not."""
    need = sb.sbvr_beam_select_workspace_bytes(R, B, V, n, ends)
    assert 0 < need <= R * (B * 4096 * 16 + 4096 * 8)
    assert beams(R=R, B=B, V=V, n=n, n_end=ends, logits_stride=V, ws_bytes=need - 1) == WORKSPACE
    assert beams(R=R, B=B, V=V, n=n, n_end=ends, logits_stride=V, ws_bytes=need, ws=FAKE + 8) == ALIGNMENT


def test_beam_workspace_is_a_requests():
    """The join holds 2816 entries of all beams of a request together, of 8 bytes, each
    part of a row has one of them at least, and a sum of 16 bytes."""
    for R, B, V, n, ends in ((1, 1, 1, 1, 0), (1, 32, 1 << 30, 64, 0), (2047, 32, 1 << 30, 1, 63), (65535, 1, 50000, 8, 2),
                             (32, 8, 131072, 8, 2), (3, 32, 1 << 30, 1, 0), (1, 1, 1 << 30, 1, 0)):
        need, keep = sb.sbvr_beam_select_workspace_bytes(R, B, V, n, ends), n + ends
        parts, rest = divmod(need, R * B * (16 + 8 * keep))
        assert rest == 0 and 1 <= parts and B * parts * keep <= max(2816, B * keep) and need <= R * 2816 * (8 + 16)


def test_workspaces_of_bad_shapes():
    for bad in ((-1, 1, 1, 1, 0), (1, 0, 1, 1, 0), (1, 33, 1, 1, 0), (1, 1, 0, 1, 0), (1, 1, 1, 0, 0), (1, 1, 1, 60, 5)):
        assert sb.sbvr_beam_select_workspace_bytes(*bad) == 0
    for bad in ((-1, 1, 1), (1, 0, 1), (1, 1, 0), (4097, 1, 1), (1, 1, (1 << 22) + 1), (1, (1 << 22) + 1, 1)):
        assert sb.sbvr_page_usage_workspace_bytes(*bad) == 0 and sb.sbvr_page_compact_workspace_bytes(*bad) == 0


def usage(R=4, P=16, pages=100, lens=FAKE, table=FAKE, width=10, stride=10, refs=FAKE, free=FAKE, counts=FAKE, ws=FAKE,
          ws_bytes=1 << 20):
    return sb.sbvr_page_usage(R, P, pages, lens, table, width, stride, refs, free, counts, ws, ws_bytes)


def compact(R=4, P=16, pages=100, lens=FAKE, table=FAKE, width=10, stride=10, out=FAKE + 4096, out_stride=10, src=FAKE,
            dst=FAKE, counts=FAKE, ws=FAKE, ws_bytes=1 << 20):
    return sb.sbvr_page_compact(R, P, pages, lens, table, width, stride, out, out_stride, src, dst, counts, ws, ws_bytes)


BOTH = [(dict(R=-1), INVALID), (dict(P=15), INVALID), (dict(P=8192), INVALID), (dict(pages=0), INVALID), (dict(width=0), INVALID),
        (dict(stride=9), INVALID), (dict(lens=None), INVALID), (dict(table=None), INVALID), (dict(counts=None), INVALID),
        (dict(R=4097), UNSUPPORTED), (dict(pages=(1 << 22) + 1), UNSUPPORTED), (dict(ws=None), WORKSPACE),
        (dict(ws_bytes=8), WORKSPACE), (dict(ws=FAKE + 4), ALIGNMENT), (dict(lens=FAKE + 2), ALIGNMENT),
        (dict(table=FAKE + 1), ALIGNMENT), (dict(counts=FAKE + 2), ALIGNMENT)]


@pytest.mark.parametrize("bad,status", BOTH + [
    (dict(refs=None), INVALID), (dict(free=None), INVALID), (dict(width=(1 << 22) + 1, stride=1 << 23), UNSUPPORTED),
    (dict(refs=FAKE + 2), ALIGNMENT), (dict(free=FAKE + 1), ALIGNMENT)])
def test_usage_refusals(bad, status):
    assert usage(**bad) == status


@pytest.mark.parametrize("bad,status", BOTH + [
    (dict(out=None), INVALID), (dict(out_stride=9), INVALID), (dict(src=None), INVALID), (dict(dst=None), INVALID),
    (dict(out=FAKE, out_stride=12), INVALID), (dict(width=(1 << 22) + 1, stride=1 << 23, out_stride=1 << 23), UNSUPPORTED),
    (dict(out=FAKE + 2), ALIGNMENT), (dict(src=FAKE + 2), ALIGNMENT)])
def test_compact_refusals(bad, status):
    assert compact(**bad) == status


def fork(groups=2, rows_in=4, rows_out=6, P=16, lens=FAKE, table=FAKE, width=10, stride=10, parents=FAKE, free=FAKE, n_free=5,
         taken=FAKE, out=FAKE + 4096, out_stride=10, out_lens=FAKE, src=FAKE, dst=FAKE, tokens=FAKE, used=FAKE):
    return sb.sbvr_page_fork(groups, rows_in, rows_out, P, lens, table, width, stride, parents, free, n_free, taken, out,
                             out_stride, out_lens, src, dst, tokens, used)


@pytest.mark.parametrize("bad,status", [
    (dict(groups=0), INVALID), (dict(groups=3), INVALID), (dict(rows_in=5), INVALID), (dict(rows_out=-2), INVALID),
    (dict(rows_in=-2), INVALID), (dict(n_free=-1), INVALID), (dict(P=24), INVALID), (dict(width=0), INVALID),
    (dict(stride=9), INVALID), (dict(out_stride=9), INVALID), (dict(lens=None), INVALID), (dict(table=None), INVALID),
    (dict(parents=None), INVALID), (dict(free=None), INVALID), (dict(out=None), INVALID), (dict(out=FAKE), INVALID),
    (dict(out_lens=None), INVALID), (dict(src=None), INVALID), (dict(dst=None), INVALID), (dict(tokens=None), INVALID),
    (dict(used=None), INVALID), (dict(rows_in=4098), UNSUPPORTED), (dict(rows_out=4098), UNSUPPORTED),
    (dict(parents=FAKE + 2), ALIGNMENT), (dict(taken=FAKE + 1), ALIGNMENT), (dict(out=FAKE + 2), ALIGNMENT),
    (dict(used=FAKE + 2), ALIGNMENT)])
def test_fork_refusals(bad, status):
    assert fork(**bad) == status


FORK_INPUTS, FORK_OUTPUTS = ("lens", "table", "parents", "free", "taken"), ("out", "out_lens", "src", "dst", "tokens", "used")


@pytest.mark.parametrize("output", FORK_OUTPUTS)
@pytest.mark.parametrize("given", FORK_INPUTS)
def test_fork_in_place_is_refused(given, output):
    """Every workgroup reads the inputs while the first one writes lengths and lists."""
    apart = {name: FAKE + 4096 * i for i, name in enumerate(FORK_INPUTS + FORK_OUTPUTS)}
    assert fork(**{**apart, output: apart[given]}) == INVALID


@pytest.mark.parametrize("caches,more,status", [
    (None, {}, INVALID), ([], {}, INVALID), ([cache()], dict(n=-1), INVALID), ([cache()], dict(src=None), INVALID),
    ([cache()], dict(dst=None), INVALID), ([cache(), cache(n_pages=5)], {}, INVALID),
    ([cache(), cache(v_token_stride=2048)], {}, INVALID), ([cache(), cache(dtype=sb.SBVR_BF16)], {}, INVALID),
    ([cache(), cache(k=None)], {}, INVALID), ([cache(page_size=17)], {}, INVALID), ([cache(k=FAKE + 8)], {}, ALIGNMENT),
    ([cache()], dict(src=FAKE + 2), ALIGNMENT), ([cache()], dict(tokens=FAKE + 1), ALIGNMENT),
    ([cache()], dict(n=0, src=None, dst=None), sb.SBVR_OK)])
def test_copy_refusals(caches, more, status):
    a = {**dict(n=3, src=FAKE, dst=FAKE, tokens=FAKE), **more}
    assert sb.sbvr_page_copy(caches, a["n"], a["src"], a["dst"], a["tokens"]) == status


def test_nothing_to_do():
    """Accepted without a HIP call (there may be no GPU here)."""
    assert sb.sbvr_rotary(rotation(T=0, q=None, k=None, q_out=None, k_out=None, positions=None, frequencies=None)) == sb.SBVR_OK
    assert write(T=0, q=None, k=None, v=None, slots=None) == sb.SBVR_OK
    assert beams(R=0, logits=None, scores=None, ws=None, ws_bytes=0) == sb.SBVR_OK
    assert sb.sbvr_rotary(None) == INVALID and sb.sbvr_beam_select(None, FAKE, 1 << 20) == INVALID
    assert sb.sbvr_rotary_write(None, cache(), FAKE, 1024, 128, FAKE) == INVALID
    assert sb.sbvr_rotary_write(rotation(k_out=None), None, FAKE, 1024, 128, FAKE) == INVALID


def test_structs_match_the_header():
    assert C.sizeof(sb.RotaryStruct) == 9 * 4 + 4 + 12 * 8 + 4 * 8
    assert C.sizeof(sb.BeamStruct) == 6 * 4 + 9 * 8


# ---------------------------------------------------------------------------
# the tensor helpers
# ---------------------------------------------------------------------------

@pytest.fixture
def calls():
    """As the step operators' binding is tested: the library's functions note
    what they are called with."""
    noted, kept, address = Calls(), [], {}
    structs = {"sbvr_rotary": sb.RotaryStruct, "sbvr_rotary_write": sb.RotaryStruct, "sbvr_beam_select": sb.BeamStruct}
    for name in step.FUNCTIONS:
        real = getattr(sb._lib, name)

        def note(*args, name=name):
            if name.endswith("_workspace_bytes"):
                return 64
            if name in structs:
                args = (structs[name].from_buffer_copy(C.string_at(args[0], C.sizeof(structs[name]))), *args[1:])
            if name == "sbvr_page_copy":
                args = ([sb.CacheStruct.from_buffer_copy(C.string_at(args[0] + i * C.sizeof(sb.CacheStruct), C.sizeof(sb.CacheStruct)))
                         for i in range(args[1])], *args[2:])
            noted.append((name, args))
            noted.seen.append(noted.device[0])
            return noted.status
        kept.append(C.CFUNCTYPE(real.restype, *real.argtypes)(note))
        address[name] = C.cast(kept[-1], C.c_void_p).value
    step._native.connect(address, sb.SBVRError, lambda index: 0, noted.exchange)
    yield noted
    step._connect()


def half(*shape, device="cuda:0", **more):
    return Shell(*shape, dtype=torch.float16, device=device, **more)


def f32(*shape, device="cuda:0"):
    return Shell(*shape, dtype=torch.float32, device=device)


def rotary(device="cuda:0", positions=None, q=None, **more):
    q = half(4, 8, 64, device=device) if q is None else q
    return sb.rotary(q, half(4, 2, 64, device=device), Shell(4, device=device) if positions is None else positions,
                     f32(32, device=device), q_out=half(4, 8, 64, device=device), k_out=half(4, 2, 64, device=device), **more)


def rotary_write(device="cuda:0"):
    kv = sb.KVCache(half(5, 16, 2, 64, device=device), half(5, 16, 2, 64, device=device))
    k = half(4, 2, 64, device=device)
    return sb.rotary_write(half(4, 8, 64, device=device), kv, k, k, Shell(4, dtype=torch.int64, device=device),
                           Shell(4, device=device), f32(32, device=device), q_out=half(4, 8, 64, device=device))


def select(device="cuda:0", n=None):
    N = n or 4
    out = sb.BeamChoice(Shell(2, N, device=device), Shell(2, N, device=device), f32(2, N, device=device),
                        f32(2, 4, device=device), Shell(2, 4, device=device))
    return sb.beam_select(half(8, 100, device=device), f32(2, 4, device=device), n=n, out=out,
                          workspace=Shell(64, dtype=torch.uint8, device=device))


def table_calls(device="cuda:0", stride=10):
    lens, table = Shell(3, device=device), Shell(3, 10, stride=(stride, 1), device=device)
    ws = Shell(64, dtype=torch.uint8, device=device)

    def ints(*sizes):
        return [Shell(*s, device=device) for s in sizes]
    sb.page_usage(lens, table, 16, 50, out=sb.PageUsage(*ints((50,), (50,), (2,))), workspace=ws)
    out = sb.PageCompaction(Shell(3, 10, stride=(stride, 1), device=device), *ints((25,), (25,), (2,)))
    sb.page_compact(lens, table, 16, 50, out=out, workspace=ws)
    out = sb.PageFork(Shell(3, 10, stride=(stride, 1), device=device), *ints((3,), (3,), (3,), (3,), (1,)))
    sb.page_fork(lens, table, Shell(1, 3, device=device), 16, Shell(9, device=device), out=out)


def copy(device="cuda:0", more=()):
    kv = half(5, 16, 2, 64, device=device)
    sb.page_copy([sb.KVCache(kv, kv), *more], Shell(3, device=device), Shell(3, device=device))


@pytest.mark.parametrize("call,names", [
    (rotary, ["rotary"]), (rotary_write, ["rotary_write"]), (select, ["beam_select"]), (copy, ["page_copy"]),
    (table_calls, ["page_usage", "page_compact", "page_fork"])])
def test_a_call_is_made_on_its_tensors_device(calls, call, names):
    for device in (1, 0, 3):
        call(f"cuda:{device}")
        assert [c[0] for c in calls] == ["sbvr_" + n for n in names]
        assert set(calls.seen) == {device} and calls.device == [0]
        calls.clear()
        calls.seen.clear()
    calls.status = -1
    with pytest.raises(sb.SBVRError):
        call("cuda:2")
    assert calls.device == [0]


@pytest.mark.parametrize("stride", [10, 64, 0, 1, 9])
def test_row_strides_are_the_tensors_own(calls, stride):
    """An expanded table or rows that overlap must not be taken for whole rows."""
    table_calls(stride=stride)
    u, c, f = [a for _, a in calls]
    assert (u[6], c[6], c[8], f[7], f[13]) == (stride,) * 5


@pytest.mark.parametrize("stride", [8, 4, 0, 1])
def test_position_strides_are_the_tensors_own(calls, stride):
    rotary(positions=Shell(2, 4, stride=(stride, 1)))
    rotary(positions=Shell(1, 4, stride=(stride, 1)))
    two, one = (a[0] for _, a in calls)
    assert two.axes == 2 and two.position_stride == stride and one.axes == 1 and one.position_stride >= 4


def test_what_reaches_the_library(calls):
    rotary(q=half(4, 8, 64, stride=(2048, 64, 1)), interleaved=True, inverse=True)
    select(n=3)
    a, b = (x[0] for _, x in calls)
    assert (a.T, a.heads, a.kv_heads, a.head_dim, a.pairs, a.interleaved, a.inverse) == (4, 8, 2, 64, 32, 1, 1)
    assert (a.q_token_stride, a.q_head_stride, a.q_out_token_stride, a.k_out_token_stride) == (2048, 64, 512, 128)
    assert (b.R, b.B, b.V, b.n, b.n_end, b.logits_stride) == (2, 4, 100, 3, 0, 100)
    calls.clear()
    kv = half(5, 16, 2, 64, stride=(4096, 64, 1024, 1))
    copy(more=[sb.KVCache(kv, kv)])
    caches, n = calls[0][1][:2]
    assert n == 3 and [c.k_token_stride for c in caches] == [128, 64] and [c.v_head_stride for c in caches] == [64, 1024]


def test_tensors_on_several_devices_are_refused(calls):
    one = half(5, 16, 2, 64, device="cuda:1")
    for call in (lambda: copy(more=[sb.KVCache(one, one)]), lambda: rotary(positions=Shell(4, device="cuda:1")),
                 lambda: rotary(q=half(4, 8, 64, device="cuda:1"))):
        with pytest.raises(AssertionError):
            call()
    assert not calls and calls.device == [0]


def test_tensor_helpers_refuse_before_any_launch():
    x, i = torch.zeros(2, 2, 64, dtype=torch.float16), torch.zeros(2, dtype=torch.int32)
    kv = torch.zeros(2, 16, 2, 64, dtype=torch.float16)
    for call in (lambda: sb.rotary(x, x, i, torch.zeros(32)), lambda: sb.beam_select(x[0], torch.zeros(1, 2)),
                 lambda: sb.rotary_write(x, sb.KVCache(kv, kv), x, x, i.long(), i, torch.zeros(32)),
                 lambda: sb.page_usage(i, i.view(2, 1), 16, 4), lambda: sb.page_compact(i, i.view(2, 1), 16, 4),
                 lambda: sb.page_fork(i, i.view(2, 1), i.view(1, 2), 16, i), lambda: sb.page_copy(sb.KVCache(kv, kv), i, i)):
        with pytest.raises(AssertionError, match="GPU"):
            call()
