"""Refusals of the operators between the products of a step, on the host: a bad
argument returns its status before any HIP call, so the pointers here are
never dereferenced."""
import pytest

import paper_2509_18172_amd as sb

FAKE = 1 << 20  # 16-byte-aligned
INVALID, UNSUPPORTED, WORKSPACE, ALIGNMENT = (sb.SBVR_E_INVALID_ARG, sb.SBVR_E_UNSUPPORTED, sb.SBVR_E_WORKSPACE,
                                              sb.SBVR_E_ALIGNMENT)


def plan(R=4, T=8, P=16, ctx=FAKE, new=FAKE, free=FAKE, n_free=9, parents=FAKE, table=FAKE, pages=10, stride=10,
         start=FAKE, request=FAKE, pos=FAKE, slots=FAKE, mask=FAKE, used=FAKE):
    return sb.sbvr_batch_plan(R, T, P, ctx, new, free, n_free, parents, table, pages, stride, start, request, pos, slots,
                              mask, used)


@pytest.mark.parametrize("bad,status", [
    (dict(R=0), INVALID), (dict(T=-1), INVALID), (dict(n_free=-1), INVALID), (dict(pages=0, stride=0), INVALID),
    (dict(stride=9), INVALID), (dict(P=15), INVALID), (dict(P=8), INVALID), (dict(P=24), INVALID), (dict(P=8192), INVALID),
    (dict(P=0), INVALID), (dict(P=-16), INVALID), (dict(ctx=None), INVALID), (dict(new=None), INVALID),
    (dict(free=None), INVALID), (dict(table=None), INVALID), (dict(start=None), INVALID), (dict(used=None), INVALID),
    (dict(request=None), INVALID), (dict(pos=None), INVALID), (dict(slots=None), INVALID), (dict(mask=None), INVALID),
    (dict(R=4097), UNSUPPORTED), (dict(ctx=FAKE + 2), ALIGNMENT), (dict(parents=FAKE + 1), ALIGNMENT),
    (dict(slots=FAKE + 4), ALIGNMENT), (dict(mask=FAKE + 4), ALIGNMENT), (dict(table=FAKE + 2), ALIGNMENT)])
def test_plan_refusals(bad, status):
    assert plan(**bad) == status


def cache(**more):
    c = dict(k=FAKE, v=FAKE, k_page_stride=16384, k_token_stride=1024, k_head_stride=128, v_page_stride=16384,
             v_token_stride=1024, v_head_stride=128, n_pages=4, page_size=16, kv_heads=8, head_dim=128,
             dtype=sb.SBVR_F16)
    c.update(more)
    return sb.CacheStruct(**c)


CACHES = [
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(n_pages=0), INVALID), (dict(kv_heads=0), INVALID),
    (dict(head_dim=0), INVALID), (dict(head_dim=100), INVALID), (dict(dtype=sb.SBVR_F32), INVALID),
    (dict(dtype=7), INVALID), (dict(page_size=48), INVALID), (dict(page_size=8), INVALID),
    (dict(k_page_stride=-8), INVALID), (dict(v_token_stride=1020), INVALID), (dict(k_head_stride=4), INVALID),
    (dict(v_page_stride=1 << 41), INVALID), (dict(head_dim=136), UNSUPPORTED), (dict(head_dim=256), UNSUPPORTED),
    (dict(kv_heads=5000), UNSUPPORTED), (dict(k_token_stride=1 << 28), UNSUPPORTED),
    (dict(k=FAKE + 8), ALIGNMENT), (dict(v=FAKE + 2), ALIGNMENT)]


def write(c=None, T=4, k=FAKE, kt=1024, kh=128, v=FAKE, vt=1024, vh=128, slots=FAKE):
    return sb.sbvr_cache_write(cache() if c is None else c, T, k, kt, kh, v, vt, vh, slots)


@pytest.mark.parametrize("bad,status", CACHES)
def test_cache_refusals(bad, status):
    assert write(cache(**bad)) == status
    assert attention(cache(**bad)) == status


@pytest.mark.parametrize("bad,status", [
    (dict(T=-1), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(slots=None), INVALID),
    (dict(kt=-8), INVALID), (dict(kh=100), INVALID), (dict(vt=1 << 41), INVALID), (dict(vh=1), INVALID),
    (dict(k=FAKE + 8), ALIGNMENT), (dict(v=FAKE + 4), ALIGNMENT), (dict(slots=FAKE + 4), ALIGNMENT)])
def test_write_refusals(bad, status):
    assert write(**bad) == status


def test_write_of_no_cache():
    assert sb.sbvr_cache_write(None, 1, FAKE, 8, 8, FAKE, 8, 8, FAKE) == INVALID


def attention(c=None, R=2, T=8, heads=32, q=FAKE, qt=4096, qh=128, table=FAKE, pages=20, stride=20, ctx=FAKE, start=FAKE,
              mask=FAKE, max_new=4, scale=0.1, out=FAKE, ws=FAKE, ws_bytes=1 << 30):
    return sb.sbvr_tree_attention(cache() if c is None else c, R, T, heads, q, qt, qh, table, pages, stride, ctx, start,
                                  mask, max_new, scale, out, ws, ws_bytes)


@pytest.mark.parametrize("bad,status", [
    (dict(R=0), INVALID), (dict(T=-1), INVALID), (dict(heads=0), INVALID), (dict(heads=4), INVALID),
    (dict(heads=30), INVALID), (dict(max_new=0), INVALID), (dict(max_new=65), INVALID), (dict(pages=0), INVALID),
    (dict(stride=19), INVALID), (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID),
    (dict(qt=-8), INVALID), (dict(qh=12), INVALID), (dict(q=None), INVALID), (dict(table=None), INVALID),
    (dict(ctx=None), INVALID), (dict(start=None), INVALID), (dict(mask=None), INVALID), (dict(out=None), INVALID),
    (dict(R=4097), UNSUPPORTED), (dict(heads=8192), UNSUPPORTED), (dict(ws=None), WORKSPACE), (dict(ws_bytes=100), WORKSPACE),
    (dict(q=FAKE + 8), ALIGNMENT), (dict(out=FAKE + 8), ALIGNMENT), (dict(mask=FAKE + 4), ALIGNMENT),
    (dict(table=FAKE + 2), ALIGNMENT), (dict(ws=FAKE + 8), ALIGNMENT),
    (dict(R=4096, pages=1 << 24, stride=1 << 24), UNSUPPORTED)])
def test_attention_refusals(bad, status):
    assert attention(**bad) == status


def test_attention_workspace_query():
    f = sb.sbvr_tree_attention_workspace_bytes
    small, large = f(1, 1, 32, 8, 128), f(1, 64, 64, 8, 128)
    assert 0 < small < large and small % 16 == 0 and large % 16 == 0
    assert f(4096, 64, 64, 8, 128) == large  # the split is over workgroups, not requests
    for bad in [(0, 1, 32, 8, 128), (1, 0, 32, 8, 128), (1, 65, 32, 8, 128), (1, 1, 30, 8, 128), (1, 1, 32, 0, 128),
                (1, 1, 32, 8, 100), (1, 1, 32, 8, 256), (5000, 1, 32, 8, 128)]:
        assert f(*bad) == 0, bad


def norm(T=2, H=64, dtype=sb.SBVR_F16, xt=sb.SBVR_F32, x=FAKE, xs=64, y=FAKE, ys=64, post=FAKE, gate=None, gs=0, scale=1.0,
         pre=FAKE, eps=1e-5, xo=FAKE, xos=64, h=FAKE, hs=64):
    return sb.sbvr_residual_norm(T, H, dtype, xt, x, xs, y, ys, post, gate, gs, scale, pre, eps, xo, xos, h, hs)


@pytest.mark.parametrize("bad,status", [
    (dict(T=-1), INVALID), (dict(H=0), INVALID), (dict(dtype=sb.SBVR_F32), INVALID), (dict(xt=sb.SBVR_BF16), INVALID),
    (dict(xt=5), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(scale=float("inf")), INVALID),
    (dict(xs=-1), INVALID), (dict(ys=-1), INVALID), (dict(xos=63), INVALID), (dict(hs=63), INVALID), (dict(x=None), INVALID),
    (dict(xo=None, h=None), INVALID), (dict(pre=None), INVALID), (dict(gate=FAKE, gs=-64), INVALID),
    (dict(H=32769, xs=40000, ys=40000, xos=40000, hs=40000), UNSUPPORTED), (dict(x=FAKE + 2), ALIGNMENT),
    (dict(y=FAKE + 1), ALIGNMENT), (dict(h=FAKE + 1), ALIGNMENT), (dict(xo=FAKE + 2), ALIGNMENT)])
def test_norm_refusals(bad, status):
    assert norm(**bad) == status


def logits(**more):
    a = dict(R=2, T=4, V=100, dtype=sb.SBVR_F16, out_dtype=sb.SBVR_F32, logits=FAKE, logits_stride=100, out=FAKE,
             out_stride=100, token_request=FAKE)
    a.update(more)
    return sb.sbvr_adjust_logits(sb.LogitsStruct(**a))


@pytest.mark.parametrize("bad,status", [
    (dict(R=0), INVALID), (dict(T=-1), INVALID), (dict(V=0), INVALID), (dict(dtype=3), INVALID), (dict(dtype=-1), INVALID),
    (dict(out_dtype=sb.SBVR_BF16), INVALID), (dict(dtype=sb.SBVR_F32, out_dtype=sb.SBVR_F16), INVALID),
    (dict(logits_stride=-1), INVALID), (dict(out_stride=99), INVALID), (dict(logits=None), INVALID), (dict(out=None), INVALID),
    (dict(history=FAKE), INVALID), (dict(bias_tokens=FAKE), INVALID), (dict(bias_tokens=FAKE, bias_start=FAKE), INVALID),
    (dict(grammar=FAKE, grammar_stride=4, grammar_count=0), INVALID), (dict(grammar=FAKE, grammar_stride=3, grammar_count=1), INVALID),
    (dict(draft_tokens=FAKE), INVALID), (dict(draft_tokens=FAKE, tree_mask=FAKE), INVALID), (dict(query_start=FAKE), INVALID),
    (dict(T=65536), UNSUPPORTED), (dict(V=(1 << 30) + 1, out_stride=1 << 31), UNSUPPORTED),
    (dict(logits=FAKE + 1), ALIGNMENT), (dict(out=FAKE + 2), ALIGNMENT), (dict(repetition=FAKE + 2), ALIGNMENT),
    (dict(draft_tokens=FAKE, query_start=FAKE, tree_mask=FAKE + 4), ALIGNMENT)])
def test_logits_refusals(bad, status):
    assert logits(**bad) == status


def test_logits_of_nothing():
    assert sb.sbvr_adjust_logits(None) == INVALID


def test_no_tokens_is_a_step():
    """Zero tokens: accepted without a HIP call (there may be no GPU here)."""
    assert write(T=0, k=None, v=None, slots=None) == sb.SBVR_OK
    assert attention(T=0, q=None, out=None, ws=None, ws_bytes=0) == sb.SBVR_OK
    assert norm(T=0, x=None, y=None, xo=None, h=None) == sb.SBVR_OK
    assert logits(T=0, logits=None, out=None) == sb.SBVR_OK


def test_structs_match_the_header():
    """The binding's structs have the C structs' sizes (checked by layout: the
    fields in order, naturally aligned)."""
    import ctypes as C
    assert C.sizeof(sb.CacheStruct) == 8 * 8 + 5 * 4 + 4
    assert C.sizeof(sb.LogitsStruct) == 5 * 4 + 4 + 4 * 8 + 12 * 8 + 8 + 8 + 4 + 4 + 3 * 8


def test_tensor_helpers_refuse_before_any_launch():
    """The native helpers load here too, and say what is wrong with tensors
    that are not theirs (these are on the CPU)."""
    torch = pytest.importorskip("torch")
    x = torch.zeros(2, 64, dtype=torch.float16)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(AssertionError, match="GPU"):
        sb.residual_norm(x, x)
    with pytest.raises(AssertionError, match="GPU"):
        sb.adjust_logits(x)
    with pytest.raises(AssertionError, match="GPU"):
        sb.batch_plan(i, i, i, i.view(2, 1), 16, 2)
    kv = torch.zeros(2, 16, 2, 64, dtype=torch.float16)
    with pytest.raises(AssertionError, match="GPU"):
        sb.cache_write(sb.KVCache(kv, kv), x.view(2, 1, 64), x.view(2, 1, 64), i.long())
    with pytest.raises(AssertionError, match="GPU"):
        sb.tree_attention(x.view(2, 1, 64), sb.KVCache(kv, kv), i.view(2, 1), i, i, i.long(), max_new=1)


@pytest.mark.parametrize("bad,status", [
    (dict(R=0), INVALID), (dict(max_new=65), INVALID), (dict(heads=30), INVALID), (dict(stride=19), INVALID),
    (dict(q=None), INVALID), (dict(out=None), INVALID), (dict(R=4097), UNSUPPORTED), (dict(ws_bytes=100), WORKSPACE),
    (dict(out=FAKE + 8), ALIGNMENT), (dict(T=0, q=None, out=None, ws=None, ws_bytes=0), sb.SBVR_OK)])
def test_whole_attention_refuses_alike(bad, status):
    a = dict(R=2, T=8, heads=32, q=FAKE, qt=4096, qh=128, table=FAKE, pages=20, stride=20, ctx=FAKE, start=FAKE, mask=FAKE,
             max_new=4, scale=0.1, out=FAKE, ws=FAKE, ws_bytes=1 << 30)
    assert sb.sbvr_tree_attention_whole(cache(), *{**a, **bad}.values()) == status
    assert attention(**bad) == status
    assert sb.sbvr_tree_attention_whole(None, *a.values()) == INVALID


def test_logits_of_no_rows_need_no_lists():
    """An empty tensor has no address: which of the lists are there says nothing
    where there are no rows.  What is wrong at any size is refused all the same."""
    none = dict(T=0, logits=None, out=None, token_request=None)
    for given in (dict(query_start=FAKE), dict(draft_tokens=FAKE), dict(tree_mask=FAKE, query_start=FAKE),
                  dict(history=FAKE), dict(history_start=FAKE), dict(bias_tokens=FAKE), dict(bias_start=FAKE),
                  dict(grammar=FAKE, grammar_stride=4, grammar_count=0), dict(grammar=FAKE, grammar_stride=0, grammar_count=0)):
        assert logits(**none, **given) == sb.SBVR_OK, given
    for bad in (dict(R=0), dict(V=0), dict(dtype=3), dict(out_dtype=sb.SBVR_BF16), dict(logits_stride=-1)):
        assert logits(**{**none, **bad}) == INVALID, bad
    assert logits(**none, V=(1 << 30) + 1) == UNSUPPORTED


def test_norm_in_place_needs_one_stride():
    """x_out may be x where each row lies on itself; with other strides rows
    would be written that are still to be read."""
    assert norm(xs=64, xos=128) == INVALID and norm(xs=128, xos=64) == INVALID
    assert norm(xs=0, xos=64) == INVALID


def test_logits_in_place_need_one_type_and_stride():
    """out may be logits where each element lies on itself."""
    assert logits() == INVALID  # (binary16 to binary32)
    same = dict(out_dtype=sb.SBVR_F16)
    assert logits(**same, out_stride=128) == INVALID and logits(**same, logits_stride=0) == INVALID
