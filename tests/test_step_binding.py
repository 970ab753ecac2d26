"""What the native tensor helpers of a step's operators hand to the library,
without a GPU: the library's functions are replaced by ones that note their
arguments, and the tensors have a GPU's device, sizes and strides but no memory."""
import ctypes as C

import pytest
import torch

import paper_2509_18172_amd as sb
from paper_2509_18172_amd import step


class Shell(torch.Tensor):
    """A tensor of a GPU without memory."""
    @staticmethod
    def __new__(cls, *shape, dtype=torch.int32, stride=None, device="cuda:0"):
        if stride is None:
            stride = [1]
            for n in reversed(shape[1:]):
                stride.insert(0, stride[0] * n)
        return torch.Tensor._make_wrapper_subclass(cls, shape, strides=stride, dtype=dtype, device=device)

    @classmethod
    def __torch_dispatch__(cls, func, types, args=(), kwargs=None):
        raise AssertionError(f"{func} on a tensor without memory")


NAMES = ("sbvr_batch_plan", "sbvr_cache_write", "sbvr_tree_attention_workspace_bytes", "sbvr_tree_attention",
         "sbvr_residual_norm", "sbvr_adjust_logits")


@pytest.fixture
def calls():
    """The list of calls (name, arguments) that reach the library."""
    noted, kept, address = [], [], {}
    for name in NAMES:
        real = getattr(sb._lib, name)

        def note(*args, name=name):
            if name == "sbvr_adjust_logits":
                args = (sb.LogitsStruct.from_buffer_copy(C.string_at(args[0], C.sizeof(sb.LogitsStruct))), *args[1:])
            if name != "sbvr_tree_attention_workspace_bytes":
                noted.append((name, args))
            return 0
        kept.append(C.CFUNCTYPE(real.restype, *real.argtypes)(note))
        address[name] = C.cast(kept[-1], C.c_void_p).value
    step._native.connect(address, sb.SBVRError, lambda index: 0)
    yield noted
    real = {name: C.cast(getattr(sb._lib, name), C.c_void_p).value for name in NAMES}
    step._native.connect(real, sb.SBVRError, getattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0))


def plan(R=3, T=4, table=None, device="cuda:0", **more):
    def i32(*shape):
        return Shell(*shape, device=device)

    def i64(*shape):
        return Shell(*shape, dtype=torch.int64, device=device)
    out = sb.BatchPlan(i32(R + 1), i32(T), i32(T), i64(T), i64(T), i32(2))
    return sb.batch_plan(i32(R), i32(R), i32(9), i32(R, 10) if table is None else table, 16, T, out=out, **more)


def attend(R=3, T=4, table=None, device="cuda:0", **more):
    def half(*shape):
        return Shell(*shape, dtype=torch.float16, device=device)
    cache = sb.KVCache(half(5, 16, 2, 64), half(5, 16, 2, 64))
    return sb.tree_attention(half(T, 4, 64), cache, Shell(R, 10, device=device) if table is None else table,
                             Shell(R, device=device), Shell(R + 1, device=device),
                             Shell(T, dtype=torch.int64, device=device), 1, out=half(T, 4, 64), **more)


def adjust(T=3, V=100, grammar=None, device="cuda:0", **more):
    def half(*shape):
        return Shell(*shape, dtype=torch.float16, device=device)
    return sb.adjust_logits(half(T, V), grammar=grammar, out=half(T, V), **more)


# (stride of a table of rows 10 wide, what the library has to be told)
STRIDES = [(10, 10), (64, 64), (0, 0), (1, 1), (9, 9)]


@pytest.mark.parametrize("stride,told", STRIDES)
def test_row_strides_are_the_tensors_own(calls, stride, told):
    """An expanded page table or grammar (stride 0), or rows that overlap, must
    not be taken for whole rows: the library refuses such strides."""
    plan(table=Shell(3, 10, stride=(stride, 1)))
    attend(table=Shell(3, 10, stride=(stride, 1)))
    adjust(V=320, grammar=Shell(3, 10, stride=(stride, 1)))
    (_, a), (_, b), (_, c) = calls
    assert (a[10], b[9], c[0].grammar_stride) == (told, told, told)


@pytest.mark.parametrize("stride", [0, 1, 9, 10, 64])
def test_a_single_rows_stride_means_nothing(calls, stride):
    plan(R=1, table=Shell(1, 10, stride=(stride, 1)))
    attend(R=1, table=Shell(1, 10, stride=(stride, 1)))
    adjust(V=320, grammar=Shell(1, 10, stride=(stride, 1)))
    (_, a), (_, b), (_, c) = calls
    assert min(a[10], b[9], c[0].grammar_stride) >= 10
