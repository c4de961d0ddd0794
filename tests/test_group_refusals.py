"""What the entry points of the 4-bit layers refuse, found on the host before anything is queued, and the binding's own checks."""
import ctypes as C
import os
import re

import pytest
import torch

from paper_2311_15806_b200 import binding as B
from paper_2311_15806_b200 import build as pipe_build
from tests import group_reference as R

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
GROUP = os.path.join(ROOT, "paper_2311_15806_b200", "csrc", "group")


@pytest.fixture(scope="module")
def lib():
    pipe_build.build()
    return B.lib()


def desc(**k):
    a = dict(O=64, I=128, g=32, dtype=torch.bfloat16, asymmetric=False, experts=1)
    a.update(k)
    return B.make_group_desc(a["O"], a["I"], a["g"], dtype=a["dtype"], asymmetric=a["asymmetric"], experts=a["experts"])


def test_layout_sizes(lib):
    lay = B.pipe_group_layout(desc(O=70, I=384, g=128, experts=3, asymmetric=True))
    assert (lay.groups, lay.codes_bytes, lay.scales_bytes, lay.zeros_bytes) == (3, 3 * 70 * 192, 3 * 3 * 70 * 2, 3 * 3 * 70)
    assert B.pipe_group_layout(desc()).zeros_bytes == 0
    big = B.pipe_group_layout(desc(O=1 << 20, I=1 << 14, experts=64))     # sizes beyond 32 bits
    assert big.codes_bytes == 64 << 33
    codes, scales, zeros = B.alloc_group(desc(O=5, I=64, asymmetric=True, experts=2), device="cpu")
    assert codes.shape == (2, 2, 5, 16) and scales.shape == (2, 2, 5) and zeros.shape == (2, 2, 5)


@pytest.mark.parametrize("field,value,status", [
    ("experts", 0, B.PIPE_ERR_INVALID_ARG), ("experts", B.MAX_EXPERTS + 1, B.PIPE_ERR_INVALID_ARG), ("out_features", 0, B.PIPE_ERR_INVALID_ARG),
    ("out_features", (1 << 29) + 1, B.PIPE_ERR_INVALID_ARG), ("in_features", (1 << 29) + 32, B.PIPE_ERR_INVALID_ARG),
    ("in_features", 0, B.PIPE_ERR_INVALID_ARG), ("in_features", -32, B.PIPE_ERR_INVALID_ARG), ("in_features", 144, B.PIPE_ERR_SHAPE),
    ("group_size", 0, B.PIPE_ERR_INVALID_ARG), ("group_size", 16, B.PIPE_ERR_UNSUPPORTED), ("group_size", 256, B.PIPE_ERR_UNSUPPORTED),
    ("dtype", 2, B.PIPE_ERR_INVALID_ARG), ("dtype", -1, B.PIPE_ERR_INVALID_ARG), ("asymmetric", 2, B.PIPE_ERR_INVALID_ARG)])
def test_bad_descriptors(lib, field, value, status):
    d = desc()
    setattr(d, field, value)
    out = B.GroupLayout()
    assert lib.pipe_group_layout(C.byref(d), C.byref(out)) == status
    assert lib.pipe_group_quantize(C.byref(d), 4096, 2, 4096, 4096, 4096, None, None, 0, None) == status
    assert lib.pipe_group_linear(C.byref(d), 4096, 4096, None, 4096, 1, 4096, None, 0, 4096, 4096, None) == status
    assert lib.pipe_expert_linear(C.byref(d), 4096, 4096, None, 4096, 1, 4096, None, 4096, 1, None, 0, 4096, 4096, None) == status


def test_null_descriptors(lib):
    assert lib.pipe_group_layout(None, C.byref(B.GroupLayout())) == B.PIPE_ERR_INVALID_ARG
    assert lib.pipe_group_layout(C.byref(desc()), None) == B.PIPE_ERR_INVALID_ARG
    assert lib.pipe_group_linear(None, 4096, 4096, None, 4096, 1, 128, None, 0, 4096, 64, None) == B.PIPE_ERR_INVALID_ARG


@pytest.mark.parametrize("change,status", [
    (dict(w=None), B.PIPE_ERR_INVALID_ARG), (dict(codes=None), B.PIPE_ERR_INVALID_ARG), (dict(scales=None), B.PIPE_ERR_INVALID_ARG),
    (dict(zeros=4096), B.PIPE_ERR_INVALID_ARG), (dict(wt=3), B.PIPE_ERR_INVALID_ARG), (dict(wt=-1), B.PIPE_ERR_INVALID_ARG),
    (dict(ldw=127), B.PIPE_ERR_INVALID_ARG), (dict(values=4096, ldv=127), B.PIPE_ERR_INVALID_ARG), (dict(w=4098), B.PIPE_ERR_ALIGNMENT),
    (dict(codes=4104), B.PIPE_ERR_ALIGNMENT), (dict(scales=4097), B.PIPE_ERR_ALIGNMENT), (dict(values=4098, ldv=128), B.PIPE_ERR_ALIGNMENT)])
def test_quantize_refuses(lib, change, status):
    a = dict(w=4096, wt=2, ldw=128, codes=4096, scales=4096, zeros=None, values=None, ldv=0)
    a.update(change)
    assert lib.pipe_group_quantize(C.byref(desc()), a["w"], a["wt"], a["ldw"], a["codes"], a["scales"], a["zeros"], a["values"], a["ldv"], None) == status
    if "zeros" not in change:
        assert lib.pipe_group_quantize(C.byref(desc(asymmetric=True)), a["w"], a["wt"], a["ldw"], a["codes"], a["scales"], None, a["values"], a["ldv"], None) == \
            B.PIPE_ERR_INVALID_ARG


BAD_PRODUCTS = [
    (dict(codes=None), B.PIPE_ERR_INVALID_ARG), (dict(scales=None), B.PIPE_ERR_INVALID_ARG), (dict(zeros=4096), B.PIPE_ERR_INVALID_ARG),
    (dict(x=None), B.PIPE_ERR_INVALID_ARG), (dict(y=None), B.PIPE_ERR_INVALID_ARG), (dict(T=-1), B.PIPE_ERR_INVALID_ARG),
    (dict(T=1 << 31), B.PIPE_ERR_INVALID_ARG), (dict(T=(1 << 30) + 1), B.PIPE_ERR_INVALID_ARG), (dict(act=5), B.PIPE_ERR_INVALID_ARG), (dict(act=-1), B.PIPE_ERR_INVALID_ARG),
    (dict(ldx=120), B.PIPE_ERR_INVALID_ARG), (dict(ldy=63), B.PIPE_ERR_INVALID_ARG), (dict(ldx=132), B.PIPE_ERR_ALIGNMENT),
    (dict(x=4104), B.PIPE_ERR_ALIGNMENT), (dict(codes=4104), B.PIPE_ERR_ALIGNMENT), (dict(scales=4097), B.PIPE_ERR_ALIGNMENT),
    (dict(bias=4097), B.PIPE_ERR_ALIGNMENT), (dict(y=4097), B.PIPE_ERR_ALIGNMENT)]


@pytest.mark.parametrize("change,status", BAD_PRODUCTS)
def test_linear_refuses(lib, change, status):
    a = dict(codes=4096, scales=4096, zeros=None, x=4096, T=2, ldx=128, bias=None, act=0, y=4096, ldy=64)
    a.update(change)
    assert lib.pipe_group_linear(C.byref(desc()), a["codes"], a["scales"], a["zeros"], a["x"], a["T"], a["ldx"], a["bias"], a["act"], a["y"], a["ldy"], None) == status


@pytest.mark.parametrize("change,status", BAD_PRODUCTS + [
    (dict(offsets=None), B.PIPE_ERR_INVALID_ARG), (dict(N=-1), B.PIPE_ERR_INVALID_ARG), (dict(N=1 << 31), B.PIPE_ERR_INVALID_ARG),
    (dict(offsets=4098), B.PIPE_ERR_ALIGNMENT), (dict(rows=4098), B.PIPE_ERR_ALIGNMENT)])
def test_expert_linear_refuses(lib, change, status):
    a = dict(codes=4096, scales=4096, zeros=None, x=4096, T=2, ldx=128, rows=None, offsets=4096, N=2, bias=None, act=0, y=4096, ldy=64)
    a.update(change)
    assert lib.pipe_expert_linear(C.byref(desc(experts=3)), a["codes"], a["scales"], a["zeros"], a["x"], a["T"], a["ldx"], a["rows"], a["offsets"], a["N"],
                                  a["bias"], a["act"], a["y"], a["ldy"], None) == status


def test_linear_is_for_one_expert_and_no_rows_are_no_work(lib):
    assert lib.pipe_group_linear(C.byref(desc(experts=2)), 4096, 4096, None, 4096, 1, 128, None, 0, 4096, 64, None) == B.PIPE_ERR_SHAPE
    assert lib.pipe_group_linear(C.byref(desc()), 4096, 4096, None, None, 0, 128, None, 0, None, 64, None) == B.PIPE_OK
    assert lib.pipe_expert_linear(C.byref(desc(experts=2)), 4096, 4096, None, None, 0, 128, None, 4096, 0, None, 0, None, 64, None) == B.PIPE_OK
    assert lib.pipe_expert_combine(None, 0, 64, None, None, 0, 2, 64, 0, None, 64, None) == B.PIPE_OK


@pytest.mark.parametrize("change,status", [
    (dict(T=-1), B.PIPE_ERR_INVALID_ARG), (dict(k=0), B.PIPE_ERR_INVALID_ARG), (dict(E=0), B.PIPE_ERR_INVALID_ARG),
    (dict(E=B.MAX_EXPERTS + 1), B.PIPE_ERR_INVALID_ARG), (dict(T=1 << 30, k=2), B.PIPE_ERR_UNSUPPORTED), (dict(choice=None), B.PIPE_ERR_INVALID_ARG),
    (dict(offsets=None), B.PIPE_ERR_INVALID_ARG), (dict(rows=None), B.PIPE_ERR_INVALID_ARG), (dict(slots=None), B.PIPE_ERR_INVALID_ARG),
    (dict(choice=4097), B.PIPE_ERR_ALIGNMENT), (dict(slots=4098), B.PIPE_ERR_ALIGNMENT)])
def test_expert_rows_refuses(lib, change, status):
    a = dict(choice=4096, T=4, k=2, E=8, offsets=4096, rows=4096, slots=4096)
    a.update(change)
    assert lib.pipe_expert_rows(a["choice"], a["T"], a["k"], a["E"], a["offsets"], a["rows"], a["slots"], None) == status


@pytest.mark.parametrize("T,k", [((1 << 31) - 2, 1), ((1 << 30) + 1, 1), ((1 << 30) - 1, 2), (1, (1 << 30) + 1)])
def test_expert_rows_refuses_places_that_its_steps_would_carry_past_31_bits(lib, T, k):
    assert lib.pipe_expert_rows(4096, T, k, 8, 4096, 4096, 4096, None) == B.PIPE_ERR_UNSUPPORTED


@pytest.mark.parametrize("change,status", [
    (dict(T=-1), B.PIPE_ERR_INVALID_ARG), (dict(N=-1), B.PIPE_ERR_INVALID_ARG), (dict(k=0), B.PIPE_ERR_INVALID_ARG), (dict(O=0), B.PIPE_ERR_INVALID_ARG),
    (dict(dtype=2), B.PIPE_ERR_INVALID_ARG), (dict(ldy=63), B.PIPE_ERR_INVALID_ARG), (dict(ldo=63), B.PIPE_ERR_INVALID_ARG),
    (dict(y=None), B.PIPE_ERR_INVALID_ARG), (dict(slots=None), B.PIPE_ERR_INVALID_ARG), (dict(weights=None), B.PIPE_ERR_INVALID_ARG),
    (dict(out=None), B.PIPE_ERR_INVALID_ARG), (dict(y=4097), B.PIPE_ERR_ALIGNMENT), (dict(out=4097), B.PIPE_ERR_ALIGNMENT),
    (dict(slots=4098), B.PIPE_ERR_ALIGNMENT), (dict(weights=4098), B.PIPE_ERR_ALIGNMENT)])
def test_expert_combine_refuses(lib, change, status):
    a = dict(y=4096, N=8, ldy=64, slots=4096, weights=4096, T=4, k=2, O=64, dtype=0, out=4096, ldo=64)
    a.update(change)
    assert lib.pipe_expert_combine(a["y"], a["N"], a["ldy"], a["slots"], a["weights"], a["T"], a["k"], a["O"], a["dtype"], a["out"], a["ldo"], None) == status


def test_the_binding_refuses_tensors_of_another_device():
    d = desc()
    codes, scales, _ = B.alloc_group(d, device="cpu")
    x, y = torch.zeros((2, 128), dtype=torch.bfloat16), torch.zeros((2, 64), dtype=torch.bfloat16)
    with pytest.raises(B.PipeError, match="current device"):
        B.pipe_group_linear(d, codes, scales, None, x, y)
    with pytest.raises(B.PipeError, match="current device"):
        B.pipe_expert_rows(torch.zeros((2, 2), dtype=torch.int32), 4, *(torch.zeros(n, dtype=torch.int32) for n in (5, 4, 4)))


@pytest.mark.parametrize("dtype", [2, -1, 7])
def test_the_binding_refuses_a_descriptor_of_another_type(dtype):
    d = desc()
    codes, scales, _ = B.alloc_group(d, device="cpu")
    d.dtype = dtype
    x, y = torch.zeros((2, 128), dtype=torch.bfloat16), torch.zeros((2, 64), dtype=torch.bfloat16)
    with pytest.raises(B.PipeError):
        B.pipe_group_linear(d, codes, scales, None, x, y)
    with pytest.raises(B.PipeError):
        B.pipe_group_quantize(d, torch.zeros((64, 128)), codes, scales)


def test_pack_and_unpack_are_inverses():
    u = torch.randint(0, 16, (2, 5, 96))
    assert torch.equal(R.unpack(R.pack(u), 96), u)
    one = torch.zeros((1, 1, 32), dtype=torch.int64)
    one[0, 0, 3] = 9                                     # code 2 * 1 + 1: nibble 5 of the first word
    assert R.pack(one)[0, 0, 0].tolist() == [0, 0, 9 << 4] + [0] * 13


def test_kernels_that_start_early_use_no_read_only_loads():
    """All of these kernels may stand on the SMs while the launch before still writes their inputs, weights included: nothing is
    read through the read-only path, whose loads the compiler may move above the dependency wait."""
    for name in sorted(os.listdir(GROUP)):
        if name.endswith((".cu", ".cuh")):
            text = re.sub(r"//[^\n]*", "", open(os.path.join(GROUP, name)).read())
            assert "__ldg(" not in text and "ld.global.nc" not in text and "__restrict__" not in text, name
