"""What the entry points of the 8-bit integer layers and of the log probabilities refuse, found on the host before anything is queued,
and the binding's own checks."""
import ctypes as C
import math
import os
import re

import pytest
import torch

from paper_2311_15806_b200 import binding as B
from paper_2311_15806_b200 import build as pipe_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2311_15806_b200", "csrc")
ARG, SHAPE, ALIGN, OVER = B.PIPE_ERR_INVALID_ARG, B.PIPE_ERR_SHAPE, B.PIPE_ERR_ALIGNMENT, B.PIPE_ERR_ACC_OVERFLOW


@pytest.fixture(scope="module")
def lib():
    pipe_build.build()
    return B.lib()


@pytest.mark.parametrize("change,status", [
    (dict(x=None), ARG), (dict(codes=None), ARG), (dict(scales=None), ARG), (dict(dtype=3), ARG), (dict(dtype=-1), ARG), (dict(T=-1), ARG),
    (dict(N=-1), ARG), (dict(T=(1 << 30) + 1, rows=4096), ARG), (dict(N=(1 << 30) + 1, rows=4096), ARG), (dict(I=0), ARG), (dict(I=(1 << 29) + 1, ldx=1 << 30, ldc=1 << 30), ARG),
    (dict(ldx=127), ARG), (dict(ldc=127), ARG), (dict(values=4096, ldv=127), ARG), (dict(ldx=1 << 32), ARG), (dict(ldc=1 << 32), ARG), (dict(values=4096, ldv=1 << 32), ARG),
    (dict(N=5), SHAPE), (dict(x=4098), ALIGN), (dict(scales=4098), ALIGN), (dict(values=4098, ldv=128), ALIGN), (dict(rows=4098), ALIGN), (dict(count=4098), ALIGN)])
def test_quantize_refuses(lib, change, status):
    a = dict(x=4096, dtype=2, T=4, I=128, ldx=128, rows=None, N=4, count=None, codes=4096, ldc=128, scales=4096, values=None, ldv=0)
    a.update(change)
    assert lib.pipe_int8_quantize(*a.values(), None) == status


@pytest.mark.parametrize("field,value,status", [
    ("experts", 0, ARG), ("experts", B.MAX_EXPERTS + 1, ARG), ("out_features", 0, ARG), ("out_features", (1 << 29) + 1, ARG), ("in_features", 0, ARG),
    ("in_features", -1, ARG), ("in_features", B.INT8_MAX_FEATURES + 1, OVER), ("dtype", 3, ARG), ("dtype", -1, ARG)])
def test_bad_descriptors(lib, field, value, status):
    d = B.make_int8_desc(64, 128)
    setattr(d, field, value)
    assert lib.pipe_int8_linear(C.byref(d), 4096, 1 << 20, 4096, 4096, 1, 1 << 20, 4096, None, 0, 4096, 1 << 30, None) == status
    assert lib.pipe_int8_expert_linear(C.byref(d), 4096, 1 << 20, 4096, 4096, 1 << 20, 4096, 4096, 1, None, 0, 4096, 1 << 30, None) == status


def test_descriptors_that_are_none_or_too_large_together(lib):
    assert lib.pipe_int8_linear(None, 4096, 128, 4096, 4096, 1, 128, 4096, None, 0, 4096, 64, None) == ARG
    d = B.make_int8_desc(1 << 28, 16, experts=8)
    assert lib.pipe_int8_expert_linear(C.byref(d), 4096, 16, 4096, 4096, 16, 4096, 4096, 1, None, 0, 4096, 1 << 28, None) == ARG
    with pytest.raises(B.PipeError):
        B.make_int8_desc(4, 4, dtype=torch.int8)


BAD = [(dict(codes=None), ARG), (dict(scales=None), ARG), (dict(x=None), ARG), (dict(sx=None), ARG), (dict(y=None), ARG), (dict(T=-1), ARG), (dict(T=(1 << 30) + 1), ARG),
       (dict(act=5), ARG), (dict(act=-1), ARG), (dict(ldw=112), ARG), (dict(ldx=112), ARG), (dict(ldy=63), ARG), (dict(ldw=1 << 40), ARG), (dict(ldx=1 << 40), ARG),
       (dict(ldy=1 << 40), ARG), (dict(ldw=136), ALIGN), (dict(ldx=136), ALIGN), (dict(codes=4104), ALIGN), (dict(x=4104), ALIGN), (dict(scales=4098), ALIGN),
       (dict(sx=4098), ALIGN), (dict(bias=4097), ALIGN), (dict(y=4097), ALIGN)]


@pytest.mark.parametrize("change,status", BAD)
def test_products_refuse(lib, change, status):
    a = dict(codes=4096, ldw=128, scales=4096, x=4096, T=2, ldx=128, sx=4096, bias=None, act=0, y=4096, ldy=64)
    a.update(change)
    assert lib.pipe_int8_linear(C.byref(B.make_int8_desc(64, 128)), *a.values(), None) == status
    assert lib.pipe_int8_expert_linear(C.byref(B.make_int8_desc(64, 128, experts=3)), a["codes"], a["ldw"], a["scales"], a["x"], a["ldx"], a["sx"], 4096, a["T"], a["bias"],
                                       a["act"], a["y"], a["ldy"], None) == status


def test_products_refuse_besides(lib):
    f32 = B.make_int8_desc(64, 128, dtype=torch.float32)
    assert lib.pipe_int8_linear(C.byref(f32), 4096, 128, 4096, 4096, 2, 128, 4096, None, 0, 4098, 64, None) == ALIGN
    assert lib.pipe_int8_linear(C.byref(f32), 4096, 128, 4096, 4096, 2, 128, 4096, 4098, 0, 4096, 64, None) == ALIGN
    many = B.make_int8_desc(64, 128, experts=3)
    assert lib.pipe_int8_linear(C.byref(many), 4096, 128, 4096, 4096, 2, 128, 4096, None, 0, 4096, 64, None) == SHAPE
    for offsets, status in ((None, ARG), (4098, ALIGN)):
        assert lib.pipe_int8_expert_linear(C.byref(many), 4096, 128, 4096, 4096, 128, 4096, offsets, 2, None, 0, 4096, 64, None) == status


def test_no_rows_are_no_work(lib):
    assert lib.pipe_int8_quantize(None, 0, 0, 8, 8, None, 0, None, None, 16, None, None, 0, None) == B.PIPE_OK
    assert lib.pipe_int8_linear(C.byref(B.make_int8_desc(64, 128)), 4096, 128, 4096, None, 0, 128, None, None, 0, None, 64, None) == B.PIPE_OK
    assert lib.pipe_int8_expert_linear(C.byref(B.make_int8_desc(64, 128, experts=3)), 4096, 128, 4096, None, 128, None, 4096, 0, None, 0, None, 64, None) == B.PIPE_OK
    assert lib.pipe_token_logprobs(None, 0, 0, 8, 8, 1.0, None, 0, None, None, 0, None, None, None) == B.PIPE_OK


@pytest.mark.parametrize("change,status", [
    (dict(l=None), ARG), (dict(dtype=3), ARG), (dict(dtype=-1), ARG), (dict(T=-1), ARG), (dict(T=(1 << 30) + 1), ARG), (dict(V=0), ARG), (dict(V=(1 << 30) + 1, ldl=1 << 31), ARG),
    (dict(ldl=99), ARG), (dict(ldl=1 << 32), ARG), (dict(n=-1), ARG), (dict(n=(1 << 20) + 1), ARG), (dict(T=1 << 25, n=1 << 16), ARG), (dict(n=0), ARG), (dict(tokens=None), ARG),
    (dict(lp=None), ARG), (dict(k=-1), ARG), (dict(k=B.MAX_TOP + 1), ARG), (dict(k=0), ARG), (dict(top=None, tlp=None), ARG), (dict(scale=0.0), ARG), (dict(scale=-1.0), ARG),
    (dict(scale=math.nan), ARG), (dict(scale=math.inf), ARG), (dict(scale=2.0 ** -21), ARG), (dict(scale=2.0 ** 21), ARG), (dict(l=4097), ALIGN), (dict(dtype=2, l=4098), ALIGN),
    (dict(tokens=4098), ALIGN), (dict(lp=4098), ALIGN), (dict(ent=4098), ALIGN), (dict(top=4098), ALIGN), (dict(tlp=4098), ALIGN)])
def test_logprobs_refuse(lib, change, status):
    a = dict(l=4096, dtype=0, T=2, V=100, ldl=100, scale=1.0, tokens=4096, n=1, lp=4096, ent=4096, k=5, top=4096, tlp=4096)
    a.update(change)
    assert lib.pipe_token_logprobs(*a.values(), None) == status


def _cpu(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype)


@pytest.mark.parametrize("what", ["codes", "scales", "x", "sx", "y", "bias", "rows", "pitch", "type"])
def test_the_binding_refuses_arrays_that_are_not_the_layers(what):
    i8, h = torch.int8, torch.bfloat16
    d = B.make_int8_desc(8, 32)
    a = dict(codes=_cpu(8, 32, dtype=i8), scales=_cpu(8), xq=_cpu(4, 32, dtype=i8), sx=_cpu(4), y=_cpu(4, 8, dtype=h), bias=_cpu(8, dtype=h))
    a.update({"codes": dict(codes=_cpu(32, 8, dtype=i8)), "scales": dict(scales=_cpu(7)), "x": dict(xq=_cpu(4, 33, dtype=i8)), "sx": dict(sx=_cpu(3)), "y": dict(y=_cpu(4, 9, dtype=h)),
              "bias": dict(bias=_cpu(8)), "rows": dict(y=_cpu(5, 8, dtype=h)), "pitch": dict(xq=_cpu(4, 64, dtype=i8)[:, ::2]), "type": dict(codes=_cpu(8, 32, dtype=torch.uint8))}[what])
    bias = a.pop("bias")
    with pytest.raises(B.PipeError):
        B.pipe_int8_linear(d, *a.values(), bias=bias)
    y = a.pop("y")
    with pytest.raises(B.PipeError):
        B.pipe_int8_expert_linear(d, *a.values(), _cpu(2, dtype=torch.int32), y, bias=bias)


def test_the_binding_refuses_tensors_of_another_device_and_other_arguments():
    i8, i32 = torch.int8, torch.int32
    with pytest.raises(B.PipeError, match="current device"):
        B.pipe_int8_quantize(_cpu(4, 32), _cpu(4, 32, dtype=i8), _cpu(4))
    with pytest.raises(B.PipeError, match="current device"):
        B.pipe_int8_linear(B.make_int8_desc(8, 32), _cpu(8, 32, dtype=i8), _cpu(8), _cpu(4, 32, dtype=i8), _cpu(4), _cpu(4, 8, dtype=torch.bfloat16))
    with pytest.raises(B.PipeError, match="current device"):
        B.pipe_token_logprobs(_cpu(4, 32), entropy=_cpu(4))
    for change in (dict(codes=_cpu(4, 31, dtype=i8)), dict(codes=_cpu(4, 32, dtype=torch.uint8)), dict(scales=_cpu(5)), dict(x=_cpu(4, 32, dtype=torch.float64)), dict(x=_cpu()),
                   dict(rows=_cpu(3, dtype=i32)), dict(rows=_cpu(4, dtype=torch.int64)), dict(count=_cpu(2, dtype=i32)), dict(values=_cpu(4, 31)), dict(values=_cpu(4, 32, dtype=torch.float16)),
                   dict(x=_cpu(4, 64)[:, ::2]), dict(x=_cpu(2, 4, 32)[:, :2])):
        a = dict(x=_cpu(4, 32), codes=_cpu(4, 32, dtype=i8), scales=_cpu(4), rows=None, count=None, values=None)
        a.update(change)
        with pytest.raises(B.PipeError):
            B.pipe_int8_quantize(**a)
    for change in (dict(logits=_cpu(32)), dict(logits=_cpu(4, 32, dtype=torch.float64)), dict(tokens=_cpu(4, 1, dtype=i32)), dict(logprobs=_cpu(4, 1)),
                   dict(tokens=_cpu(4, 1, dtype=torch.int64), logprobs=_cpu(4, 1)), dict(tokens=_cpu(4, 2, dtype=i32), logprobs=_cpu(4, 1)), dict(tokens=_cpu(3, dtype=i32), logprobs=_cpu(3)),
                   dict(entropy=_cpu(4, 1)), dict(entropy=_cpu(8)[::2]), dict(top=_cpu(4, 2)), dict(top=_cpu(4, 2, dtype=i32), top_logprobs=_cpu(4, 3)), dict(logits=_cpu(4, 64)[:, ::2])):
        a = dict(logits=_cpu(4, 32))
        a.update(change)
        with pytest.raises(B.PipeError):
            B.pipe_token_logprobs(**a)


def test_arrays_are_given_the_pitch_that_products_want():
    codes, scales = B.alloc_int8(5, 33, device="cpu")
    assert codes.shape == (5, 33) and codes.stride() == (48, 1) and scales.shape == (5,)
    codes, scales = B.alloc_int8(5, 33, device="cpu", experts=2)
    assert codes.shape == (2, 5, 33) and B._pitch_of("", codes, 33) == 48 and scales.shape == (2, 5)
    assert B._pitch_of("", torch.zeros((1, 33), dtype=torch.int8), 33) == 48          # one row: any pitch will do
    assert B._pitch_of("", torch.zeros((1, 1, 33), dtype=torch.int8), 33) == 48
    assert B._pitch_of("", torch.zeros((3, 1, 48), dtype=torch.int8)[..., :33], 33) == 48
    with pytest.raises(B.PipeError):
        B._pitch_of("", torch.zeros((2, 8, 48), dtype=torch.int8)[:, :5], 48)         # experts at another distance than their rows


def test_kernels_that_start_early_use_no_read_only_loads():
    """All of these kernels may stand on the SMs while the launch before still writes their inputs: nothing is read through the read-only
    path, whose loads the compiler may move above the dependency wait."""
    seen = 0
    for folder in ("int8", "logprob"):
        for name in sorted(os.listdir(os.path.join(CSRC, folder))):
            if name.endswith((".cu", ".cuh")):
                text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, folder, name)).read())
                seen += 1
                assert "__ldg(" not in text and "ld.global.nc" not in text and "__restrict__" not in text, name
                assert "return PIPE_ERR_CUDA" not in text and "cudaFuncSetAttribute" not in text, name   # (runtime_failed, allow_dynamic_smem)
    assert seen >= 4


def test_long_rows_are_given_whole_lines():
    for I, pitch in ((512, 512), (513, 640), (700, 768), (4096, 4096)):
        codes, _ = B.alloc_int8(3, I, device="cpu")
        assert codes.stride() == (pitch, 1)
        codes, _ = B.alloc_int8(3, I, device="cpu", experts=2)
        assert codes.stride() == (3 * pitch, pitch, 1)
