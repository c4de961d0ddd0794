"""Calls from a host thread that has made no other CUDA call before: a server's worker that is handed everything."""
import threading

import numpy as np
import pytest
import torch

from paper_2311_15806_b200 import binding as B
from tests import gpu_harness as H

pytestmark = pytest.mark.gpu


def _in_a_thread(call):
    raised = []

    def work():
        try:
            call()
        except Exception as e:
            raised.append(e)

    t = threading.Thread(target=work)
    t.start()
    t.join()
    torch.cuda.synchronize()
    assert raised == [] and B.pipe_poll_status() == B.PIPE_OK


@pytest.mark.parametrize("T", [1, 16, 40, 300])
def test_layers_with_group_scales(T):
    gen = torch.Generator()
    gen.manual_seed(T)
    d = B.make_group_desc(136, 256, 64)
    codes, scales, _ = B.alloc_group(d)
    W = torch.randn((136, 256), generator=gen).cuda()
    x = torch.randn((T, 256), generator=gen).to(torch.bfloat16).cuda()
    offsets = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    _in_a_thread(lambda: B.pipe_group_quantize(d, W, codes, scales))
    want, y, z = (torch.full((T, 136), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    B.pipe_group_linear(d, codes, scales, None, x, want)
    _in_a_thread(lambda: B.pipe_group_linear(d, codes, scales, None, x, y))
    _in_a_thread(lambda: B.pipe_expert_linear(d, codes, scales, None, x, offsets, z))
    assert torch.equal(y, want) and torch.equal(z, want)


def test_rows_and_weighted_sum():
    choice = torch.tensor([[0, 2], [2, 1], [1, 0]], dtype=torch.int32, device="cuda")
    offsets, rows, slots = (torch.empty(s, dtype=torch.int32, device="cuda") for s in ((4,), (6,), (3, 2)))
    _in_a_thread(lambda: B.pipe_expert_rows(choice, 3, offsets, rows, slots))
    assert offsets.tolist() == [0, 2, 4, 6] and rows.tolist() == [0, 2, 1, 2, 0, 1]
    y = torch.eye(6, dtype=torch.bfloat16, device="cuda")
    out = torch.empty((3, 6), dtype=torch.bfloat16, device="cuda")
    _in_a_thread(lambda: B.pipe_expert_combine(y, slots, torch.ones((3, 2), device="cuda"), out))
    assert torch.equal(out, y[slots[:, 0].long()] + y[slots[:, 1].long()])


@pytest.mark.parametrize("T,kernel", [(1, B.KERNEL_AUTO), (16, B.KERNEL_STREAM), (16, B.KERNEL_DECODE_TC), (200, B.KERNEL_TCGEN05), (200, B.KERNEL_TCGEN05_PAIR)])
def test_expanded_layers(T, kernel):
    rng = np.random.default_rng(T)
    layer = H.gpu_expand(H.desc_of(384, 512, 4, 3, 8, 24, 1), rng.standard_normal((384, 512)).astype(np.float32))
    xq, sx = H.gpu_quantize(rng.standard_normal((T, 512)).astype(np.float32))
    want, _ = H.gpu_linear(layer, xq, sx, want_partials=False, kernel=kernel)
    y = torch.full((T, 384), float("nan"), device="cuda")
    B.pipe_diag_select_kernel(kernel)
    try:
        _in_a_thread(lambda: B.pipe_expanded_linear(layer.desc, layer.blob, xq, sx, y))
    finally:
        B.pipe_diag_select_kernel(B.KERNEL_AUTO)
    np.testing.assert_array_equal(y.cpu().numpy(), want)
