"""Calls of two host threads at once: neither may see what the other's launch asks the runtime for."""
import threading

import pytest
import torch

from paper_2311_15806_b200 import binding as B

pytestmark = pytest.mark.gpu


def _together(*calls, times=4000):
    """Every call `times` times, each from a thread and on a stream of its own; what they raised."""
    raised, start = [], threading.Barrier(len(calls))

    def work(call):
        try:
            stream = torch.cuda.Stream()
            start.wait()
            for i in range(times):
                call(stream)
                if i % 256 == 255:
                    stream.synchronize()
            stream.synchronize()
        except Exception as e:
            raised.append(e)

    threads = [threading.Thread(target=work, args=(c,)) for c in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert B.pipe_poll_status() == B.PIPE_OK
    return raised


def test_layers_of_one_kernel_with_tiles_of_different_size():
    """32 and 18944 tokens of a layer with 128 channels: tiles of 32 and of 128 rows, in different amounts of shared memory."""
    gen = torch.Generator()
    gen.manual_seed(5)
    desc = B.make_group_desc(128, 256, 64)
    codes, scales, _ = B.alloc_group(desc)
    codes.copy_(torch.randint(0, 256, codes.shape, generator=gen, dtype=torch.uint8))
    scales.copy_(torch.rand(scales.shape, generator=gen) * 0.02)
    calls, pairs = [], []
    for T in (32, 18944):
        x = torch.randn((T, 256), generator=gen).to(torch.bfloat16).cuda()
        alone, y = (torch.empty((T, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        B.pipe_group_linear(desc, codes, scales, None, x, alone)
        calls.append(lambda stream, x=x, y=y: B.pipe_group_linear(desc, codes, scales, None, x, y, stream=stream))
        pairs.append((alone, y))
    torch.cuda.synchronize()
    assert _together(*calls) == []
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in pairs)


def test_rows_of_different_numbers_of_experts():
    """512 and 1024 experts: 64 and 128 KB of shared memory."""
    calls, outs = [], []
    for E in (512, 1024):
        choice = (torch.arange(200, dtype=torch.int32, device="cuda").view(100, 2) * 7) % E
        out = (torch.empty(E + 1, dtype=torch.int32, device="cuda"), torch.empty(200, dtype=torch.int32, device="cuda"),
               torch.empty((100, 2), dtype=torch.int32, device="cuda"))
        alone = tuple(torch.empty_like(t) for t in out)
        B.pipe_expert_rows(choice, E, *alone)
        calls.append(lambda stream, c=choice, E=E, o=out: B.pipe_expert_rows(c, E, *o, stream=stream))
        outs += zip(alone, out)
    torch.cuda.synchronize()
    assert _together(*calls) == []
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in outs)
