"""Scales near the end of the type's range: a weight s (u - z) that the type cannot hold is a number of the layer all the same."""
import pytest
import torch

from paper_2311_15806_b200 import binding as B
from tests import group_reference as R

pytestmark = pytest.mark.gpu
LARGE = {"fp16": (5000.0, 60000.0, 2.0 ** -11), "bf16": (2.0 ** 125, 2.0 ** 127, 2.0 ** -100)}   # scales, and what the activations are times


def _gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def _layer(gen, E, O, I, g, dtype, asym):
    """A layer whose every third channel has one group of a large scale."""
    u, s, z = R.random_layer(gen, E, O, I, g, dtype, asym)
    lo, hi, _ = LARGE[dtype]
    wide = torch.zeros((E, O), dtype=torch.bool)
    for e in range(E):
        for o in range(e, O, 3):
            wide[e, o] = True
            at = int(torch.randint(0, I // g, (1,), generator=gen))
            s[e, at, o] = lo + (hi - lo) * float(torch.rand(1, generator=gen))
            if o % 2:
                s[e, at, o] *= -1
    return u, s, z, wide


def _check(y, x, W, b, wide, dtype, g, few, tag):
    for channels, exact in ((wide, True), (~wide, few)):
        if channels.any():
            R.check_product(y.cpu()[:, channels], x, W[channels], None if b is None else b[channels], 0, dtype, g, exact, tag)


@pytest.mark.parametrize("dtype,asym,g", [("fp16", False, 64), ("fp16", True, 32), ("bf16", True, 128), ("bf16", False, 32)])
@pytest.mark.parametrize("T,O,I", [(1, 130, 384), (16, 130, 384), (17, 130, 384), (17, 140, 2048), (90, 300, 256), (300, 300, 128), (2100, 1000, 128)])
def test_linear(T, O, I, dtype, asym, g):
    gen, h = _gen(T + O), R.TYPES[dtype]
    u, s, z, wide = _layer(gen, 1, O, I, g, dtype, asym)
    x = (torch.randn((T, I), generator=gen) * LARGE[dtype][2]).to(h)
    b = torch.randn((O,), generator=gen).to(h)
    y = torch.full((T, O + 3), 7.0, dtype=h, device="cuda")
    desc = B.make_group_desc(O, I, g, dtype=h, asymmetric=asym)
    B.pipe_group_linear(desc, R.pack(u).cuda(), s.cuda(), None if z is None else z.cuda(), x.cuda(), y[:, :O], bias=b.cuda())
    torch.cuda.synchronize()
    assert B.pipe_poll_status() == B.PIPE_OK
    _check(y[:, :O], x, R.dense(u, s, z, g)[0], b, wide[0], dtype, g, R.few(T), f"T {T} O {O} I {I}")
    assert (y[:, O:] == 7).all()


@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("dtype,asym,g", [("fp16", True, 64), ("bf16", False, 128)])
@pytest.mark.parametrize("counts,O", [([3, 0, 9], 70), ([40, 0, 7, 100], 130), ([300, 1, 700], 600)])
def test_experts(counts, O, dtype, asym, g, gather):
    """Rows whose index lies outside, which read as zeros, among them."""
    gen, h, E, I, T = _gen(O), R.TYPES[dtype], len(counts), 256, 33
    u, s, z, wide = _layer(gen, E, O, I, g, dtype, asym)
    N = sum(counts) + 2
    offsets = torch.zeros(E + 1, dtype=torch.int32)
    offsets[1:] = torch.tensor(counts).cumsum(0)
    x = (torch.randn((T if gather else N, I), generator=gen) * LARGE[dtype][2]).to(h)
    rows = None
    read = x
    if gather:
        rows = torch.randint(0, T, (N,), generator=gen, dtype=torch.int32)
        rows[1], rows[N - 4] = -1, T
        inside = (rows >= 0) & (rows < T)
        read = torch.where(inside[:, None], x[rows.clamp(0, T - 1).long()], torch.zeros((), dtype=h))
    b = torch.randn((E, O), generator=gen).to(h)
    y = torch.full((N, O), 7.0, dtype=h, device="cuda")
    B.pipe_expert_linear(B.make_group_desc(O, I, g, dtype=h, asymmetric=asym, experts=E), R.pack(u).cuda(), s.cuda(), None if z is None else z.cuda(), x.cuda(),
                         offsets.cuda(), y, rows=None if rows is None else rows.cuda(), bias=b.cuda())
    torch.cuda.synchronize()
    assert B.pipe_poll_status() == B.PIPE_OK
    W = R.dense(u, s, z, g)
    for e in range(E):
        lo, hi = int(offsets[e]), int(offsets[e + 1])
        if lo < hi:
            _check(y[lo:hi], read[lo:hi], W[e], b[e], wide[e], dtype, g, R.few(-(-N // E)), f"expert {e}")
    assert (y[N - 2:] == 7).all()
