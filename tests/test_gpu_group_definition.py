"""The products against the definition itself, W = s (u - z) as it stands, at every number of rows."""
import pytest
import torch

from paper_2311_15806_b200 import binding as B
from tests import group_reference as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,asym,g", [("bf16", False, 128), ("bf16", True, 32), ("fp16", False, 64), ("fp16", True, 128)])
@pytest.mark.parametrize("T,O,I", [(1, 272, 640), (16, 272, 640), (17, 272, 640), (64, 130, 2048), (300, 272, 640), (2049, 600, 384)])
def test_linear(T, O, I, dtype, asym, g):
    """Distance allowed: up to 16 rows a group's products are exact and are added in binary32 (counted as in check_product); beyond,
    every weight may be off by half a step of the type, eps / 2 of itself, which x meets as eps / 2 of the sum of magnitudes, and the
    I / 16 steps of the sum cut at 2^-20 of the largest addend each.  Then half a step of the output.  As a whole, the rounded weights
    being independent, the squares add up: the distance's norm is bounded by the output's and the weights' roundings, each at most half a
    step and uniform, 1 / sqrt 3 of it, of numbers between one and two steps' units: eps / 2 / sqrt 3 of the norm for either."""
    gen, h = torch.Generator(), R.TYPES[dtype]
    gen.manual_seed(T + O)
    u, s, z = R.random_layer(gen, 1, O, I, g, dtype, asym)
    x = torch.randn((T, I), generator=gen).to(h)
    y = torch.empty((T, O), dtype=h, device="cuda")
    B.pipe_group_linear(B.make_group_desc(O, I, g, dtype=h, asymmetric=asym), R.pack(u).cuda(), s.cuda(), None if z is None else z.cuda(), x.cuda(), y)
    torch.cuda.synchronize()
    assert B.pipe_poll_status() == B.PIPE_OK
    W, xd, half = R.dense(u, s, z, g)[0], x.double(), torch.finfo(h).eps / 2
    want, terms = xd @ W.t(), xd.abs() @ W.abs().t()
    few = R.few(T)
    steps = 8 * 2.0 ** -20 + (I // g + 64) * 2.0 ** -24 if few else half + (1 + half) * (I / 16 + 8) * 2.0 ** -20
    tol = steps * terms
    tol = tol + half * (want.abs() + tol) + torch.finfo(h).smallest_normal * torch.finfo(h).eps
    off = (y.cpu().double() - want).abs()
    assert float((off / tol).max()) <= 1
    parts = 1 if few else 2 ** 0.5
    assert float(off.norm() / want.norm()) <= parts * half / 3 ** 0.5 * 1.05   # (5 %: a norm of thousands of samples)
