"""Products of the 8-bit integer layers whose reduction axis several CTAs share: narrow layers with long axes on few rows."""
import pytest
import torch

from paper_2311_15806_b200 import binding as B
from tests import int8_reference as R

pytestmark = pytest.mark.gpu


def _gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def _layer(gen, E, O, I):
    """Codes, scales, and the codes on the GPU."""
    w = torch.randint(-128, 128, (E, O, I), generator=gen, dtype=torch.int8)
    sw = torch.rand((E, O), generator=gen) * 0.01 + 0.001
    codes, _ = B.alloc_int8(O, I, experts=E)
    return w, sw, codes.copy_(w)


@pytest.mark.parametrize("T,O,I", [(1, 3584, 18944), (13, 2560, 14336), (32, 200, 11008), (8, 1411, 11009), (5, 31, 30001), (63, 384, 28672), (1, 1, 11008), (40, 129, 9000),
                                   (64, 100, 65536), (3, 768, B.INT8_MAX_FEATURES)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_layers(T, O, I, dtype):
    gen, h = _gen(T + O), R.TYPES[dtype]
    w, sw, codes = _layer(gen, 1, O, I)
    x = torch.randint(-128, 128, (T, I), generator=gen, dtype=torch.int8)
    xq, _ = B.alloc_int8(T, I)
    xq.copy_(x)
    sx = torch.rand((T,), generator=gen) * 1e-3
    b = torch.randn((O,), generator=gen).to(h)
    y = torch.full((T, O + 5), -7.0, dtype=h, device="cuda")
    B.pipe_int8_linear(B.make_int8_desc(O, I, dtype=h), codes, sw.cuda(), xq, sx.cuda(), y[:, :O], bias=b.cuda(), activation=T % 2)
    torch.cuda.synchronize()
    assert B.pipe_poll_status() == B.PIPE_OK
    R.check_product(y[:, :O], x, sx, w[0], sw[0], b, T % 2, dtype, f"{T} {O} {I}")
    assert (y[:, O:] == -7).all()


@pytest.mark.parametrize("O,I", [(200, 11008), (1411, 14336)])
def test_a_row_is_the_same_among_many(O, I):
    """Few rows share the axis, many do not."""
    gen = _gen(2)
    _, sw, codes = _layer(gen, 1, O, I)
    xq, _ = B.alloc_int8(600, I)
    xq.copy_(torch.randint(-128, 128, (600, I), generator=gen, dtype=torch.int8))
    sx, sw, d = torch.rand((600,), generator=gen).cuda(), sw.cuda(), B.make_int8_desc(O, I)
    whole = torch.empty((600, O), dtype=torch.bfloat16, device="cuda")
    B.pipe_int8_linear(d, codes, sw, xq, sx, whole, activation=B.ACT_SILU)
    for n in (1, 4, 17, 40):
        y = torch.empty((n, O), dtype=torch.bfloat16, device="cuda")
        B.pipe_int8_linear(d, codes, sw, xq[:n], sx[:n], y, activation=B.ACT_SILU)
        torch.cuda.synchronize()
        assert B.pipe_poll_status() == B.PIPE_OK
        assert torch.equal(y, whole[:n]), n


@pytest.mark.parametrize("counts", [[1], [0, 3], [2, 0, 1, 5], [17, 0, 40], [0, 0, 64], [1] * 8])
@pytest.mark.parametrize("O,I", [(200, 11008), (100, 18945)])
def test_experts(counts, O, I):
    """Fewer tiles than clusters, as a rule: some have none."""
    gen, E = _gen(sum(counts)), len(counts)
    w, sw, codes = _layer(gen, E, O, I)
    N = sum(counts) + 2
    off = torch.zeros(E + 1, dtype=torch.int32)
    off[1:] = torch.tensor(counts).cumsum(0)
    x = torch.randint(-128, 128, (N, I), generator=gen, dtype=torch.int8)
    xq, _ = B.alloc_int8(N, I)
    xq.copy_(x)
    sx = torch.rand((N,), generator=gen) * 1e-3
    y = torch.full((N, O), -7.0, device="cuda")
    B.pipe_int8_expert_linear(B.make_int8_desc(O, I, dtype=torch.float32, experts=E), codes, sw.cuda(), xq, sx.cuda(), off.cuda(), y)
    torch.cuda.synchronize()
    assert B.pipe_poll_status() == B.PIPE_OK
    for e in range(E):
        lo, hi = int(off[e]), int(off[e + 1])
        R.check_product(y[lo:hi], x[lo:hi], sx[lo:hi], w[e], sw[e], None, 0, "fp32", f"expert {e}")
    assert (y[-2:] == -7).all()
