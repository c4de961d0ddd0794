"""sigma of the 4-bit layers where it is delicate: every finite value of the layer's type, far tails among them, NaN and infinities."""
import pytest
import torch

from paper_2311_15806_b200 import binding as B
from tests import group_reference as R

pytestmark = pytest.mark.gpu
KINDS = [B.ACT_IDENTITY, B.ACT_RELU, B.ACT_SILU, B.ACT_GELU, B.ACT_SIGMOID]
# (tokens, reduction length): the kernel for few rows, the tensor-core kernel, and its form whose CTAs share an axis (few channels then)
FORMS = [(1, 32), (20, 32), (20, 2048)]


def _outputs(v, T, I, h, kind):
    """sigma(0 + v): activations of zero, v as the bias."""
    desc = B.make_group_desc(v.numel(), I, 32, dtype=h)
    codes, scales, _ = B.alloc_group(desc)
    codes.fill_(0x5A)
    scales.fill_(0.01)
    x = torch.zeros((T, I), dtype=h, device="cuda")
    y = torch.empty((T, v.numel()), dtype=h, device="cuda")
    B.pipe_group_linear(desc, codes, scales, None, x, y, bias=v.cuda(), activation=kind)
    torch.cuda.synchronize()
    assert B.pipe_poll_status() == B.PIPE_OK
    return y.cpu()


def _finite(h):
    v = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(h)
    return v[torch.isfinite(v)]


@pytest.mark.parametrize("T,I", FORMS)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("kind", KINDS)
def test_every_value_of_the_type(kind, dtype, T, I):
    """Distance allowed, as a fraction of sigma(v): half a step of the output, and
      SiLU, sigmoid   |v| 2^-23 + 2^-20: the exponential's argument is a product with a rounded constant (2^-26 + 2^-24 of |v| log2 e,
                      an exponent of two), the exponential 2^-22, the reciprocal 2^-23, the other roundings 2^-24 each
      GELU            (v^2 + 2) 2^-23 + 2^-20: erfc's argument z = |v| / sqrt 2 is off by less than 2^-23 of itself, which erfc answers
                      with at most 2 z^2 + 2 of that; erfcf is documented to 4 units in the last place (2^-21), the products 2^-24 each
    and behind that where an exponential is no normal number any more its spacing, |v| 2^-147, and half the type's smallest number."""
    h = R.TYPES[dtype]
    v = _finite(h)
    if I > 32:
        v = v[::61]
    got = _outputs(v, T, I, h, kind).double()
    d = v.double()
    # (erfc, not the normal distribution, which is 0 in 64 bits from -8.3 on: (1 + erf) / 2)
    want = 0.5 * d * torch.special.erfc(-d / 2 ** 0.5) if kind == B.ACT_GELU else R.sigma(d, kind)
    part = {B.ACT_SILU: d.abs() * 2.0 ** -23 + 2.0 ** -20, B.ACT_SIGMOID: d.abs() * 2.0 ** -23 + 2.0 ** -20,
            B.ACT_GELU: (d * d + 2) * 2.0 ** -23 + 2.0 ** -20}.get(kind, torch.zeros_like(d))
    tol = torch.where(want == 0, 0, part * want.abs()) + (0 if kind <= B.ACT_RELU else (d.abs().clamp(max=200) + 1) * 2.0 ** -147)
    tol = tol + torch.finfo(h).eps / 2 * (want.abs() + tol) + torch.finfo(h).smallest_normal * torch.finfo(h).eps / 2
    off = (got - want[None]).abs()
    worst = off / tol
    at = int(worst.max(0).values.argmax())
    assert torch.isfinite(got).all() and float(worst.max()) <= 1, f"v {float(d[at])}: {float(got[0, at])}, not {float(want[at])}"
    assert torch.equal(got, got[:1].expand_as(got))


@pytest.mark.parametrize("T,I", FORMS)
@pytest.mark.parametrize("kind", KINDS)
def test_a_nan_stays_a_nan(kind, T, I):
    h, O = torch.bfloat16, 130
    desc = B.make_group_desc(O, I, 32)
    codes, scales, _ = B.alloc_group(desc)
    codes.fill_(0x5A)
    scales.fill_(0.01)
    x = torch.zeros((T, I), dtype=h)
    x[T - 1, 3] = float("nan")
    bias = torch.zeros(O, dtype=h)
    bias[7] = float("nan")
    y = torch.empty((T, O), dtype=h, device="cuda")
    B.pipe_group_linear(desc, codes, scales, None, x.cuda(), y, bias=bias.cuda(), activation=kind)
    torch.cuda.synchronize()
    assert B.pipe_poll_status() == B.PIPE_OK
    nan = torch.isnan(y.cpu())
    want = torch.zeros_like(nan)
    want[T - 1] = True
    want[:, 7] = True
    assert torch.equal(nan, want)


@pytest.mark.parametrize("T,I", FORMS)
def test_infinities(T, I):
    inf = float("inf")
    v = torch.tensor([inf, -inf], dtype=torch.bfloat16)
    for kind, want in ((B.ACT_IDENTITY, [inf, -inf]), (B.ACT_RELU, [inf, 0]), (B.ACT_SIGMOID, [1, 0])):
        assert _outputs(v, T, I, torch.bfloat16, kind)[0].tolist() == want
    for kind in (B.ACT_SILU, B.ACT_GELU):
        assert float(_outputs(v, T, I, torch.bfloat16, kind)[0, 0]) == inf
