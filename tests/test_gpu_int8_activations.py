"""sigma of the 8-bit integer layers where it is delicate: far tails, every finite value of the 16-bit types, NaN and infinities, through
every form of the kernel."""
import pytest
import torch

from paper_2311_15806_b200 import binding as B
from tests import int8_reference as R

pytestmark = pytest.mark.gpu
KINDS = [B.ACT_IDENTITY, B.ACT_RELU, B.ACT_SILU, B.ACT_GELU, B.ACT_SIGMOID]
# tokens, reduction length, most channels, pitch beyond the channels: single CTAs, pairs, pairs whose rows begin anywhere, CTAs that share an axis
FORMS = {"single": (3, 16, 1 << 20, 0), "pair": (300, 16, 1 << 20, 0), "anywhere": (300, 16, 1 << 20, 3), "split": (3, 11008, 4096, 0)}


def _outputs(v, form, h, kind):
    """h(sigma(v)): sums of one, v as the channels' scales."""
    T, I, most, beyond = FORMS[form]
    out = []
    for part in v.split(most):
        O = part.numel()
        w, x = torch.zeros((O, I), dtype=torch.int8, device="cuda"), torch.zeros((T, I), dtype=torch.int8, device="cuda")
        w[:, I // 2] = 1
        x[:, I // 2] = 1
        y = torch.empty((T, O + beyond), dtype=h, device="cuda")[:, :O]
        B.pipe_int8_linear(B.make_int8_desc(O, I, dtype=h), w, part.cuda(), x, torch.ones(T, device="cuda"), y, activation=kind)
        torch.cuda.synchronize()
        assert B.pipe_poll_status() == B.PIPE_OK
        bits = y.view(torch.int32 if h == torch.float32 else torch.int16)
        assert torch.equal(bits, bits[:1].expand(T, O))
        out.append(y[0].cpu())
    return torch.cat(out)


def _values(h, form):
    """Every finite number of the 16-bit types; of the 32-bit one those of bf16, and others from where sigma is near 0 to where it is near 1
    or v."""
    v = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16 if h == torch.float32 else h)
    v = v[torch.isfinite(v)].float()
    if h == torch.float32:
        g = torch.Generator()
        g.manual_seed(3)
        u = torch.rand((1 << 16,), generator=g)
        v = torch.cat([v, -110 + 130 * u, 6 * u - 4, -torch.exp2(20 * u - 13)])
    return v[::31] if form == "split" else v


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("kind", KINDS)
def test_every_value(kind, dtype, form):
    """Distance allowed, as a fraction of sigma(v): half a step of a 16-bit output, and
      outputs of 32 bits   SiLU, sigmoid 2^-20, GELU 2^-19 (what include/pipe.h says)
      of 16 bits           SiLU, sigmoid |v| 2^-23 + 2^-20: the exponential's argument is a rounded product with a rounded constant (2^-26 +
                           2^-24 of |v| log2 e, an exponent of two), the exponential 2^-22, the reciprocal 2^-23, the others 2^-24 each;
                           GELU v^2 2^-23 + 2^-19: three such roundings of v^2 / 2 log2 e, the polynomial and the products 2^-20
    and behind that, where an exponential is no normal number any more, some of its spacings, (|v| + 1) 2^-147, and half the type's
    smallest number."""
    h = R.TYPES[dtype]
    v = _values(h, form)
    got = _outputs(v, form, h, kind).double()
    d = v.double()
    # (erfc, not the normal distribution, which is 0 in 64 bits from -8.3 on)
    want = 0.5 * d * torch.special.erfc(-d / 2 ** 0.5) if kind == B.ACT_GELU else R.sigma(d, kind)
    if dtype == "fp32":
        part = {B.ACT_SILU: 2.0 ** -20, B.ACT_SIGMOID: 2.0 ** -20, B.ACT_GELU: 2.0 ** -19}.get(kind, 0.0) + torch.zeros_like(d)
    else:
        part = {B.ACT_SILU: d.abs() * 2.0 ** -23 + 2.0 ** -20, B.ACT_SIGMOID: d.abs() * 2.0 ** -23 + 2.0 ** -20,
                B.ACT_GELU: d * d * 2.0 ** -23 + 2.0 ** -19}.get(kind, torch.zeros_like(d))
    tol = torch.where(want == 0, 0, part * want.abs()) + (0 if kind <= B.ACT_RELU else (d.abs().clamp(max=200) + 1) * 2.0 ** -147)
    if dtype != "fp32":
        tol = tol + torch.finfo(h).eps / 2 * (want.abs() + tol)
    tol = tol + torch.finfo(h).smallest_normal * torch.finfo(h).eps / 2
    worst = (got - want).abs() / tol
    at = int(worst.argmax())
    assert torch.isfinite(got).all() and float(worst.max()) <= 1, f"v {float(d[at])}: {float(got[at])}, not {float(want[at])}: {float(worst.max()):.2f}"


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("kind", [B.ACT_SILU, B.ACT_GELU, B.ACT_SIGMOID])
def test_every_form_gives_the_same_bits(kind, dtype):
    h = R.TYPES[dtype]
    v = _values(h, "split")
    first = _outputs(v, "single", h, kind)
    for form in ("pair", "anywhere", "split"):
        assert torch.equal(_outputs(v, form, h, kind), first), form


@pytest.mark.parametrize("T,I,O", [(3, 16, 130), (300, 16, 700), (3, 11008, 4096)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kind", KINDS)
def test_a_nan_stays_a_nan(kind, dtype, T, I, O):
    h = R.TYPES[dtype]
    w, x = torch.ones((O, I), dtype=torch.int8, device="cuda"), torch.ones((T, I), dtype=torch.int8, device="cuda")
    sx, bias = torch.ones(T, device="cuda"), torch.zeros(O, dtype=h, device="cuda")
    sx[T - 1], bias[7] = float("nan"), float("nan")
    y = torch.empty((T, O), dtype=h, device="cuda")
    B.pipe_int8_linear(B.make_int8_desc(O, I, dtype=h), w, torch.ones(O, device="cuda"), x, sx, y, bias=bias, activation=kind)
    torch.cuda.synchronize()
    assert B.pipe_poll_status() == B.PIPE_OK
    nan = torch.isnan(y.cpu())
    want = torch.zeros_like(nan)
    want[T - 1] = True
    want[:, 7] = True
    assert torch.equal(nan, want)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_infinities(dtype, form):
    inf = float("inf")
    v = torch.tensor([inf, -inf] * 64)
    for kind, want in ((B.ACT_IDENTITY, [inf, -inf]), (B.ACT_RELU, [inf, 0]), (B.ACT_SIGMOID, [1, 0])):
        assert _outputs(v, form, R.TYPES[dtype], kind)[:2].tolist() == want
    for kind in (B.ACT_SILU, B.ACT_GELU):
        assert float(_outputs(v[::2], form, R.TYPES[dtype], kind)[0]) == inf
