"""4-bit layers with group scales on the GPU: the quantizer bit for bit, the products against 64 bits."""
import pytest
import torch

from paper_2311_15806_b200 import binding as B
from tests import group_reference as R

pytestmark = pytest.mark.gpu
ACTS = [B.ACT_IDENTITY, B.ACT_RELU, B.ACT_SILU, B.ACT_GELU, B.ACT_SIGMOID]


def _gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def _ok():
    torch.cuda.synchronize()
    assert B.pipe_poll_status() == B.PIPE_OK


# ---- quantizer ------------------------------------------------------------------------------------------------------------------
def quantized64(w, g, h, asym):
    """scales [E, G, O], zeros, codes [E, O, I] of the definition; quotients in 64 bits, where ties and near ties are told apart."""
    E, O, I = w.shape
    v = w.float().view(E, O, I // g, g)
    if asym:
        lo, hi = v.amin(3).clamp(max=0), v.amax(3).clamp(min=0)
        s = ((hi - lo).double() / 15).float().to(h)
    else:
        s = (v.abs().amax(3).double() / 7).float().to(h)
    d = s.double()
    some = d > 0
    safe = torch.where(some, d, torch.ones_like(d))
    if asym:
        z = torch.where(some, torch.round(-lo.double() / safe).clamp(0, 15), torch.zeros_like(d))
        u = torch.where(some[..., None], (torch.round(v.double() / safe[..., None]) + z[..., None]).clamp(0, 15), z[..., None].expand(v.shape))
    else:
        z = torch.full_like(d, 8)
        u = torch.where(some[..., None], torch.round(v.double() / safe[..., None]).clamp(-7, 7) + 8, torch.full_like(v.double(), 8))
    return s.transpose(1, 2), z.transpose(1, 2).to(torch.uint8), u.view(E, O, I).long()


def _weights(gen, E, O, I, g, src):
    w = torch.randn((E, O, I), generator=gen) * 0.02
    w[:, ::3] = torch.round(w[:, ::3] * 400) / 400            # a coarse grid: many quotients on a tie
    w[0, 0, :g] = 0                                           # an empty group
    w[0, -1, :g] = 3e-8                                       # a scale at the end of fp16's range
    w[0, O // 2] = w[0, O // 2].abs()                         # one-sided groups
    return w.to({"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[src])


@pytest.mark.parametrize("asym", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("src", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("E,O,I,g", [(1, 1, 32, 32), (1, 17, 96, 32), (3, 5, 192, 64), (1, 33, 640, 128), (2, 130, 2080, 32)])
def test_quantizer_is_the_definition(E, O, I, g, src, dtype, asym):
    h = R.TYPES[dtype]
    w = _weights(_gen(O * I + g), E, O, I, g, src)
    desc = B.make_group_desc(O, I, g, dtype=h, asymmetric=asym, experts=E)
    codes, scales, zeros = B.alloc_group(desc)
    values = torch.full((E, O, I), float("nan"), device="cuda")
    B.pipe_group_quantize(desc, w.cuda(), codes, scales, zeros, values=values)
    _ok()
    s, z, u = quantized64(w, g, h, asym)
    assert torch.equal(scales.cpu().view(torch.int16), s.contiguous().view(torch.int16))
    if asym:
        assert torch.equal(zeros.cpu(), z)
    assert torch.equal(R.unpack(codes, I), u)
    assert torch.equal(values.cpu().double(), R.dense(u, s, z if asym else None, g))


@pytest.mark.parametrize("src", [torch.float32, torch.bfloat16])
def test_quantizer_on_pitched_and_unaligned_rows(src):
    O, I, g = 19, 160, 32
    big = (torch.randn((O, I + 11), generator=_gen(5)) * 0.05).to(src).cuda()
    for view in (big[:, :I], big[:, 3:3 + I]):                # rows at an odd pitch, rows that start anywhere
        desc = B.make_group_desc(O, I, g)
        codes, scales, _ = B.alloc_group(desc)
        values = torch.full((O, I + 5), -1.0, device="cuda")
        B.pipe_group_quantize(desc, view, codes, scales, values=values[:, 1:1 + I])
        _ok()
        s, _, u = quantized64(view.cpu()[None], g, torch.bfloat16, False)
        assert torch.equal(R.unpack(codes, I), u)
        assert torch.equal(values[:, 1:1 + I].cpu().double(), R.dense(u, s, None, g)[0])
        assert (values[:, 0] == -1).all() and (values[:, 1 + I:] == -1).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_quantizer_reports_what_is_not_finite(bad):
    w = torch.randn((8, 64), generator=_gen(1)).cuda()
    w[3, 40] = bad
    desc = B.make_group_desc(8, 64, 32)
    codes, scales, _ = B.alloc_group(desc)
    B.pipe_group_quantize(desc, w, codes, scales)
    assert B.pipe_poll_status() == B.PIPE_ERR_NONFINITE
    # a finite weight whose scale fp16 cannot hold
    desc = B.make_group_desc(8, 64, 32, dtype=torch.float16)
    codes, scales, _ = B.alloc_group(desc)
    w = torch.full((8, 64), 1e6, device="cuda")
    B.pipe_group_quantize(desc, w, codes, scales)
    assert B.pipe_poll_status() == B.PIPE_ERR_NONFINITE
    assert B.pipe_poll_status() == B.PIPE_OK


# ---- products ---------------------------------------------------------------------------------------------------------------------
def _linear(O, I, g, T, dtype, asym, bias, kind, seed, ldx=None, ldy=None):
    gen, h = _gen(seed), R.TYPES[dtype]
    u, s, z = R.random_layer(gen, 1, O, I, g, dtype, asym)
    ldx, ldy = ldx or I, ldy or O
    x = torch.randn((T, ldx), generator=gen).to(h)
    b = torch.randn((O,), generator=gen).to(h) if bias else None
    y = torch.full((T, ldy), 7.0, dtype=h, device="cuda")
    desc = B.make_group_desc(O, I, g, dtype=h, asymmetric=asym)
    xd = x.cuda()
    B.pipe_group_linear(desc, R.pack(u).cuda(), s.cuda(), None if z is None else z.cuda(), xd[:, :I], y[:, :O],
                        bias=None if b is None else b.cuda(), activation=kind)
    _ok()
    W = R.dense(u, s, z, g)[0]
    R.check_product(y[:, :O], x[:, :I], W, b, kind, dtype, g, R.few(T), f"O {O} I {I} g {g} T {T} {dtype}")
    assert (y[:, O:] == 7).all()


@pytest.mark.parametrize("dtype,asym,g", [("bf16", False, 128), ("bf16", True, 32), ("fp16", False, 64), ("fp16", True, 128)])
@pytest.mark.parametrize("T", [1, 2, 7, 8, 9, 16, 17, 31, 33, 64, 65, 127, 130, 257, 300])
def test_linear_over_token_counts(T, dtype, asym, g):
    _linear(272, 640, g, T, dtype, asym, True, B.ACT_IDENTITY, T)


@pytest.mark.parametrize("O,I,g", [(1, 32, 32), (1, 128, 128), (7, 96, 32), (15, 64, 64), (129, 160, 32), (255, 192, 64), (256, 256, 128), (385, 2080, 32),
                                   (64, 4160, 64), (2049, 384, 128)])
@pytest.mark.parametrize("T", [1, 13, 40])
def test_linear_over_layer_sizes(O, I, g, T):
    _linear(O, I, g, T, "bf16", O % 2 == 0, O % 3 == 0, B.ACT_IDENTITY, O + I)
    _linear(O, I, g, T, "fp16", O % 2 == 1, O % 3 != 0, B.ACT_IDENTITY, O + I + 1)


@pytest.mark.parametrize("kind", ACTS)
@pytest.mark.parametrize("T", [3, 50])
def test_linear_activations(kind, T):
    _linear(200, 256, 64, T, "bf16", False, True, kind, 17 + kind)


@pytest.mark.parametrize("T", [1, 5, 16, 90])
@pytest.mark.parametrize("ldx,ldy", [(328, 201), (320, 204), (512, 1000)])
def test_linear_on_pitched_rows(T, ldx, ldy):
    _linear(200, 320, 32, T, "fp16", True, True, B.ACT_IDENTITY, T, ldx, ldy)


@pytest.mark.parametrize("T", [1, 16, 200])
def test_linear_long_reduction_and_many_channels(T):
    _linear(96, 11008, 128, T, "bf16", False, False, B.ACT_IDENTITY, 3)
    _linear(11008, 128, 128, T, "bf16", True, False, B.ACT_IDENTITY, 4)


@pytest.mark.parametrize("O,I,g,T", [(11008, 256, 64, 700), (2500, 640, 128, 2049), (130, 96, 32, 20001), (5003, 352, 32, 1000)])
def test_linear_with_more_tiles_than_sms(O, I, g, T):
    _linear(O, I, g, T, "bf16", False, True, B.ACT_IDENTITY, O)
    _linear(O, I, g, T, "fp16", True, False, B.ACT_SIGMOID, O + 1)


@pytest.mark.parametrize("T", [4, 100])
def test_a_token_that_is_not_finite_stays_alone(T):
    gen = _gen(9)
    u, s, z = R.random_layer(gen, 1, 70, 256, 32, "bf16", True)
    x = torch.randn((T, 256), generator=gen).to(torch.bfloat16)
    bad = x.clone()
    bad[1] = float("nan")
    bad[T - 1, 5] = float("inf")
    desc = B.make_group_desc(70, 256, 32, asymmetric=True)
    ys = []
    for v in (x, bad):
        y = torch.empty((T, 70), dtype=torch.bfloat16, device="cuda")
        B.pipe_group_linear(desc, R.pack(u).cuda(), s.cuda(), z.cuda(), v.cuda(), y)
        ys.append(y.cpu())
    _ok()
    same = [t for t in range(T) if t not in (1, T - 1)]
    assert torch.equal(ys[0][same], ys[1][same])
    assert torch.isnan(ys[1][1]).all() and not torch.isfinite(ys[1][T - 1]).all()


def test_scales_that_are_zero_and_large():
    gen = _gen(11)
    u, s, _ = R.random_layer(gen, 1, 48, 128, 64, "bf16", False)
    s[0, 0, ::2] = 0
    s[0, 1, ::3] = 2.0 ** 60
    x = torch.randn((20, 128), generator=gen).to(torch.bfloat16)
    desc = B.make_group_desc(48, 128, 64)
    W = R.dense(u, s, None, 64)[0]
    for T in (2, 20):
        y = torch.empty((T, 48), dtype=torch.bfloat16, device="cuda")
        B.pipe_group_linear(desc, R.pack(u).cuda(), s.cuda(), None, x[:T].cuda(), y)
        _ok()
        R.check_product(y, x[:T], W, None, 0, "bf16", 64, R.few(T))


def test_no_tokens_is_no_launch():
    desc = B.make_group_desc(64, 128, 32)
    codes, scales, _ = B.alloc_group(desc)
    n = B.pipe_launch_count()
    B.pipe_group_linear(desc, codes, scales, None, torch.empty((0, 128), dtype=torch.bfloat16, device="cuda"),
                        torch.empty((0, 64), dtype=torch.bfloat16, device="cuda"))
    assert B.pipe_launch_count() == n


@pytest.mark.parametrize("T", [1, 12, 80])
def test_linear_is_the_same_every_time_and_in_a_graph(T):
    gen = _gen(T)
    desc = B.make_group_desc(1000, 2048, 128)
    u, s, _ = R.random_layer(gen, 1, 1000, 2048, 128, "bf16", False)
    codes, s = R.pack(u).cuda(), s.cuda()
    x = torch.randn((T, 2048), generator=gen).to(torch.bfloat16).cuda()
    ys = [torch.empty((T, 1000), dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    B.pipe_group_linear(desc, codes, s, None, x, ys[0])
    B.pipe_group_linear(desc, codes, s, None, x, ys[1])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.pipe_group_linear(desc, codes, s, None, x, ys[2])
    ys[2].zero_()
    g.replay()
    _ok()
    assert torch.equal(ys[0], ys[1]) and torch.equal(ys[0], ys[2])
    x.mul_(2)                                                 # a replay reads what the buffers hold then
    g.replay()
    B.pipe_group_linear(desc, codes, s, None, x, ys[0])
    _ok()
    assert torch.equal(ys[0], ys[2])


def test_calls_on_two_streams_at_once():
    """No call shares anything with another: two layers on two streams, and on the default one, give what they give alone."""
    gen = _gen(31)
    layers = []
    for O, I, g, asym in ((1500, 2048, 128, False), (700, 4096, 32, True)):
        u, s, z = R.random_layer(gen, 1, O, I, g, "bf16", asym)
        layers.append((B.make_group_desc(O, I, g, asymmetric=asym), R.pack(u).cuda(), s.cuda(), None if z is None else z.cuda()))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for T in (1, 12, 40, 300):
        xs = [torch.randn((T, d[0].in_features), generator=gen).to(torch.bfloat16).cuda() for d in layers]
        alone = [torch.empty((T, d[0].out_features), dtype=torch.bfloat16, device="cuda") for d in layers]
        for d, x, y in zip(layers, xs, alone):
            B.pipe_group_linear(*d, x, y)
        torch.cuda.synchronize()
        both = [[torch.empty_like(y) for _ in range(8)] for y in alone]
        for i in range(8):
            for k, st in enumerate(streams):
                B.pipe_group_linear(*layers[k], xs[k], both[k][i], stream=st)
        _ok()
        for k in range(2):
            assert all(torch.equal(alone[k], y) for y in both[k])


def test_quantize_then_multiply_without_a_synchronization():
    """The weights of every call are made by the call before it on the same stream."""
    gen = _gen(2)
    O, I, g = 512, 1024, 64
    desc = B.make_group_desc(O, I, g)
    codes, scales, _ = B.alloc_group(desc)
    ws = [(torch.randn((O, I), generator=gen) * 0.05).cuda() for _ in range(4)]
    for T in (1, 16, 40):
        x = torch.randn((T, I), generator=gen).to(torch.bfloat16).cuda()
        ys = []
        for w in ws:
            B.pipe_group_quantize(desc, w, codes, scales)
            y = torch.empty((T, O), dtype=torch.bfloat16, device="cuda")
            B.pipe_group_linear(desc, codes, scales, None, x, y)
            ys.append(y)
        _ok()
        for w, y in zip(ws, ys):
            s, _, u = quantized64(w.cpu()[None], g, torch.bfloat16, False)
            R.check_product(y, x, R.dense(u, s, None, g)[0], None, 0, "bf16", g, R.few(T))


def test_residual_orders_add_up():
    """The framework's expansion with group scales: the second layer quantizes what the first leaves; two products come closer to
    the unquantized one than one does."""
    gen = _gen(6)
    O, I, g, T = 128, 512, 32, 4
    W = (torch.randn((O, I), generator=gen) * 0.02).cuda()
    desc = B.make_group_desc(O, I, g, dtype=torch.float16)
    x = torch.randn((T, I), generator=gen).half().cuda()
    r, got = W, []
    total = torch.zeros((T, O), dtype=torch.float64)
    for _ in range(2):
        codes, scales, _z = B.alloc_group(desc)
        values = torch.empty_like(W)
        B.pipe_group_quantize(desc, r, codes, scales, values=values)
        y = torch.empty((T, O), dtype=torch.float16, device="cuda")
        B.pipe_group_linear(desc, codes, scales, None, x, y)
        r = r - values
        total = total + y.cpu().double()
        got.append(float((total - x.cpu().double() @ W.cpu().double().t()).norm()))
    _ok()
    assert got[1] < got[0] / 4   # a second order divides the error by 2 qmax = 14, but for the roundings of fp16
