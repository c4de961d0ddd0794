"""The 8-bit integer layers on the GPU: rows to int8, products, products grouped by expert."""
import pytest
import torch

from paper_2311_15806_b200 import binding as B
from tests import int8_reference as R

pytestmark = pytest.mark.gpu


def _gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def _ok():
    torch.cuda.synchronize()
    assert B.pipe_poll_status() == B.PIPE_OK


# ---- rows to int8 -----------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("N,I,ldx,ldc", [(1, 1, 1, 16), (3, 5, 7, 5), (9, 33, 33, 48), (8, 256, 256, 256), (17, 1000, 1008, 1000), (5, 1024, 1024, 1024), (4, 1025, 1025, 1040),
                                         (7, 4096, 4100, 4096), (3, 4099, 4099, 4112), (2, 16384, 16384, 16384), (2, 16390, 16396, 16400), (1, 70001, 70001, 70016)])
def test_rows_to_int8(dtype, N, I, ldx, ldc):
    gen = _gen(N + I)
    x = (torch.randn((N, ldx), generator=gen) * torch.exp2(torch.rand((N, 1), generator=gen) * 12 - 6)).to(R.TYPES[dtype])
    x[0, :I] = 0
    if N > 2:
        x[2, :I] = (torch.randint(-254, 255, (I,), generator=gen) / 2).to(x.dtype)     # ties: the scale is 1
        x[2, 0] = 127
    codes = torch.full((N, ldc), 99, dtype=torch.int8, device="cuda")
    scales = torch.full((N,), -1.0, device="cuda")
    values = torch.full((N, I + 3), -1.0, device="cuda")
    B.pipe_int8_quantize(x.cuda()[:, :I], codes[:, :I], scales, values=values[:, :I])
    _ok()
    s, q = R.quantized(x[:, :I])
    assert torch.equal(scales.cpu(), s) and torch.equal(codes[:, :I].cpu(), q)
    assert torch.equal(values[:, :I].cpu(), (q.double() * s.double()[:, None]).float())
    assert (codes[:, I:] == 99).all() and (values[:, I:] == -1).all()
    only = torch.full((N, ldc), 99, dtype=torch.int8, device="cuda")                    # without values: the same codes
    B.pipe_int8_quantize(x.cuda()[:, :I], only[:, :I], scales)
    _ok()
    assert torch.equal(only, codes)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_of_any_size_and_alignment(dtype):
    """Magnitudes from the smallest to the largest of the type, rows that start anywhere."""
    gen = _gen(3)
    f = torch.finfo(R.TYPES[dtype])
    x = torch.randn((40, 301), generator=gen).double() * torch.exp2(torch.linspace(-140, 120, 40).double())[:, None]
    x[5] = f.max
    x[6] = f.smallest_normal * f.eps                  # the scale is 0 or has few bits
    x[7] = 0
    x[7, 11] = -f.smallest_normal * f.eps * 300
    x = x.clamp(f.min, f.max).to(R.TYPES[dtype])
    for shift in range(1, 5):
        flat = torch.zeros(40 * 301 + shift, dtype=x.dtype, device="cuda")
        at = flat[shift:].view(40, 301)
        at.copy_(x)
        raw = torch.zeros(40 * 301 + shift, dtype=torch.int8, device="cuda")
        scales = torch.empty(40, device="cuda")
        B.pipe_int8_quantize(at, raw[shift:].view(40, 301), scales)
        _ok()
        s, q = R.quantized(x)
        assert torch.equal(scales.cpu(), s) and torch.equal(raw[shift:].view(40, 301).cpu(), q) and (raw[:shift] == 0).all()


def test_gathered_rows_and_slots_behind_the_last():
    gen = _gen(4)
    T, N, I = 37, 90, 200
    x = torch.randn((T, I), generator=gen).to(torch.float16)
    rows = torch.randint(0, T, (N,), generator=gen, dtype=torch.int32)
    rows[3], rows[8], rows[70] = -1, T, 2 ** 31 - 1
    for count in (None, 0, 1, 64, N, N + 5, -3):
        codes = torch.full((N, 208), 99, dtype=torch.int8, device="cuda")
        scales = torch.full((N,), -1.0, device="cuda")
        values = torch.full((N, I), -1.0, device="cuda")
        c = None if count is None else torch.tensor([count], dtype=torch.int32, device="cuda")
        B.pipe_int8_quantize(x.cuda(), codes[:, :I], scales, rows=rows.cuda(), count=c, values=values)
        _ok()
        n = N if count is None else min(max(count, 0), N)
        inside = (rows >= 0) & (rows < T)
        want = torch.where(inside[:, None], x[rows.clamp(0, T - 1).long()], torch.zeros((), dtype=x.dtype))
        s, q = R.quantized(want)
        assert torch.equal(scales[:n].cpu(), s[:n]) and torch.equal(codes[:n, :I].cpu(), q[:n])
        assert (scales[n:] == -1).all() and (codes[n:] == 99).all() and (values[n:] == -1).all()
    # no tokens at all: every row is one of zeros
    B.pipe_int8_quantize(x.cuda()[:0], codes[:, :I], scales, rows=rows.cuda())
    _ok()
    assert (codes[:, :I] == 0).all() and (scales == 0).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("dtype,I", [("bf16", 40), ("fp16", 3000), ("fp32", 20000)])
def test_numbers_that_are_none(bad, dtype, I):
    x = torch.randn((6, I), generator=_gen(5)).to(R.TYPES[dtype])
    s, q = R.quantized(x)
    x[3, I - 1] = bad
    codes, scales = torch.zeros((6, I), dtype=torch.int8, device="cuda"), torch.zeros(6, device="cuda")
    B.pipe_int8_quantize(x.cuda(), codes, scales)
    torch.cuda.synchronize()
    assert B.pipe_poll_status() == B.PIPE_ERR_NONFINITE and B.pipe_poll_status() == B.PIPE_OK
    others = [0, 1, 2, 4, 5]
    assert torch.equal(codes.cpu()[others], q[others]) and torch.equal(scales.cpu()[others], s[others])
    rows = torch.tensor(others, dtype=torch.int32, device="cuda")     # not read: not reported
    B.pipe_int8_quantize(x.cuda(), codes[:5], scales[:5], rows=rows)
    _ok()


# ---- products -----------------------------------------------------------------------------------------------------------------------
def _pitched(t, pitch):
    out = torch.full((*t.shape[:-1], pitch), 77, dtype=t.dtype, device="cuda")[..., :t.shape[-1]]
    return out.copy_(t)


def _layer(gen, E, O, I, pitch=None):
    w = torch.randint(-128, 128, (E, O, I), generator=gen, dtype=torch.int8)
    return w, torch.rand((E, O), generator=gen) * 0.01 + 0.001, _pitched(w, pitch or I + 15 & ~15)


def _linear(T, O, I, dtype, kind, bias, seed, ldw=None, ldx=None, ldy=None):
    gen, h = _gen(seed), R.TYPES[dtype]
    w, sw, wd = _layer(gen, 1, O, I, ldw)
    x = torch.randint(-128, 128, (T, I), generator=gen, dtype=torch.int8)
    sx = torch.rand((T,), generator=gen) * 0.05 + 0.001
    b = (torch.randn((O,), generator=gen)).to(h) if bias else None
    ldy = ldy or O
    y = torch.full((T, ldy), -7.0, dtype=h, device="cuda")
    d = B.make_int8_desc(O, I, dtype=h)
    B.pipe_int8_linear(d, wd, sw.cuda(), _pitched(x, ldx or I + 15 & ~15), sx.cuda(), y[:, :O], bias=b.cuda() if bias else None, activation=kind)
    _ok()
    R.check_product(y[:, :O], x, sx, w[0], sw[0], b, kind, dtype, f"T {T} O {O} I {I} {dtype}")
    assert (y[:, O:] == -7).all()


@pytest.mark.parametrize("T", [1, 2, 7, 8, 9, 15, 16, 17, 31, 32, 33, 64, 65, 100, 127, 128, 129, 200, 255, 256, 257, 300, 511, 513])
@pytest.mark.parametrize("O,I", [(200, 264), (136, 1000)])
def test_rows_of_every_number(T, O, I):
    _linear(T, O, I, ["bf16", "fp16", "fp32"][T % 3], T % 5, T % 2 == 0, T + O)


@pytest.mark.parametrize("O,I", [(1, 1), (1, 16), (2, 3), (7, 33), (8, 127), (63, 128), (64, 129), (127, 255), (128, 4096), (129, 96), (255, 500), (256, 513), (257, 640), (1000, 31), (4001, 177)])
@pytest.mark.parametrize("T", [1, 5, 40, 270])
def test_layers_of_every_size(T, O, I):
    _linear(T, O, I, ["fp32", "bf16", "fp16"][(O + I) % 3], (T + O) % 5, I % 2 == 0, O * 3 + I)


@pytest.mark.parametrize("T,O,I", [(1, 11008, 4096), (13, 4096, 11008), (600, 4096, 4096), (2048, 1408, 2048), (3, 50001, 512), (130, 2048, 2048), (2500, 3000, 700)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_large_layers(T, O, I, dtype):
    _linear(T, O, I, dtype, 2, True, T)


@pytest.mark.parametrize("kind", range(5))
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("T", [3, 150])
def test_activations(kind, dtype, T):
    _linear(T, 300, 320, dtype, kind, kind % 2 == 0, 11 + kind)


@pytest.mark.parametrize("T,ldw,ldx,ldy", [(2, 208, 224, 131), (50, 256, 192, 130), (300, 208, 4096, 257)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_pitches(T, ldw, ldx, ldy, dtype):
    _linear(T, 130, 190, dtype, 0, True, 5, ldw, ldx, ldy)


def test_outputs_that_start_anywhere():
    gen = _gen(8)
    for dtype, T, shift in (("bf16", 5, 1), ("fp16", 70, 3), ("fp32", 300, 1), ("bf16", 300, 5)):
        O, I, h = 77, 160, R.TYPES[dtype]
        w, sw, wd = _layer(gen, 1, O, I)
        x = torch.randint(-128, 128, (T, I), generator=gen, dtype=torch.int8)
        sx = torch.rand((T,), generator=gen)
        flat = torch.full((T * O + shift + 9,), -7.0, dtype=h, device="cuda")
        y = flat[shift:shift + T * O].view(T, O)
        B.pipe_int8_linear(B.make_int8_desc(O, I, dtype=h), wd, sw.cuda(), x.cuda(), sx.cuda(), y)
        _ok()
        R.check_product(y, x, sx, w[0], sw[0], None, 0, dtype)
        assert (flat[:shift] == -7).all() and (flat[shift + T * O:] == -7).all()


def test_the_largest_sums():
    """Codes of -128 on both sides at the greatest length: the sum is 2^31 - 2^14."""
    for T in (1, 40, 300):
        I = B.INT8_MAX_FEATURES
        w = torch.full((1, 20, I), -128, dtype=torch.int8)
        w[0, 3] = 127
        x = torch.full((T, I), -128, dtype=torch.int8)
        y = torch.empty((T, 20), device="cuda")
        B.pipe_int8_linear(B.make_int8_desc(20, I, dtype=torch.float32), _pitched(w, I + 15 & ~15), torch.ones(20, device="cuda"),
                           _pitched(x, I + 15 & ~15), torch.ones(T, device="cuda"), y)
        _ok()
        want = torch.full((T, 20), 16384.0 * I).double()
        want[:, 3] = -128.0 * 127 * I
        assert torch.equal(y.cpu(), want.float())


def test_a_row_does_not_depend_on_the_others():
    gen = _gen(9)
    O, I = 333, 1040
    _, sw, wd = _layer(gen, 1, O, I)
    x = torch.randint(-128, 128, (700, I), generator=gen, dtype=torch.int8).cuda()
    sx, d = torch.rand((700,), generator=gen).cuda(), B.make_int8_desc(O, I)
    whole = torch.empty((700, O), dtype=torch.bfloat16, device="cuda")
    B.pipe_int8_linear(d, wd, sw.cuda(), x, sx, whole, activation=3)
    for n in (1, 2, 16, 17, 64, 200, 257, 699):
        y = torch.empty((n, O), dtype=torch.bfloat16, device="cuda")
        B.pipe_int8_linear(d, wd, sw.cuda(), x[:n], sx[:n], y, activation=3)
        _ok()
        assert torch.equal(y, whole[:n]), n


def test_scales_of_any_size():
    """Zero, tiny and huge scales: the result is rounded like a product of binary32 numbers, never made NaN on the way."""
    gen = _gen(10)
    T, O, I = 20, 40, 64
    w, _, wd = _layer(gen, 1, O, I)
    x = torch.randint(-128, 128, (T, I), generator=gen, dtype=torch.int8)
    sw = torch.exp2(torch.linspace(-60, 60, O))
    sx = torch.exp2(torch.linspace(50, -50, T))
    sw[3], sx[4] = 0, 0
    y = torch.empty((T, O), device="cuda")
    B.pipe_int8_linear(B.make_int8_desc(O, I, dtype=torch.float32), wd, sw.cuda(), x.cuda(), sx.cuda(), y)
    _ok()
    R.check_product(y, x, sx, w[0], sw, None, 0, "fp32")


# ---- products grouped by expert -------------------------------------------------------------------------------------------------------
def _expert(E, O, I, dtype, counts, bias, kind, seed, spare=3, ldy=None, offsets=None):
    gen, h = _gen(seed), R.TYPES[dtype]
    w, sw, wd = _layer(gen, E, O, I)
    N = sum(counts) + spare
    off = torch.zeros(E + 1, dtype=torch.int32)
    off[1:] = torch.tensor(counts).cumsum(0)
    x = torch.randint(-128, 128, (N, I), generator=gen, dtype=torch.int8)
    sx = torch.rand((N,), generator=gen) * 0.05 + 0.001
    b = torch.randn((E, O), generator=gen).to(h) if bias else None
    y = torch.full((N, ldy or O), -7.0, dtype=h, device="cuda")
    B.pipe_int8_expert_linear(B.make_int8_desc(O, I, dtype=h, experts=E), wd, sw.cuda(), _pitched(x, I + 15 & ~15), sx.cuda(),
                              (off if offsets is None else offsets).cuda(), y[:, :O], bias=b.cuda() if bias else None, activation=kind)
    _ok()
    for e in range(E):
        lo, hi = int(off[e]), int(off[e + 1])
        R.check_product(y[lo:hi, :O], x[lo:hi], sx[lo:hi], w[e], sw[e], b[e] if bias else None, kind, dtype, f"expert {e}")
    assert (y[int(off[E]):] == -7).all() and (y[:, O:] == -7).all()


@pytest.mark.parametrize("counts", [[0], [1], [40], [0, 0, 0], [1, 0, 2], [0, 5, 0, 0, 17], [33, 1, 64, 0, 200], [300, 3, 0, 513], [16] * 8, [2, 0, 1, 0, 0, 1, 3, 0] * 8])
@pytest.mark.parametrize("dtype,O,I", [("bf16", 200, 264), ("fp16", 129, 33), ("fp32", 65, 512)])
def test_experts(counts, dtype, O, I):
    _expert(len(counts), O, I, dtype, counts, len(counts) % 2 == 0, len(counts) % 5, sum(counts) + O)


def test_many_experts():
    gen = _gen(12)
    _expert(64, 1408, 512, "bf16", torch.randint(0, 4, (64,), generator=gen).tolist(), False, 2, 1, ldy=1411)
    _expert(64, 256, 1408, "fp16", torch.randint(0, 190, (64,), generator=gen).tolist(), True, 0, 2)
    _expert(1024, 24, 48, "fp32", torch.randint(0, 3, (1024,), generator=gen).tolist(), True, 1, 3)
    _expert(8, 2048, 1024, "bf16", [700, 0, 3, 1500, 64, 256, 255, 257], False, 3, 4, spare=0)


@pytest.mark.parametrize("offsets,read_as", [([0, 4, 2, 9], [0, 4, 4, 9]), ([-5, 3, 100, 100], [0, 3, 12, 12]), ([6, 2, 1, 0], [6, 6, 6, 6]), ([2, 2, 5, 9], [2, 2, 5, 9])])
def test_offsets_out_of_order(offsets, read_as):
    gen = _gen(13)
    E, O, I, N = 3, 50, 80, 12
    w, sw, wd = _layer(gen, E, O, I)
    x = torch.randint(-128, 128, (N, I), generator=gen, dtype=torch.int8)
    sx = torch.rand((N,), generator=gen)
    y = torch.full((N, O), -7.0, device="cuda")
    B.pipe_int8_expert_linear(B.make_int8_desc(O, I, dtype=torch.float32, experts=E), wd, sw.cuda(), x.cuda(), sx.cuda(),
                              torch.tensor(offsets, dtype=torch.int32, device="cuda"), y)
    _ok()
    for e in range(E):
        lo, hi = read_as[e], read_as[e + 1]
        R.check_product(y[lo:hi], x[lo:hi], sx[lo:hi], w[e], sw[e], None, 0, "fp32")
    assert (y[:read_as[0]] == -7).all() and (y[read_as[E]:] == -7).all()


def test_an_experts_row_is_that_of_a_layer_alone():
    gen = _gen(14)
    E, O, I = 3, 140, 400
    _, sw, wd = _layer(gen, E, O, I)
    x = torch.randint(-128, 128, (90, I), generator=gen, dtype=torch.int8).cuda()
    sx = torch.rand((90,), generator=gen).cuda()
    off = torch.tensor([0, 10, 11, 90], dtype=torch.int32, device="cuda")
    y = torch.empty((90, O), dtype=torch.float16, device="cuda")
    B.pipe_int8_expert_linear(B.make_int8_desc(O, I, dtype=torch.float16, experts=E), wd, sw.cuda(), x, sx, off, y, activation=2)
    for e, (lo, hi) in enumerate(((0, 10), (10, 11), (11, 90))):
        one = torch.empty((hi - lo, O), dtype=torch.float16, device="cuda")
        B.pipe_int8_linear(B.make_int8_desc(O, I, dtype=torch.float16), wd[e], sw[e].cuda(), x[lo:hi], sx[lo:hi], one, activation=2)
        _ok()
        assert torch.equal(one, y[lo:hi])


# ---- used together ----------------------------------------------------------------------------------------------------------------
def test_a_layer_of_experts_from_router_to_sum():
    gen = _gen(15)
    T, k, E, I, O = 61, 3, 7, 272, 190
    W = (torch.randn((E, O, I), generator=gen) * 0.05).to(torch.bfloat16).cuda()
    x = torch.randn((T, I), generator=gen).to(torch.bfloat16).cuda()
    choice = torch.randint(-1, E, (T, k), generator=gen, dtype=torch.int32).cuda()
    mix = torch.softmax(torch.randn((T, k), generator=gen), 1).cuda()
    codes, scales = B.alloc_int8(O, I, experts=E)
    B.pipe_int8_quantize(W, codes, scales)
    i32 = dict(dtype=torch.int32, device="cuda")
    offsets, rows, slots = torch.empty(E + 1, **i32), torch.full((T * k,), -1, **i32), torch.empty((T, k), **i32)
    B.pipe_expert_rows(choice, E, offsets, rows, slots)
    xq, sx = B.alloc_int8(T * k, I)
    B.pipe_int8_quantize(x, xq, sx, rows=rows, count=offsets[E:])
    h = torch.zeros((T * k, O), dtype=torch.bfloat16, device="cuda")
    B.pipe_int8_expert_linear(B.make_int8_desc(O, I, experts=E), codes, scales, xq, sx, offsets, h, activation=B.ACT_SILU)
    out = torch.empty((T, O), dtype=torch.bfloat16, device="cuda")
    B.pipe_expert_combine(h, slots, mix, out)
    _ok()
    sw, wq = R.quantized(W)
    assert torch.equal(codes.cpu(), wq) and torch.equal(scales.cpu(), sw)
    st, xt = R.quantized(x)
    want, room = torch.zeros((T, O), dtype=torch.float64), torch.zeros((T, O), dtype=torch.float64)
    for t in range(T):
        for j in range(k):
            e = int(choice[t, j])
            if e >= 0:
                v, tol = R.product(xt[t:t + 1], st[t:t + 1], wq[e], sw[e], None, 2, "bf16")
                want[t] += float(mix[t, j]) * v[0]
                room[t] += float(mix[t, j]) * (tol[0] + 2.0 ** -22 * v[0].abs())
    room = room + 2.0 ** -8 * (want.abs() + room) + 1e-30
    assert ((out.cpu().double() - want).abs() <= room).all()


# ---- streams, captures, offsets past 31 bits ----------------------------------------------------------------------------------------
@pytest.mark.parametrize("T,O,I", [(3, 2048, 4096), (5, 300, 11008), (90, 1000, 640), (700, 2048, 512)])
def test_captured_and_replayed_and_on_two_streams_at_once(T, O, I):
    """One token's form, a split axis, single CTAs and pairs: the same bits from a graph, from another stream, from both streams at once."""
    gen = _gen(T)
    _, sw, wd = _layer(gen, 1, O, I)
    sw = sw.cuda()
    d = B.make_int8_desc(O, I)
    x = [torch.randn((T, I), generator=gen).to(torch.bfloat16).cuda() for _ in range(2)]
    q = [B.alloc_int8(T, I) for _ in range(2)]
    y = [torch.empty((T, O), dtype=torch.bfloat16, device="cuda") for _ in range(2)]

    def forward(i, stream=None):
        B.pipe_int8_quantize(x[i], *q[i], stream=stream)
        B.pipe_int8_linear(d, wd, sw, *q[i], y[i], activation=2, stream=stream)

    want = []
    for i in range(2):
        forward(i)
        want.append(y[i].clone())
        y[i].zero_()
    _ok()
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for i in range(2):
            forward(i, streams[i])
    _ok()
    assert torch.equal(y[0], want[0]) and torch.equal(y[1], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        forward(0)
        forward(0)
    x[0].copy_(x[1])
    for _ in range(3):
        graph.replay()
    _ok()
    assert torch.equal(y[0], want[1])


def test_weights_and_outputs_beyond_31_bits():
    gen = _gen(21)
    # rows of weights, and of an expert, that begin beyond 2^31 bytes
    O, I = 530000, 4112
    codes = torch.empty((O, I), dtype=torch.int8, device="cuda")
    codes.random_(-128, 128)
    sw = torch.rand(O, device="cuda") * 0.01
    for T in (2, 70):
        x = torch.randint(-128, 128, (T, I), generator=gen, dtype=torch.int8)
        sx = torch.rand((T,), generator=gen)
        y = torch.empty((T, O), dtype=torch.bfloat16, device="cuda")
        B.pipe_int8_linear(B.make_int8_desc(O, I), codes, sw, x.cuda(), sx.cuda(), y)
        _ok()
        for part in (slice(0, 300), slice(O - 300, O)):
            R.check_product(y[:, part], x, sx, codes[part], sw[part], None, 0, "bf16")
        half = torch.empty((T, O // 2), dtype=torch.float32, device="cuda")
        B.pipe_int8_expert_linear(B.make_int8_desc(O // 2, I, dtype=torch.float32, experts=2), codes.view(2, O // 2, I), sw, x.cuda(), sx.cuda(),
                                  torch.tensor([0, 1, T], dtype=torch.int32, device="cuda"), half)
        _ok()
        R.check_product(half[1:, -300:], x[1:], sx[1:], codes[-300:], sw[-300:], None, 0, "fp32")
    del codes, y, half
    # outputs beyond 2^31 values
    T, O, I = 70000, 32000, 16
    w, sw, wd = _layer(gen, 1, O, I)
    x = torch.randint(-128, 128, (T, I), generator=gen, dtype=torch.int8)
    sx = torch.rand((T,), generator=gen)
    y = torch.empty((T, O), dtype=torch.bfloat16, device="cuda")
    B.pipe_int8_linear(B.make_int8_desc(O, I), wd, sw.cuda(), x.cuda(), sx.cuda(), y)
    _ok()
    for part in (slice(0, 40), slice(T - 40, T)):
        R.check_product(y[part], x[part], sx[part], w[0], sw[0], None, 0, "bf16")


def test_rows_to_int8_far_apart():
    gen = _gen(22)
    I, pitch = 1003, (1 << 31) + 8
    flat = torch.empty(pitch + I, dtype=torch.bfloat16, device="cuda")
    x = torch.randn((2, I), generator=gen).to(torch.bfloat16)
    at = flat.as_strided((2, I), (pitch, 1))
    at.copy_(x)
    raw = torch.empty(pitch + I, dtype=torch.int8, device="cuda")
    codes, scales = raw.as_strided((2, I), (pitch, 1)), torch.empty(2, device="cuda")
    B.pipe_int8_quantize(at, codes, scales)
    _ok()
    s, q = R.quantized(x)
    assert torch.equal(codes.cpu(), q) and torch.equal(scales.cpu(), s)


def test_ties_of_16_bit_values():
    """Rows whose quotients come to halves by the few bits of their values: every multiple of a half up to the largest."""
    for dtype in ("bf16", "fp16"):
        x = torch.stack([torch.arange(-254, 255) * 0.5 * 2.0 ** e for e in range(-6, 4)])
        x = torch.cat([x, torch.arange(509).double().repeat(3, 1) * torch.tensor([[1.0], [0.375], [3.0]])]).to(R.TYPES[dtype])
        codes, scales = B.alloc_int8(x.shape[0], x.shape[1])
        values = torch.empty(x.shape, device="cuda")
        s, q = R.quantized(x)
        B.pipe_int8_quantize(x.cuda(), codes, scales)
        _ok()
        assert torch.equal(codes.cpu(), q) and torch.equal(scales.cpu(), s)
        B.pipe_int8_quantize(x.cuda(), codes, scales, values=values)
        _ok()
        assert torch.equal(codes.cpu(), q) and torch.equal(values.cpu(), (q.double() * s.double()[:, None]).float())


@pytest.mark.parametrize("T,O,I", [(5000, 50, 200), (3000, 64, 130), (2600, 1, 16), (9000, 65, 48)])
def test_narrow_layers_on_many_rows(T, O, I):
    _linear(T, O, I, "bf16", 1, True, T)


def test_narrow_experts_on_many_rows():
    _expert(3, 40, 96, "fp16", [700, 0, 2000], True, 2, 30)
    _expert(5, 8, 300, "fp32", [150, 151, 0, 149, 600], False, 0, 31)


@pytest.mark.parametrize("T,O,I", [(2095, 479, 230), (300, 1003, 96), (37, 501, 700), (13, 77, 5000)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_outputs_are_the_same_wherever_rows_begin(T, O, I, dtype):
    gen, h = _gen(T), R.TYPES[dtype]
    w, sw, wd = _layer(gen, 1, O, I)
    x = _pitched(torch.randint(-128, 128, (T, I), generator=gen, dtype=torch.int8), I + 15 & ~15)
    sx, b = torch.rand((T,), generator=gen).cuda() * 0.02, torch.randn((O,), generator=gen).to(h).cuda()
    got = []
    for ldy in (O + 15 & ~15, (O + 15 & ~15) + 2, O, O + 9):
        y = torch.full((T, ldy), -7.0, dtype=h, device="cuda")
        B.pipe_int8_linear(B.make_int8_desc(O, I, dtype=h), wd, sw.cuda(), x, sx, y[:, :O], bias=b, activation=2)
        _ok()
        assert (y[:, O:] == -7).all()
        got.append(y[:, :O].contiguous())
    R.check_product(got[0], x.cpu(), sx.cpu(), w[0], sw[0], b.cpu(), 2, dtype)
    assert all(torch.equal(g, got[0]) for g in got[1:])
