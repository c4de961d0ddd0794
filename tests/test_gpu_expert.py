"""Products grouped by expert on the GPU, with the sort of the rows before and the sum behind them."""
import pytest
import torch

from paper_2311_15806_b200 import binding as B
from tests import group_reference as R

pytestmark = pytest.mark.gpu


def _gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def _ok():
    torch.cuda.synchronize()
    assert B.pipe_poll_status() == B.PIPE_OK


def sorted_rows(choice, E):
    T, k = choice.shape
    offsets, rows, slots = [0], [], torch.full((T, k), -1, dtype=torch.int32)
    flat = choice.reshape(-1).tolist()
    by = [[] for _ in range(E)]
    for i, e in enumerate(flat):
        if 0 <= e < E:
            by[e].append(i)
    for members in by:
        for i in members:
            slots[i // k, i % k] = len(rows)
            rows.append(i // k)
        offsets.append(len(rows))
    return torch.tensor(offsets, dtype=torch.int32), torch.tensor(rows, dtype=torch.int32), slots


@pytest.mark.parametrize("T,k,E", [(1, 1, 1), (1, 1, 1024), (3, 2, 5), (31, 1, 2), (33, 3, 64), (100, 8, 361), (1000, 8, 512), (1024, 8, 8), (1025, 8, 8),
                                   (5000, 6, 1024), (40000, 2, 3)])
def test_rows_by_expert(T, k, E):
    gen = _gen(T + E)
    choice = torch.randint(-1, E + 1, (T, k), generator=gen, dtype=torch.int32)   # some outside on either side, the same one twice
    choice[T // 2] = 0
    offsets = torch.full((E + 1,), -7, dtype=torch.int32, device="cuda")
    rows = torch.full((T * k,), -7, dtype=torch.int32, device="cuda")
    slots = torch.full((T, k), -7, dtype=torch.int32, device="cuda")
    B.pipe_expert_rows(choice.cuda(), E, offsets, rows, slots)
    _ok()
    o, r, s = sorted_rows(choice, E)
    assert torch.equal(offsets.cpu(), o) and torch.equal(slots.cpu(), s)
    n = r.numel()
    assert torch.equal(rows.cpu()[:n], r) and (rows.cpu()[n:] == -7).all()


def test_rows_of_no_tokens_and_of_one_expert():
    offsets = torch.full((5,), 9, dtype=torch.int32, device="cuda")
    e = torch.empty((0, 2), dtype=torch.int32, device="cuda")
    B.pipe_expert_rows(e, 4, offsets, torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty((0, 2), dtype=torch.int32, device="cuda"))
    _ok()
    assert (offsets == 0).all()
    T, k = 700, 3
    choice = torch.full((T, k), 2, dtype=torch.int32, device="cuda")
    rows, slots = torch.empty(T * k, dtype=torch.int32, device="cuda"), torch.empty((T, k), dtype=torch.int32, device="cuda")
    B.pipe_expert_rows(choice, 4, offsets, rows, slots)
    _ok()
    assert offsets.tolist() == [0, 0, 0, T * k, T * k]
    assert torch.equal(slots.cpu().reshape(-1), torch.arange(T * k, dtype=torch.int32))


def _expert(E, O, I, g, dtype, asym, counts, T, gather, bias, kind, seed, spare=3, ldx=None, ldy=None):
    """counts: the rows of every expert; `spare` rows behind them that have to stay."""
    gen, h = _gen(seed), R.TYPES[dtype]
    u, s, z = R.random_layer(gen, E, O, I, g, dtype, asym)
    n = sum(counts)
    N = n + spare
    offsets = torch.zeros(E + 1, dtype=torch.int32)
    offsets[1:] = torch.tensor(counts).cumsum(0)
    T = T if gather else N
    ldx, ldy = ldx or I, ldy or O
    x = torch.randn((T, ldx), generator=gen).to(h)
    rows = torch.randint(0, T, (N,), generator=gen, dtype=torch.int32) if gather else None
    b = torch.randn((E, O), generator=gen).to(h) if bias else None
    y = torch.full((N, ldy), 7.0, dtype=h, device="cuda")
    desc = B.make_group_desc(O, I, g, dtype=h, asymmetric=asym, experts=E)
    cu = lambda t: None if t is None else t.cuda()  # noqa: E731
    xd = x.cuda()
    B.pipe_expert_linear(desc, cu(R.pack(u)), cu(s), cu(z), xd[:, :I], cu(offsets), y[:, :O], rows=cu(rows), bias=cu(b), activation=kind)
    _ok()
    few = R.few(-(-N // E))
    W = R.dense(u, s, z, g)
    for e in range(E):
        lo, hi = int(offsets[e]), int(offsets[e + 1])
        xe = x[lo:hi] if rows is None else x[rows[lo:hi].long()]
        R.check_product(y[lo:hi, :O], xe[:, :I], W[e], None if b is None else b[e], kind, dtype, g, few, f"expert {e}: rows {lo}..{hi}")
    assert (y[n:] == 7).all() and (y[:, O:] == 7).all()


@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("dtype,asym,g", [("bf16", False, 128), ("fp16", True, 32), ("bf16", True, 64)])
@pytest.mark.parametrize("counts", [[1], [0, 1, 0], [3, 0, 0, 9, 1], [17, 40, 0, 8], [0, 0, 0, 0], [100, 1, 0, 300], [64, 128, 256], [5] * 40, [513, 2]])
def test_experts_over_ragged_sizes(counts, dtype, asym, g, gather):
    _expert(len(counts), 144, 384, g, dtype, asym, counts, 50, gather, True, B.ACT_SILU, len(counts) + g)


@pytest.mark.parametrize("O,I,g", [(1, 32, 32), (129, 160, 32), (300, 128, 128), (256, 2112, 64)])
@pytest.mark.parametrize("counts", [[2, 0, 5], [30, 0, 71]])
def test_experts_over_layer_sizes(O, I, g, counts):
    _expert(3, O, I, g, "bf16", False, counts, 29, True, False, B.ACT_IDENTITY, O)
    _expert(3, O, I, g, "fp16", True, counts, 29, False, True, B.ACT_RELU, O + 1, ldx=I + 8, ldy=O + 3)


@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("E,O,mean", [(64, 401, 20), (64, 400, 40), (32, 514, 100), (12, 1100, 300), (9, 2051, 260)])
def test_experts_with_more_tiles_than_sms(E, O, mean, gather):
    """Enough tiles for pairs of SMs and for several tiles each, at every tile width; experts without rows among them."""
    gen = _gen(E + O)
    counts = [0 if e % 7 == 3 else int(v) for e, v in enumerate(torch.randint(1, 2 * mean, (E,), generator=gen))]
    _expert(E, O, 160, 32, "bf16", O % 2 == 0, counts, 333, gather, True, B.ACT_SILU, O)
    _expert(E, O, 256, 128, "fp16", O % 2 == 1, counts, 333, gather, False, B.ACT_IDENTITY, O + 1)


@pytest.mark.parametrize("E,O,I,g", [(40, 1500, 256, 64), (64, 1411, 2048, 128), (24, 5000, 96, 32)])
def test_few_rows_on_many_tiles(E, O, I, g):
    """The kernel for few rows at each height of its tiles, one to seventeen rows an expert, some of them none."""
    gen = _gen(E * O)
    counts = [0 if e % 5 == 2 else int(v) for e, v in enumerate(torch.randint(1, 6, (E,), generator=gen))]
    _expert(E, O, I, g, "bf16", False, counts, 20, True, True, B.ACT_SILU, O)
    counts[1] = 17
    _expert(E, O, I, g, "fp16", True, counts, 20, False, False, B.ACT_GELU, O + 1)
    _expert(E, O, I, g, "bf16", True, [9 + e % 7 for e in range(E)], 20, True, False, B.ACT_IDENTITY, O + 2)


@pytest.mark.parametrize("counts", [[1], [16], [17], [200]])
def test_one_expert_is_a_plain_layer(counts):
    _expert(1, 130, 160, 32, "bf16", True, counts, 40, False, True, B.ACT_RELU, counts[0])
    _expert(1, 130, 2176, 128, "fp16", False, counts, 40, True, True, B.ACT_IDENTITY, counts[0] + 1)


@pytest.mark.parametrize("N", [3, 500])
def test_rows_without_any_tokens_are_sigma_of_the_bias(N):
    """T = 0: every row index lies outside, every row reads as zeros."""
    gen = _gen(N)
    E, O, I, g = 2, 37, 64, 32
    u, s, _ = R.random_layer(gen, E, O, I, g, "bf16", False)
    b = torch.randn((E, O), generator=gen).to(torch.bfloat16)
    for rows in (None, torch.zeros(N, dtype=torch.int32, device="cuda")):
        y = torch.full((N, O), 7.0, dtype=torch.bfloat16, device="cuda")
        B.pipe_expert_linear(B.make_group_desc(O, I, g, experts=E), R.pack(u).cuda(), s.cuda(), None, torch.empty((0, I), dtype=torch.bfloat16, device="cuda"),
                             torch.tensor([0, 1, N - 1], dtype=torch.int32).cuda(), y, rows=rows, bias=b.cuda(), activation=B.ACT_RELU)
        _ok()
        assert torch.equal(y[:1].cpu(), b[:1].clamp(min=0)) and torch.equal(y[1:N - 1].cpu(), b[1:].clamp(min=0).expand(N - 2, O)) and (y[N - 1] == 7).all()


def test_more_experts_than_a_warp_looks_at():
    gen = _gen(3)
    counts = torch.randint(0, 3, (1024,), generator=gen).tolist()
    _expert(1024, 16, 32, 32, "bf16", False, counts, 64, True, True, B.ACT_IDENTITY, 5)
    counts = [0] * 1000 + [40] * 24
    _expert(1024, 16, 32, 32, "bf16", False, counts, 64, True, True, B.ACT_IDENTITY, 5, spare=20000)


@pytest.mark.parametrize("N", [6, 200])
def test_bad_offsets_and_rows_stay_in_bounds(N):
    """Offsets are clamped to the rows there are, a row index outside the tokens reads as zeros."""
    gen = _gen(8)
    E, O, I, g, T = 2, 40, 64, 32, 5
    u, s, _ = R.random_layer(gen, E, O, I, g, "bf16", False)
    x = torch.randn((T, I), generator=gen).to(torch.bfloat16)
    rows = torch.zeros(N, dtype=torch.int32)
    rows[1], rows[2], rows[3] = -1, T, 2 ** 31 - 1
    y = torch.full((N, O), 7.0, dtype=torch.bfloat16, device="cuda")
    desc = B.make_group_desc(O, I, g, experts=E)
    b = torch.randn((E, O), generator=gen).to(torch.bfloat16)
    B.pipe_expert_linear(desc, R.pack(u).cuda(), s.cuda(), None, x.cuda(), torch.tensor([-5, 4, 10 ** 6], dtype=torch.int32).cuda(), y, rows=rows.cuda(), bias=b.cuda())
    _ok()
    W = R.dense(u, s, None, g)
    xe = torch.zeros((N, I), dtype=torch.bfloat16)
    for i in range(N):
        if 0 <= rows[i] < T:
            xe[i] = x[rows[i]]
    R.check_product(y[:4], xe[:4], W[0], b[0], 0, "bf16", g, R.few(N // 2))
    R.check_product(y[4:], xe[4:], W[1], b[1], 0, "bf16", g, R.few(N // 2))


@pytest.mark.parametrize("scale", [1, 10])
@pytest.mark.parametrize("offsets", [[0, 30, 10, 40, 20], [40, 30, 20, 10, 0], [0, 25] + [3] * 35 + [40, 38, 39], [0, -7, 4, 2, 99, 8, 8]])
def test_offsets_out_of_order_count_as_the_highest_before_them(offsets, scale):
    """No row gets two experts' results: the offsets in use are the running maximum of the clamped ones."""
    gen = _gen(9)
    E, O, I, g, N = len(offsets) - 1, 72, 96, 32, 40 * scale
    off = torch.tensor(offsets) * scale
    used = torch.cummax(off.clamp(0, N), 0).values
    u, s, _ = R.random_layer(gen, E, O, I, g, "bf16", False)
    x = torch.randn((N, I), generator=gen).to(torch.bfloat16)
    y = torch.full((N, O), 7.0, dtype=torch.bfloat16, device="cuda")
    B.pipe_expert_linear(B.make_group_desc(O, I, g, experts=E), R.pack(u).cuda(), s.cuda(), None, x.cuda(), off.to(torch.int32).cuda(), y)
    _ok()
    W = R.dense(u, s, None, g)
    for e in range(E):
        a, b = int(used[e]), int(used[e + 1])
        if a < b:
            R.check_product(y[a:b], x[a:b], W[e], None, 0, "bf16", g, R.few((N + E - 1) // E))
    for a, b in ((0, int(used[0])), (int(used[-1]), N)):
        assert torch.all(y[a:b].cpu() == 7.0)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("T,k,O,ldy,ldo", [(1, 1, 1, 1, 1), (5, 2, 64, 64, 64), (7, 8, 72, 80, 88), (33, 3, 65, 65, 67), (200, 6, 520, 520, 520), (9, 17, 24, 24, 24)])
def test_combine(T, k, O, ldy, ldo, dtype):
    gen, h = _gen(T * k + O), R.TYPES[dtype]
    N = T * k
    y = torch.randn((N, ldy), generator=gen).to(h)
    slots = torch.randperm(N, generator=gen).view(T, k).to(torch.int32)
    slots[0, 0] = -1
    slots[T // 2, k - 1] = N
    w = torch.rand((T, k), generator=gen)
    out = torch.full((T, ldo), 7.0, dtype=h, device="cuda")
    B.pipe_expert_combine(y.cuda()[:, :O], slots.cuda(), w.cuda(), out[:, :O])
    _ok()
    inside = (slots >= 0) & (slots < N)
    terms = torch.where(inside[..., None], y.double()[slots.clamp(0, N - 1).long()][..., :O], torch.zeros(())) * w.double()[..., None]
    want, size = terms.sum(1), terms.abs().sum(1)
    eps = torch.finfo(h).eps / 2
    tol = k * 2.0 ** -24 * size                            # one FMA per expert
    tol = tol + eps * (want.abs() + tol) + torch.finfo(h).smallest_normal * torch.finfo(h).eps
    assert ((out[:, :O].cpu().double() - want).abs() <= tol).all()
    assert (out[:, O:] == 7).all()


@pytest.mark.parametrize("T", [3, 70])
def test_a_whole_layer_of_experts(T):
    """choice -> rows -> up projection with SiLU -> down projection -> weighted sum, on one stream without a synchronization, then
    captured and replayed on other inputs."""
    gen = _gen(21)
    E, k, D, F, g = 6, 2, 256, 384, 64
    h = torch.bfloat16
    up, down = (torch.randn((E, F, D), generator=gen) * 0.06).cuda(), (torch.randn((E, D, F), generator=gen) * 0.06).cuda()
    du, dd = B.make_group_desc(F, D, g, experts=E), B.make_group_desc(D, F, g, asymmetric=True, experts=E)
    cu, su, zu = B.alloc_group(du)
    cd, sd, zd = B.alloc_group(dd)
    vu, vd = torch.empty_like(up), torch.empty_like(down)
    x = torch.empty((T, D), dtype=h, device="cuda")
    choice, weights = torch.empty((T, k), dtype=torch.int32, device="cuda"), torch.empty((T, k), device="cuda")
    offsets = torch.empty(E + 1, dtype=torch.int32, device="cuda")
    rows, slots = torch.empty(T * k, dtype=torch.int32, device="cuda"), torch.empty((T, k), dtype=torch.int32, device="cuda")
    mid, y, out = (torch.empty(n, dtype=h, device="cuda") for n in ((T * k, F), (T * k, D), (T, D)))
    B.pipe_group_quantize(du, up, cu, su, zu, values=vu)
    B.pipe_group_quantize(dd, down, cd, sd, zd, values=vd)

    def layer():
        B.pipe_expert_rows(choice, E, offsets, rows, slots)
        B.pipe_expert_linear(du, cu, su, zu, x, offsets, mid, rows=rows, activation=B.ACT_SILU)
        B.pipe_expert_linear(dd, cd, sd, zd, mid, offsets, y)
        B.pipe_expert_combine(y, slots, weights, out)

    def inputs(seed):
        q = _gen(seed)
        x.copy_(torch.randn((T, D), generator=q).to(h))
        choice.copy_(torch.stack([torch.randperm(E, generator=q)[:k] for _ in range(T)]).to(torch.int32))
        weights.copy_(torch.softmax(torch.randn((T, k), generator=q), 1))

    def check():
        _ok()
        want = torch.zeros((T, D), dtype=torch.float64)
        for t in range(T):
            for j in range(k):
                e = int(choice[t, j])
                m = R.sigma(vu[e].cpu().double() @ x[t].cpu().double(), 2)
                want[t] += float(weights[t, j]) * (vd[e].cpu().double() @ m)
        # four roundings to bf16 on the way (weights, middle, weights, outputs), each half a step: relative 2^-8 of sums whose terms
        # add up like their squares
        off = (out.cpu().double() - want).norm() / want.norm()
        assert off < 4 * 2.0 ** -8, off

    inputs(1)
    layer()
    check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer()
    for seed in (2, 3):
        inputs(seed)
        graph.replay()
        check()
