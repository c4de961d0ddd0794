"""Log probabilities of given tokens, entropy and top alternatives on the GPU."""
import math

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


def _call(l, tokens, k, scale=1.0, entropy=True):
    """Runs l (on the GPU already) and returns outputs with guards behind them looked at."""
    T, n = tokens.shape
    f32 = dict(dtype=torch.float32, device="cuda")
    raw = [torch.full((T * n + 8,), -7.0, **f32), torch.full((T + 8,), -7.0, **f32), torch.full((T * k + 8,), -7, dtype=torch.int32, device="cuda"), torch.full((T * k + 8,), -7.0, **f32)]
    lp, ent, top, tlp = raw[0][:T * n].view(T, n), raw[1][:T], raw[2][:T * k].view(T, k), raw[3][:T * k].view(T, k)
    B.pipe_token_logprobs(l, tokens.cuda() if n else None, lp if n else None, entropy=ent if entropy else None, top=top if k else None,
                          top_logprobs=tlp if k else None, scale=scale)
    torch.cuda.synchronize()
    for r in raw:
        assert (r[-8:] == -7).all()
    assert entropy or (ent == -7).all()
    return lp, ent, top, tlp


def _check(l, tokens, k, scale=1.0, on=None, tag=""):
    lp, ent, top, tlp = _call(l.cuda() if on is None else on, tokens, k, scale)
    assert B.pipe_poll_status() == B.PIPE_OK
    w_lp, w_ent, w_ids, w_top, tol, ent_tol = R.logprobs(l, tokens, k, scale)
    size = lambda w: torch.where(torch.isinf(w), 0.0, w.abs()) + 1  # noqa: E731
    R.close(lp, w_lp, tol, size(w_lp), tag + " lp")
    R.close(ent, w_ent, ent_tol, 1 + w_ent.abs(), tag + " entropy")
    assert torch.equal(top.cpu(), w_ids), tag
    R.close(tlp, w_top, tol, size(w_top), tag + " top")


def _logits(gen, T, V, dtype, spread=3.0):
    l = torch.randn((T, V), generator=gen) * spread
    l[torch.arange(T), torch.randint(0, V, (T,), generator=gen)] += torch.rand((T,), generator=gen) * 15
    return l.to(R.TYPES[dtype])


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("T,V,n,k", [(1, 1, 1, 1), (1, 2, 3, 5), (3, 7, 1, 7), (2, 31, 2, 1), (5, 255, 1, 20), (4, 1000, 4, 64), (2, 4097, 1, 10), (1, 32000, 1, 5), (7, 50001, 3, 20),
                                     (300, 515, 1, 3), (2, 128000, 1, 64), (700, 2048, 1, 0), (150, 9001, 2, 8), (33, 32000, 1, 10)])
def test_sizes(dtype, T, V, n, k):
    gen = _gen(T + V)
    l = _logits(gen, T, V, dtype)
    tokens = torch.randint(-2, V + 2, (T, n), generator=gen, dtype=torch.int32)
    tokens[0, 0] = int(l[0].float().argmax())
    _check(l, tokens, k, tag=f"{T} {V}")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("scale", [1e-6, 0.1, 1.25, 40.0])
def test_scales(dtype, scale):
    gen = _gen(2)
    _check(_logits(gen, 6, 3001, dtype), torch.randint(0, 3001, (6, 2), generator=gen, dtype=torch.int32), 9, scale)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_masks(dtype):
    """Masked tokens, rows with one token left, none at all, the type's lowest and highest numbers."""
    gen = _gen(3)
    T, V, k = 12, 5003, 12
    l = _logits(gen, T, V, "fp32")
    h, f = R.TYPES[dtype], torch.finfo(R.TYPES[dtype])
    l[1, torch.rand((V,), generator=gen) < 0.5] = -math.inf
    l[2] = -math.inf
    l[3] = -math.inf
    l[3, 4000] = 2.0
    l[4, 100:] = f.min                                  # masked by the lowest number: all but the first hundred have probability 0
    l[5] = f.min                                        # every token so: all alike
    l[6] = -math.inf
    l[6, [7, 5002, 0]] = torch.tensor([f.min, f.max, 0.0])
    l[7] = -math.inf
    l[7, :5] = torch.tensor([1.0, 3.0, 3.0, -2.0, 3.0])
    l[8] = 0.0                                          # all alike
    l[9] = torch.where(torch.arange(V) % 2 == 0, 0.0, -0.0)
    l[10] = f.max
    l[11, ::2] = 7.0                                    # many equal ones at the top
    l = l.clamp(f.min, f.max) if dtype == "fp16" else l
    l = torch.where(torch.isneginf(l), -math.inf, l).to(h)
    if dtype == "fp16":
        l[2] = -math.inf
        l[3] = -math.inf
        l[3, 4000] = 2.0
        l[7, 5:] = -math.inf
    tokens = torch.randint(0, V, (T, 3), generator=gen, dtype=torch.int32)
    tokens[3, 0], tokens[7, 0], tokens[6, 1] = 4000, 1, 5002
    _check(l, tokens, k)
    _check(l, tokens, 64, 0.5)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V", [3000, 40000])
def test_equal_logits_are_listed_in_order(dtype, V):
    """Logits of few values: whole stretches of equal ones, of which the first are listed."""
    gen = _gen(4)
    l = torch.randint(0, 4, (40, V), generator=gen).to(R.TYPES[dtype])
    l[1] = 5
    l[2, :-3] = 1
    l[2, -3:] = 2
    l[3, V // 2:] = 9
    l[4] = torch.arange(V) // 50.0                     # ascending
    l[5] = -(torch.arange(V) // 50.0)
    _check(l, torch.zeros((40, 1), dtype=torch.int32), 20)
    _check(l, torch.zeros((40, 1), dtype=torch.int32), 64)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_rows_that_start_anywhere(dtype):
    gen = _gen(5)
    T, V, ldl = 5, 777, 781
    l = _logits(gen, T, V, dtype)
    for shift in range(8):
        flat = torch.full((T * ldl + 16,), math.nan, dtype=R.TYPES[dtype], device="cuda")   # what lies between the rows is not read
        at = flat[shift:shift + T * ldl].view(T, ldl)[:, :V]
        at.copy_(l)
        _check(l, torch.randint(0, V, (T, 1), generator=gen, dtype=torch.int32), 6, on=at)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("V", [50, 20000])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_rows_that_are_no_distribution(bad, V, dtype):
    gen = _gen(6)
    l = _logits(gen, 4, V, dtype)
    tokens = torch.randint(0, V, (4, 2), generator=gen, dtype=torch.int32)
    tokens[2, 1] = -1
    clean = _call(l.cuda(), tokens, 5)
    assert B.pipe_poll_status() == B.PIPE_OK
    for at in (0, V // 2, V - 1):
        one = l.clone()
        one[2, at] = bad
        lp, ent, top, tlp = _call(one.cuda(), tokens, 5)
        assert B.pipe_poll_status() == B.PIPE_ERR_NONFINITE
        assert math.isnan(lp[2, 0]) and lp[2, 1] == 0 and math.isnan(ent[2]) and (top[2] == -1).all() and torch.isnan(tlp[2]).all()
        for got, want in zip((lp, ent, top, tlp), clean):
            assert torch.equal(got[[0, 1, 3]], want[[0, 1, 3]])
    one = l.clone()
    one[2] = -math.inf                                   # nothing left but a NaN
    one[2, 3] = math.nan
    lp, ent, top, tlp = _call(one.cuda(), tokens, 5)
    assert B.pipe_poll_status() == B.PIPE_ERR_NONFINITE and math.isnan(lp[2, 0]) and math.isnan(ent[2]) and (top[2] == -1).all()


def test_outputs_asked_for_one_by_one():
    gen = _gen(7)
    l = _logits(gen, 9, 6000, "bf16").cuda()
    tokens = torch.randint(0, 6000, (9, 1), generator=gen, dtype=torch.int32)
    lp, ent, top, tlp = _call(l, tokens, 4)
    none = torch.zeros((9, 0), dtype=torch.int32)
    assert torch.equal(_call(l, none, 4)[2], top) and torch.equal(_call(l, none, 4, entropy=False)[3], tlp)
    assert torch.equal(_call(l, none, 0)[1], ent) and torch.equal(_call(l, tokens, 0, entropy=False)[0], lp)
    flat = torch.empty(9, device="cuda")                 # tokens [T]
    B.pipe_token_logprobs(l, tokens[:, 0].contiguous().cuda(), flat)
    only = torch.empty((9, 4), dtype=torch.int32, device="cuda")
    B.pipe_token_logprobs(l, top=only)
    rest = torch.empty((9, 4), device="cuda")
    B.pipe_token_logprobs(l, top_logprobs=rest)
    _ok()
    assert torch.equal(flat, lp[:, 0]) and torch.equal(only, top) and torch.equal(rest, tlp)
    B.pipe_token_logprobs(l)                             # nothing asked for
    B.pipe_token_logprobs(l[:0], entropy=ent[:0])
    _ok()


def test_rows_far_apart():
    """Rows more than 2^31 values apart."""
    gen = _gen(8)
    V, pitch = 1003, (1 << 31) + 40
    flat = torch.empty(pitch + V, dtype=torch.bfloat16, device="cuda")
    at = flat.as_strided((2, V), (pitch, 1))
    l = _logits(gen, 2, V, "bf16")
    at.copy_(l)
    _check(l, torch.randint(0, V, (2, 2), generator=gen, dtype=torch.int32), 5, on=at)


def test_the_head_of_a_model_and_what_it_says():
    """Hidden states to int8, the head's product in 32 bits, log probabilities: against 64 bits from the codes on."""
    gen = _gen(9)
    T, I, V = 21, 520, 6007
    x = torch.randn((T, I), generator=gen).to(torch.bfloat16).cuda()
    W = (torch.randn((V, I), generator=gen) * 0.1).to(torch.bfloat16).cuda()
    codes, scales = B.alloc_int8(V, I)
    xq, sx = B.alloc_int8(T, I)
    logits = torch.empty((T, V), device="cuda")
    tokens = torch.randint(0, V, (T, 2), generator=gen, dtype=torch.int32)
    lp, ent = torch.empty((T, 2), device="cuda"), torch.empty(T, device="cuda")
    top, tlp = torch.empty((T, 8), dtype=torch.int32, device="cuda"), torch.empty((T, 8), device="cuda")

    def forward():
        B.pipe_int8_quantize(x, xq, sx)
        B.pipe_int8_linear(B.make_int8_desc(V, I, dtype=torch.float32), codes, scales, xq, sx, logits)
        B.pipe_token_logprobs(logits, tokens_gpu, lp, entropy=ent, top=top, top_logprobs=tlp)

    tokens_gpu = tokens.cuda()
    B.pipe_int8_quantize(W, codes, scales)
    forward()
    _ok()
    st, xt = R.quantized(x)
    sw, wq = R.quantized(W)
    R.check_product(logits, xt, st, wq, sw, None, 0, "fp32")
    w_lp, w_ent, w_ids, w_top, tol, ent_tol = R.logprobs(logits, tokens, 8, 1.0)
    R.close(lp, w_lp, tol, 1 + w_lp.abs())
    R.close(ent, w_ent, ent_tol, 1 + w_ent.abs())
    assert torch.equal(top.cpu(), w_ids)
    R.close(tlp, w_top, tol, 1 + w_top.abs())
    # captured once, replayed on other inputs: the same bits as calls one by one
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        forward()
    x.copy_(torch.randn((T, I), generator=gen).to(torch.bfloat16))
    graph.replay()
    _ok()
    replayed = [t.clone() for t in (logits, lp, ent, top, tlp)]
    forward()
    _ok()
    for a, b in zip(replayed, (logits, lp, ent, top, tlp)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("low", [-1e4, -1e7, -1e9, -1e20, -1e29, -1e30, -3e38])
@pytest.mark.parametrize("scale", [1.0, 2.0 ** -20, 2.0 ** 20])
def test_masks_of_any_large_number(dtype, low, scale):
    """Tokens masked by adding or writing a large negative number, before others and behind, in parts of a row and in all of it."""
    gen = _gen(11)
    T, V = 8, 40009
    l = torch.randn((T, V), generator=gen) * 3
    l[0, :V - 50] = low
    l[1, 50:] = low
    l[2, torch.rand((V,), generator=gen) < 0.999] = low
    l[3] = low
    l[4] = low
    l[4, 20000] = low * 0.5
    l[5, ::2] = -math.inf
    l[5, 1::4] = low
    l[6, 8192:8192 * 4] = low
    l[7] += -low * 2.0 ** -6                              # large positive ones
    l = l.to(R.TYPES[dtype])
    _check(l, torch.randint(0, V, (T, 2), generator=gen, dtype=torch.int32), 4, scale, tag=f"{low}")
    _check(l[:, :3001].contiguous(), torch.randint(0, 3001, (T, 2), generator=gen, dtype=torch.int32), 4, scale, tag=f"{low} short")


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("k", [0, 10, 64])
@pytest.mark.parametrize("T,V", [(460, 3001), (460, 12007), (460, 40009), (170, 90001), (46, 40009), (20, 12007)])
def test_rows_for_every_number_of_threads(dtype, k, T, V):
    """Few and many rows, short and long ones: CTAs of 128, 256 and 512 threads, one or more to a row.  Every row is one of ten kinds."""
    gen = _gen(12)
    kinds = 10
    l = torch.randn((kinds, V), generator=gen) * 3
    l[1, torch.rand((V,), generator=gen) < 0.99] = -math.inf
    l[2] = -math.inf
    l[3] = 1.5
    l[4] = torch.randint(0, 4, (V,), generator=gen).float()
    l[5] = torch.arange(V) / 64.0
    l[6] = -torch.arange(V) / 64.0
    l[7, :V - 3] = -math.inf
    l[8, V // 2:V // 2 + 200] = 60.0
    l[9, 5:] = -60000.0
    l = l.to(R.TYPES[dtype])
    tokens = torch.randint(-1, V + 1, (kinds, 3), generator=gen, dtype=torch.int32)
    tokens[7, 0] = V - 1
    on = torch.full((T, V + 5), math.nan, dtype=R.TYPES[dtype], device="cuda")[:, :V]
    row = torch.arange(T) % kinds
    on.copy_(l.cuda()[row.cuda()])
    lp, ent, top, tlp = _call(on, tokens[row].contiguous(), k)
    _ok()
    w_lp, w_ent, w_ids, w_top, tol, ent_tol = (w[row] for w in R.logprobs(l, tokens, max(k, 1), 1.0))
    size = lambda w: torch.where(torch.isinf(w), 0.0, w.abs()) + 1  # noqa: E731
    R.close(lp, w_lp, tol, size(w_lp), f"{T} {V} lp")
    R.close(ent, w_ent, ent_tol, 1 + w_ent.abs(), f"{T} {V} entropy")
    if k:
        assert torch.equal(top.cpu(), w_ids)
        R.close(tlp, w_top, tol, size(w_top), f"{T} {V} top")
