"""Plain 64-bit restatement of the 8-bit integer layers and of the log probabilities of given tokens (include/pipe.h), and the distance
that a kernel may keep from it."""
import math

import torch

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def quantized(x):
    """scales float32 [.., rows] and codes int8 of finite rows.  The quotient of two binary32 numbers is at an odd multiple of one half or
    at least 2^-33 of itself away from it, so its rounding to binary64 settles the code."""
    x = x.cpu().double()
    s = (x.abs().amax(-1) / 127).float()
    d = torch.where(s == 0, 1.0, s.double())[..., None]
    q = torch.where(s[..., None] == 0, 0.0, torch.round(x / d).clamp(-127, 127))
    return s, q.to(torch.int8)


def sigma(v, kind):
    if kind == 1:
        return v.clamp(min=0)
    if kind == 2:
        return v * torch.special.expit(v)
    if kind == 3:
        return v * torch.special.ndtr(v)
    return torch.special.expit(v) if kind == 4 else v


def product(xq, sx, wq, sw, bias, kind, dtype):
    """Outputs [T, O] in 64 bits, and the distance that is allowed: the sum is exact, then four roundings of binary32 (the sum, two
    products, the addition of the bias), the activation (slope at most 1.13; 2^-21 of its value for its approximations), half a step of
    the output's type."""
    h = TYPES[dtype]
    v = (xq.cpu().double() @ wq.cpu().double().t()) * sw.cpu().double() * sx.cpu().double()[:, None]
    size = v.abs()
    if bias is not None:
        v, size = v + bias.cpu().double(), size + bias.cpu().double().abs()
    want = sigma(v, kind)
    tol = 1.13 * 4 * 2.0 ** -24 * size + (2.0 ** -21 * want.abs() if kind else 0)
    tol = tol + torch.finfo(h).eps / 2 * (want.abs() + tol) + torch.finfo(h).smallest_normal * torch.finfo(h).eps
    return want, tol


def check_product(got, xq, sx, wq, sw, bias, kind, dtype, tag=""):
    want, tol = product(xq, sx, wq, sw, bias, kind, dtype)
    assert got.dtype == TYPES[dtype]
    assert torch.isfinite(got.float()).all(), tag
    off = (got.cpu().double() - want).abs()
    worst = float((off / tol).max()) if off.numel() else 0.0
    assert worst <= 1.0, f"{tag}: {worst:.3f} of the tolerance at {torch.unravel_index((off / tol).argmax(), off.shape)}"


def logprobs(l, tokens, k, scale):
    """lp of tokens, entropy, top ids, top lp in 64 bits, of rows without NaN or +Inf; and the distance allowed for the two kinds of sums.

    A term exp(z), z = scale (l - m), is off by the roundings of l - m, of scale log2 e and of their product (3 * 2^-24 |z| of it)
    and by the exponential's 2^-22; rescaled at most once for every 32 terms of a thread, and once for each of at most 12 joins, by such a
    factor; a thread adds at most V / 256 + 1 terms in a chain (its products with l - m likewise).  A log probability is z - log(sum):
    those, the three roundings of z, the logarithm's 2^-22 and the last rounding."""
    z = l.cpu().double() * scale
    T, V = z.shape
    m = z.amax(1, keepdim=True)
    alive = torch.isfinite(m)
    d = torch.where(alive, z - m, 0.0)
    e = torch.where(torch.isinf(d), 0.0, torch.exp(d))
    S = e.sum(1, keepdim=True)
    norm = torch.log(S)
    lp_all = torch.where(alive, d - norm, -math.inf)
    p = torch.where(alive, e / S, 0.0)
    mean = (p * torch.where(torch.isinf(d), 0.0, d).abs()).sum(1, keepdim=True)
    steps = (V / 256 + 1 + 16) * 2.0 ** -24 + (V / 8192 + 12 + 1) * 2.0 ** -22
    rel = steps + 3 * 2.0 ** -24 * 2 * (mean + 1)        # (the terms' |z|, weighted by the terms; twice, for the rescalings' too)
    lp = torch.zeros(tokens.shape, dtype=torch.float64)
    inside = (tokens >= 0) & (tokens < V)
    got = lp_all.gather(1, tokens.clamp(0, V - 1).long())
    lp[inside] = got[inside]
    ent = torch.where(alive, norm + (p * torch.where(torch.isinf(d), 0.0, -d)).sum(1, keepdim=True), 0.0)[:, 0]
    ids = torch.full((T, k), -1, dtype=torch.int32)
    top = torch.full((T, k), -math.inf, dtype=torch.float64)
    order = torch.sort(l.cpu().double() + 0.0, dim=1, descending=True, stable=True).indices[:, :k]   # (+ 0: -0 and 0 are equal anyhow)
    v = lp_all.gather(1, order)
    listed = l.cpu().double().gather(1, order) > -math.inf
    ids[:, :order.shape[1]] = torch.where(listed, order, -1).int()
    top[:, :order.shape[1]] = torch.where(listed, v, -math.inf)
    second = ((p * torch.where(torch.isinf(d), 0.0, d) ** 2).sum(1, keepdim=True))
    ent_tol = rel * (1 + 2 * mean) + 6 * 2.0 ** -24 * second + 2.0 ** -21 * (norm.abs() + mean)
    return lp, ent, ids, top, rel + 2.0 ** -22 * norm.abs(), ent_tol[:, 0]


def close(got, want, tol, size, tag=""):
    """got against want: infinities alike, else within tol + 2^-22 of the size of what was subtracted."""
    got = got.cpu().double()
    want = torch.where(want < -torch.finfo(torch.float32).max, -math.inf, want)   # (twice the type's lowest number has no binary32 of its own)
    inf = torch.isinf(want)
    assert torch.equal(torch.isinf(got), inf) and torch.equal(got[inf], want[inf]), tag
    off = torch.where(inf, 0.0, (got - want).abs())
    room = (tol + 2.0 ** -22 * size).expand_as(off)
    room = torch.where(inf, 1.0, room)
    assert not torch.isnan(off).any(), tag
    worst = float((off / room).max()) if off.numel() else 0.0
    assert worst <= 1.0, f"{tag}: {worst:.3f} of the tolerance"
