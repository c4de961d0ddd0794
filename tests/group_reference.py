"""Plain 64-bit restatement of the 4-bit layers with group scales and of the products grouped by expert (include/pipe.h), and the
distance that a kernel may keep from it."""
import torch

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def few(rows):
    """Whether that many rows (per expert, rounded up) go to the kernel on exact operands."""
    return rows <= 16


def unpack(codes, I):
    """[E, I/32, O, 16] bytes -> int64 [E, O, I], nibble by nibble from the documented positions."""
    b = codes.cpu().to(torch.int64)
    E, nb, O, _ = b.shape
    out = torch.empty((E, O, nb, 32), dtype=torch.int64)
    for w in range(4):
        word = b[..., 4 * w] | (b[..., 4 * w + 1] << 8) | (b[..., 4 * w + 2] << 16) | (b[..., 4 * w + 3] << 24)
        for i in range(4):
            out[..., 8 * w + 2 * i] = ((word >> (4 * i)) & 15).transpose(1, 2)
            out[..., 8 * w + 2 * i + 1] = ((word >> (4 * (i + 4))) & 15).transpose(1, 2)
    return out.reshape(E, O, I)


def pack(u):
    """int [E, O, I] -> uint8 [E, I/32, O, 16]."""
    E, O, I = u.shape
    v = u.to(torch.int64).view(E, O, I // 32, 4, 8)
    word = torch.zeros(v.shape[:-1], dtype=torch.int64)
    for i in range(4):
        word |= (v[..., 2 * i] << (4 * i)) | (v[..., 2 * i + 1] << (4 * (i + 4)))
    b = torch.stack([(word >> (8 * j)) & 255 for j in range(4)], -1)      # [E, O, nb, 4, 4]
    return b.view(E, O, I // 32, 16).transpose(1, 2).contiguous().to(torch.uint8)


def dense(u, scales, zeros, g):
    """float64 [E, O, I] of codes [E, O, I], scales [E, I/g, O] and zeros of the same shape (or None)."""
    s = scales.cpu().double().transpose(1, 2).repeat_interleave(g, 2)
    z = 8.0 if zeros is None else zeros.cpu().double().transpose(1, 2).repeat_interleave(g, 2)
    return (u.double() - z) * s


def sigma(v, kind):
    if kind == 1:
        return v.clamp(min=0)
    if kind == 2:
        return v * torch.special.expit(v)
    if kind == 3:
        return v * torch.special.ndtr(v)
    return torch.special.expit(v) if kind == 4 else v


def random_layer(gen, E, O, I, g, dtype, asym):
    u = torch.randint(0, 16, (E, O, I), generator=gen)
    scales = (torch.rand((E, I // g, O), generator=gen) * 0.03 + 0.002).to(TYPES[dtype])
    zeros = torch.randint(0, 16, (E, I // g, O), generator=gen).to(torch.uint8) if asym else None
    return u, scales, zeros


def check_product(got, x, W, bias, kind, dtype, g, exact_operands, tag=""):
    """One expert's outputs [n, O] against sigma(x W^T + b) in 64 bits.

    exact_operands: codes as they are, a group's sum is at most 8 MMA steps of 16 products each, whose 17 addends are
    aligned and cut at 24 bits (2^-20 of the largest for a step, with room), then one binary32 FMA per group and one addition per
    warp and CTA (at most 64).  Otherwise the weights are rounded to the layer's type first (the reference rounds them too) and
    all I / 16 steps form one chain.  Then the activation (slope at most 1.13; 2^-21 of its value for the device's exp and erf)
    and half a step of the output's type."""
    h = TYPES[dtype]
    W = W if exact_operands else W.to(h).double()
    x = x.cpu().double()
    n, I = x.shape[0], W.shape[1]
    v, terms = x @ W.t(), x.abs() @ W.abs().t()
    if bias is not None:
        v = v + bias.cpu().double()
        terms = terms + bias.cpu().double().abs()
    steps = 8 * 2.0 ** -20 + (I // g + 64) * 2.0 ** -24 if exact_operands else (I / 16 + 8) * 2.0 ** -20
    want = sigma(v, kind)
    tol = 1.13 * steps * terms + 2.0 ** -21 * want.abs()
    tol = tol + torch.finfo(h).eps / 2 * (want.abs() + tol) + torch.finfo(h).smallest_normal * torch.finfo(h).eps
    off = (got.cpu().double() - want).abs()
    assert torch.isfinite(got.float()).all(), tag
    worst = float((off / tol).max()) if off.numel() else 0.0
    assert worst <= 1.0, f"{tag}: {worst:.3f} of the tolerance at {torch.unravel_index((off / tol).argmax(), off.shape)}"
