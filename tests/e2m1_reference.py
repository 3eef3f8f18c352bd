"""A 4-bit cache in 64 bits for the tests: what its codes and scales stand for, and what has to be written into it."""
import numpy as np
import torch

F8, BF16 = torch.float8_e4m3fn, torch.bfloat16
STEPS = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
VALUES = torch.cat((STEPS, -STEPS))


def codes_of(packed):
    """Codes 0..15 [..., D] of packed bytes [..., D/2]."""
    b = packed.cpu().long()
    return torch.stack((b % 16, b // 16), -1).flatten(-2)


def scales_of(scales):
    return scales.cpu().view(torch.uint8).view(F8).double()


def widen(packed, scales):
    """code * scale, float64."""
    return VALUES[codes_of(packed)] * scales_of(scales).repeat_interleave(16, -1)


def pack(codes):
    c = codes.to(torch.uint8)
    return c[..., 0::2] | (c[..., 1::2] << 4)


def nearest(y):
    """Code of each float64 value of y: the nearest of E2M1's magnitudes, ties to the even code, saturating at 6."""
    m = y.abs()
    mid = (STEPS[1:] + STEPS[:-1]) / 2
    code = (m[..., None] > mid).sum(-1)
    tie = (m[..., None] == mid).any(-1)
    code = code + (tie & (code % 2 == 1)).long()
    return code + 8 * (torch.signbit(y)).long()


def quantise(x, unit):
    """(codes, scales) of x [..., 16 n] float64, as include/qknorm_attn.h says, in exact arithmetic but for the roundings it names
    (and an fp32 reciprocal of `unit`, which is exact for the powers of two that the tests use)."""
    b = (x / unit).unflatten(-1, (-1, 16))
    f = (b.abs().amax(-1) / 6.0).clamp(max=448.0).to(F8)
    w = f.double()[..., None]
    return nearest(torch.where(w > 0, b / w.clamp(min=1e-30), b * 0.0)).flatten(-2), f


def check_written(x, packed, scales, unit, off):
    """What the kernel has written for x (float64, known to `off` relative to the block's largest): every scale is
    amax/6 rounded to E4M3, allowing for `off`, and every code the nearest to x / (unit * that scale), allowing for it."""
    b = (x / unit).unflatten(-1, (-1, 16))
    amax = b.abs().amax(-1)
    f = scales_of(scales)
    low, high = (amax / 6 * (1 - off)).clamp(max=448).to(F8).double(), (amax / 6 * (1 + off)).clamp(max=448).to(F8).double()
    assert ((f >= low) & (f <= high)).all(), "a block's scale is not amax/6 rounded"
    y = torch.where(f[..., None] > 0, b / f[..., None].clamp(min=1e-30), b * 0.0)
    got = VALUES[codes_of(packed)].unflatten(-1, (-1, 16))
    slack = 2 * off * y.abs().amax(-1, keepdim=True) + 1e-12
    gap = (y.clamp(-6, 6)[..., None] - VALUES).abs().amin(-1)
    assert ((got - y.clamp(-6, 6)).abs() <= gap + 2 * slack).all(), "a code is not the nearest"


def random_pool(g, shape, sigma=1.0, unit=1.0):
    """(packed, scales) of normal values [..., D]."""
    x = torch.randn(shape, generator=g, dtype=torch.float64) * sigma
    c, f = quantise(x, unit)
    return pack(c), f
