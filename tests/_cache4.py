"""A cache in 4 bits from its definition: what is written of 16 elements, and what it stands for."""
import math

import torch

LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
E2M1 = [*LEVELS, *(-x for x in LEVELS)]
E4M3 = [math.nan if c & 127 == 127 else (-1.0 if c & 128 else 1.0)
        * math.ldexp(c & 7 if c & 120 == 0 else 8 + (c & 7), max(c >> 3 & 15, 1) - 10) for c in range(256)]


def nearest(values, x):
    """Index of the value (ascending; halfway: of even index) nearest to x >= 0, both in 64 bits."""
    v = torch.tensor(values, dtype=torch.float64)
    hi = torch.searchsorted(v, x.contiguous()).clamp(max=len(values) - 1)
    lo = (hi - 1).clamp(min=0)
    below, above = x - v[lo], v[hi] - x
    return torch.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)


def written(x, scale):
    """(codes [.., D / 2], scales [.., D / 16]) uint8 of x [.., D], on the CPU.  A product of two fp32
    numbers is exact in 64 bits; a reciprocal that is rounded twice is the one rounded once, as the
    step has 28 significant bits at most."""
    r32 = lambda t: t.float().double()  # noqa: E731
    scale = float(torch.tensor(scale, dtype=torch.float32))  # (the pool's number is fp32)
    y = x.double().cpu().unflatten(-1, (-1, 16))
    most = y.abs().amax(-1)
    units = float(torch.tensor(1.0 / (6.0 * scale), dtype=torch.float32))
    t = r32(most * units)
    s = nearest(E4M3[:127], t.nan_to_num(0.0, posinf=448.0).clamp(max=448.0))
    step = r32(torch.tensor(E4M3, dtype=torch.float64)[s] * scale)
    r = torch.where(step > 0, r32(1.0 / step), 0.0)
    z = r32(y * r[..., None]).nan_to_num(0.0, posinf=6.0, neginf=-6.0).clamp(-6.0, 6.0)
    c = (nearest(LEVELS, z.abs()) + 8 * torch.signbit(z)).flatten(-2)
    s = torch.where(most.isnan(), 127, s)
    return (c[..., ::2] | c[..., 1::2] << 4).to(torch.uint8), s.to(torch.uint8)


def values(codes, scales, scale):
    """What they stand for, in 64 bits, where they are."""
    e2m1, e4m3 = (torch.tensor(t, dtype=torch.float64, device=codes.device) for t in (E2M1, E4M3))
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    s = e4m3[scales.view(torch.uint8).long()].repeat_interleave(16, -1)
    return e2m1[c.long()] * s * float(torch.tensor(scale, dtype=torch.float32))
