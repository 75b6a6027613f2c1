"""Rotary positions and per-head norms in 64 bits, from their definitions, for the tests."""
import math

import torch


def frequencies(rotary, axes, base=10000.0, scaling=0, factor=1.0, trained=0, fast=32.0, slow=1.0):
    """Radians per position of the pairs of one axis, and the factor of cosine and sine."""
    pairs = rotary // 2 // axes
    dim = 2 * pairs
    if scaling == 2:
        base = base * factor ** (dim / max(dim - 2, 1))
    f = [base ** (-2 * i / dim) for i in range(pairs)]
    if scaling == 1:
        f = [v / factor for v in f]
    gain = 1.0
    if scaling == 3:
        def pair_of(turns):
            return dim * math.log(trained / (turns * 2 * math.pi)) / (2 * math.log(base))
        low, high = max(math.floor(pair_of(fast)), 0), min(math.ceil(pair_of(slow)), dim - 1)
        ramp = [min(1.0, max(0.0, (i - low) / max(high - low, 0.001))) for i in range(pairs)]
        f = [v * (1 - r) + v / factor * r for v, r in zip(f, ramp)]
        gain = 1 + 0.1 * math.log(factor)
    return torch.tensor(f, dtype=torch.float64), gain


def rotate(x, positions, rotary, layout, axes, f, gain, transpose=False):
    """x [b, h, n, d]; positions [n(, axes)] or [b, n(, axes)].  Returns (result, size of what each element is formed from)."""
    x = x.double()
    p = positions.double().to(x.device)
    f = f.to(x.device)
    if axes == 2:
        a = torch.cat([p[..., :1] * f, p[..., 1:] * f], -1)
    else:
        a = p[..., None] * f
    a = a[:, None] if a.dim() == 3 else a[None, None]
    if transpose:
        a = -a
    half = rotary // 2
    i0 = torch.arange(half, device=x.device) if layout == 0 else 2 * torch.arange(half, device=x.device)
    i1 = i0 + half if layout == 0 else i0 + 1
    y, size = x.clone(), x.abs()
    x0, x1 = x[..., i0], x[..., i1]
    y[..., i0] = gain * (x0 * a.cos() - x1 * a.sin())
    y[..., i1] = gain * (x0 * a.sin() + x1 * a.cos())
    size[..., i0] = size[..., i1] = gain * (x0.abs() + x1.abs())
    return y, size


def normalise(x, norm, eps, weight=None, gain=None):
    x = x.double()
    if norm == 1:
        x = x / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    if norm == 2:
        x = x / x.square().sum(-1, keepdim=True).sqrt().clamp_min(eps)
    if weight is not None:
        x = x * weight.double()
    if gain is not None:
        x = x * gain.double()[:, None, None]
    return x


def bound(ref, size, dtype):
    """The rounding of the result, at most half a step, and some thirty fp32 roundings (each 2^-24 of what an element is
    formed from: products, the sum of squares, cosine and sine with their angle) on the way."""
    return torch.finfo(dtype).eps / 2 * ref.abs() + 32 * 2.0 ** -24 * size
