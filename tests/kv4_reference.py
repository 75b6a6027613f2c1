"""The 4-bit cache and its attention in 64 bits, from the definitions, for the tests."""
import math

import torch

SCALES = torch.tensor([(8 + b % 8) / 8 * 2.0 ** (b // 8 - 20) for b in range(256)], dtype=torch.float64)


def quantise(x):
    """Rows [..., dim] -> codes c [..., dim] (int64), scale bytes [..., dim / 16], values (64 bits)."""
    table = SCALES.to(x.device)
    blocks = torch.nan_to_num(x.double(), nan=0.0, posinf=math.inf, neginf=-math.inf).unflatten(-1, (-1, 16))
    top = blocks.abs().amax(-1, keepdim=True)
    byte = (7 * table < top).sum(-1).clamp_max(255)          # how many scales are too small
    s = table[byte][..., None]
    c = (blocks / s).round().clamp(-7, 7)
    return c.long().flatten(-2), byte, (c * s).flatten(-2)


def pack(c):
    u = (c + 8).to(torch.uint8).unflatten(-1, (-1, 2))
    return u[..., 0] | (u[..., 1] << 4)


def values(codes, scales):
    """Planes' rows -> values in 64 bits."""
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).double() - 8
    return (c.unflatten(-1, (-1, 16)) * SCALES.to(codes.device)[scales.long()][..., None]).flatten(-2)


def attend(q, k, v, length, nq, scale, causal=False, window=0, n_sink=0):
    """One stored head: q [group, n, d] (the first nq tokens count), k, v [rows, d] in 64 bits.  Returns (out, spread, size, logit):
    sum p v, sum p |v - out|, sum p |v|, and the largest sum |q k| scale over the rows a query sees."""
    q, k, v = q[:, :nq].double(), k[:length], v[:length]
    j = torch.arange(length, device=q.device)[None]
    at = (length - nq + torch.arange(nq, device=q.device))[:, None]
    see = torch.ones(nq, length, dtype=torch.bool, device=q.device)
    if causal:
        see &= j <= at
    if window:
        see &= (j < n_sink) | (j > at - window)
    z = (q @ k.T * scale).masked_fill(~see, -math.inf)
    some = see.any(-1)
    p = torch.where(some[:, None], torch.softmax(z, -1), torch.zeros((), dtype=torch.float64, device=q.device))
    out = p @ v
    spread = (p[..., None] * (v - out[..., None, :]).abs()).sum(-2)
    logit = (q.abs() @ k.abs().T * scale).masked_fill(~see, 0).amax(-1, keepdim=True) if length else torch.zeros(q.shape[:2] + (1,), device=q.device)
    return out, spread, p @ v.abs(), logit


def bound(out, spread, size, logit, dtype, dim, length):
    """How far the kernel's result may be.  The result is rounded to its type once (half a step of |out|).  bf16: a probability is
    rounded for the product with the values (half a step, 2^-8 of it), and so is the sum it is divided by, which
    leaves 2^-8 sum p |v - out|.  fp32 arithmetic: a logit is a sum of dim products (every addition 2^-23 of the partial sum:
    matrix instructions may truncate), the exponential and its argument a few more, and an output a chain of one addition for every
    16 rows; an error e of a logit changes every term by e of itself, in the numerator and in the denominator."""
    u = 2.0 ** -23
    half = torch.finfo(dtype).eps / 2
    e = u * ((dim + 8) * logit + 16 + length / 16)
    return half * out.abs() + (1.02 * half * spread if dtype == torch.bfloat16 else 0) + 2 * e * (size + out.abs()) + 1e-30
