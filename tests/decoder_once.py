"""Rounding of 64-bit values to bf16, once, and inputs of the rotation whose exact results lie next to a border of it."""
import torch


def to_bf16_once(x):
    """x in 64 bits (finite, and in bf16's range of normal numbers) -> the nearest bf16, of two as near the one with an even last bit: by comparing
    distances, which are exact in 64 bits for neighbours this close."""
    near = x.float().bfloat16()
    bits = near.view(torch.int16)
    best, off = near, (x - near.double()).abs()
    for step in (-1, 1):
        other = (bits + step).view(torch.bfloat16)
        d = (x - other.double()).abs()
        even = (bits + step) & 1 == 0
        take = torch.isfinite(other) & ((d < off) | ((d == off) & even & (best.view(torch.int16) & 1 == 1)))
        best, off = torch.where(take, other, best), torch.where(take, d, off)
    return torch.where(x == 0, torch.zeros_like(best), best)


def next_to_ties(rows, heads, axes, generator, device):
    """q [rows, heads, 64] in bf16, cos and sin [rows, 32 / axes] in fp32: powers of two turned by a cosine of 1 + 2^-8 or 1 + 3 * 2^-8, the middle
    between two neighbours of bf16 (the even one below, or above), and sines of 0 or +-2^-30 to 2^-45: the exact result lies off the middle by less than
    fp32 can tell, or on it."""
    pairs = 32 // axes

    def pick(values, *shape):
        return torch.tensor(values, device=device)[torch.randint(0, len(values), shape, generator=generator, device=device)]
    q = pick([1.0, -1.0, 2.0, -2.0, 0.5, -4.0], rows, heads, 64).bfloat16()
    cos = pick([1 + 2.0 ** -8, 1 + 3 * 2.0 ** -8], rows, pairs).float()
    sin = pick([0.0] + [s * 2.0 ** -e for e in (30, 32, 37, 45) for s in (1, -1)], rows, pairs).float()
    return q, cos, sin
