"""Inputs of which every piece of a long sequence counts, and what attention over them may be off by.

Few of the keys are planted: they are alike, q . k is 22 or more above what other keys reach, and together they have all of a row's weight but
some 1e-9.  A planted value is one channel, another one from key to key.  Channel c of out is then 4 n_c / n, n_c of n planted keys being its own,
all of one sign: a planted key that is lost, or one too many, is off by 1 / n_c of the channel, and n_c is 40 at most, whatever the
length.  (Random values over millions of keys average out to less than any bound that grows with the magnitudes.)
"""
import math

import torch

from tests.decoder_util import U, half_step

UNIT = 64


def planted_tokens(m, device):
    """A token of every unit of 64, or of every so many that there are 2500 at most, at changing places; the first and the last."""
    units = (m + UNIT - 1) // UNIT
    u = torch.arange(0, units, (units + 2499) // 2500, device=device)
    t = torch.minimum(u * UNIT + u * 37 % UNIT, torch.tensor(m - 1, device=device))
    return torch.unique(torch.cat((t, torch.tensor([0, m - 1], device=device))))


def plant(q, k, v, heads_of):
    """In place: q [n, heads, 64] all of one direction for a head of keys, k and v [m, kv_heads, 64] at the planted tokens.  All of it is held
    exactly by bf16 and by 4 bits.  heads_of: query heads that share a head of keys."""
    n, m = q.shape[0], k.shape[0]
    at = planted_tokens(m, q.device)
    i = torch.arange(64, device=q.device)
    for kv in range(k.shape[1]):
        sign = torch.where((i * (kv + 3) // 7) % 2 == 0, 1.0, -1.0)
        row = 1 + 0.25 * (torch.arange(n, device=q.device) % 3)
        q[:, kv * heads_of:(kv + 1) * heads_of] = (2 * row[:, None] * sign)[:, None].to(q.dtype)
        k[at, kv] = (2 * sign).to(k.dtype)
        x = torch.zeros((len(at), 64), device=q.device)
        x[torch.arange(len(at), device=q.device), (torch.arange(len(at), device=q.device) + 5 * kv) % 64] = 4.0
        v[at, kv] = x.to(v.dtype)
    return at


def planted_reference(q, k, v, scale, dtype, pieces, left_out=None, seen=None):
    """One head in 64 bits, and its bounds: the score's error d (64 products, for fp32 in parts 400 u of their magnitudes; the exponential's
    argument; twice, for the row's maximum and sum), h for a probability rounded to bf16, h |out| for the store.  Sums: a wave adds the
    keys of its piece one after the other, m / pieces of them, 16 waves are joined and 256 pieces: that many roundings, no more.
    left_out: tokens that a mistake leaves out; seen [n, m]: what each row sees, None: all."""
    q, k, v = q.double(), k.double(), v.double()
    m, f32 = k.shape[0], dtype == torch.float32
    h = half_step(dtype)
    s = (q @ k.t()) * scale
    if left_out is not None:
        s[:, left_out] = -math.inf
    if seen is not None:
        s = s.masked_fill(~seen, -math.inf)
    size = float(((q.abs() @ k.abs().t()) * scale).max())
    d = 2 * ((400 if f32 else 64) * U * size + (size + 4) * U)
    chain = (math.ceil(m / pieces / UNIT) * UNIT + 16 + 256) * U
    lse = torch.logsumexp(s, 1)
    p = torch.exp(s - lse[:, None])
    out, weighted = p @ v, p @ v.abs()
    return {"out": out, "out_tol": (d + (0 if f32 else h) + chain) * weighted + h * out.abs(),
            "lse": lse, "lse_tol": torch.full_like(lse, d + chain + 4 * U) + 4 * U * lse.abs()}
