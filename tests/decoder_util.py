"""Plain 64-bit forms of cross attention, its gradient and the 4-bit cache, and how far the kernels may be from them.

Bounds.  u = 2^-24 is half a step of fp32, h half a step of the tensors' type (bf16 2^-8, fp32 2^-24).
  scores   64 products are added in fp32 in some order: off by at most 64 u S, S_ij = scale sum_c |q_ic k_jc| (products of bf16
           are exact; of fp32 operands in three bf16 parts six of nine products are kept, the others are below 4 u each of
           the product's magnitude, and the six sums are of 6 * 64 terms: 400 u S covers both), the exponent's fma and the
           exponential another (|s| + 4) u.  In what follows d_ij is that error, times 2 for the row's maximum and sum.
  P        off by d P, and by h P where it enters a product in bf16 (fp32: parts hold it exactly).
  out      sum_j (d + h) P |v| from P, accumulation of n keys (n / 8 + 64) u sum_j P |v|, and h |out| for the store.
  dP       as the scores, with |d_out| |v|.   D: in fp32 sum_c |d_out| err(out) + 64 u sum |d_out out|; in bf16 the rounding of out
           is taken out again, by the sum of dS over the keys, and what is left is (d + n u) sum_j P |dP - D| + sum_j P err(dP) and
           h times the rounding itself, from P k in bf16.
           In bf16 dq is mended by the sum of the rounded dS: at most h sum_j |dS| more, through P |k|.
  dS       P ((d + h) |dP - D| + err(D) + err(dP)), which passes through |k| and |q|; dv: (d + h) P^T |d_out|.
"""
import math

import torch

U = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def attention(q, k, v, seen, scale, dtype, d_out=None):
    """One head of one sequence in 64 bits: q [n, 64], k, v [m, 64], seen [n or 1, m].  A dict of results and, under
    "<name>_tol", their bounds."""
    q, k, v = q.double(), k.double(), v.double()
    n, m = q.shape[0], k.shape[0]
    f32 = dtype == torch.float32
    h, hp = half_step(dtype), 0.0 if f32 else half_step(dtype)
    seen = seen.expand(n, m)
    used = seen.any(0)
    k, v = torch.where(used[:, None], k, 0.0), torch.where(used[:, None], v, 0.0)
    s = (q @ k.t()) * scale
    size = (q.abs() @ k.abs().t()) * scale
    s = s.masked_fill(~seen, -math.inf)
    if m == 0:
        out = torch.zeros_like(q)
        r = {"out": out, "out_tol": out, "lse": torch.full((n,), -math.inf, dtype=torch.float64, device=q.device),
             "lse_tol": torch.zeros(n, dtype=torch.float64, device=q.device)}
        if d_out is not None:
            for name, like in (("dq", q), ("dk", k), ("dv", v)):
                r[name] = r[name + "_tol"] = torch.zeros_like(like)
        return r
    lse = torch.logsumexp(s, 1)
    p = torch.where(seen, torch.exp(s - torch.where(lse == -math.inf, 0.0, lse)[:, None]), 0.0)
    terms = 400 if f32 else 64
    d = (terms * U * size + (torch.where(seen, s, 0.0).abs() + 4) * U).masked_fill(~seen, 0.0).amax(1, keepdim=True) * 2
    chain = (m / 8 + 64) * U
    out, weighted = p @ v, p @ v.abs()
    out_tol = (d + hp + chain) * weighted + h * out.abs()
    r = {"out": out, "out_tol": out_tol, "lse": lse, "lse_tol": d[:, 0] + chain + 4 * U * torch.where(lse == -math.inf, 0.0, lse).abs() + 4 * U}
    if d_out is None:
        return r
    g = d_out.double()
    dp, delta = g @ v.t(), (g * out).sum(1, keepdim=True)
    d_err = (g.abs() * out_tol).sum(1, keepdim=True) + 64 * U * (g * out).abs().sum(1, keepdim=True)
    dp_err = terms * U * (g.abs() @ v.abs().t())
    ds = p * (dp - delta)
    if not f32:
        d_err = hp * d_err + (d + chain + 4 * U) * ds.abs().sum(1, keepdim=True) + (p * dp_err).sum(1, keepdim=True)
        # the key gradient's D and the query gradient's dS, rounded with the D that lacks it
        d_err = d_err + hp * (g.abs() * out_tol).sum(1, keepdim=True)
    err = p * ((d + hp + 4 * U) * (dp - delta).abs() + d_err + dp_err) + hp * ds.abs() * 2 ** -7
    pairs = (max(n, m) / 8 + 64) * U
    for name, a, b, e in (("dq", ds, k, err), ("dk", ds.t(), q, err.t()), ("dv", p.t(), g, (p * (d + hp)).t())):
        f = 1.0 if name == "dv" else scale
        x = f * (a @ b)
        r[name] = x
        if name == "dq" and not f32:       # what is taken out for the rounding of dS, at most the sum of its roundings
            e = e + p * (hp * ds.abs().sum(1, keepdim=True) + hp * d_err)
        r[name + "_tol"] = f * (e @ b.abs() + (pairs + (400 if f32 else 0) * U) * (a.abs() @ b.abs())) + h * x.abs()
    return r


def check(name, got, want, tol, floor=1e-30):
    """Every element within its bound; equal infinities and NaNs in the same places."""
    got, want = got.double(), want.to(got.device)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{name}: NaN in other places"
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), f"{name}: infinities differ"
    off = ((got - want).abs() / (tol.to(got.device) + floor))[fine]
    worst = float(off.max()) if off.numel() else 0.0
    print(f"{name}: {worst:.3f} of its bound", flush=True)
    assert worst <= 1.0, f"{name}: off by {worst} times its bound"


def cross_reference(q, k, v, spans, mask, scale, d_out=None):
    """The whole batch; spans: (first, rows, first key, keys) of each sequence.  Rows outside stay NaN."""
    H, KH = q.shape[1], k.shape[1]
    like = {"out": q, "lse": q[:, :, 0].t()}
    if d_out is not None:
        like.update(dq=q, dk=k, dv=v)
    r = {}
    for name, t in like.items():
        r[name] = torch.full(t.shape, math.nan, dtype=torch.float64, device=q.device)
        r[name + "_tol"] = torch.zeros(t.shape, dtype=torch.float64, device=q.device)
    for q0, n, k0, m in spans:
        seen = torch.ones((1, m), dtype=torch.bool, device=q.device) if mask is None else (mask[k0:k0 + m] != 0)[None]
        for name in ("dk", "dv") if d_out is not None else ():
            r[name][k0:k0 + m] = 0.0
        for h in range(H):
            kh = h // (H // KH)
            x = attention(q[q0:q0 + n, h], k[k0:k0 + m, kh], v[k0:k0 + m, kh], seen, scale, q.dtype,
                          None if d_out is None else d_out[q0:q0 + n, h])
            r["out"][q0:q0 + n, h], r["lse"][h, q0:q0 + n] = x["out"], x["lse"]
            r["out_tol"][q0:q0 + n, h], r["lse_tol"][h, q0:q0 + n] = x["out_tol"], x["lse_tol"]
            if d_out is not None:
                r["dq"][q0:q0 + n, h], r["dq_tol"][q0:q0 + n, h] = x["dq"], x["dq_tol"]
                for name in ("dk", "dv"):
                    r[name][k0:k0 + m, kh] += x[name]
                    r[name + "_tol"][k0:k0 + m, kh] += x[name + "_tol"]
    return r


# ---- the 4-bit form, by tables ------------------------------------------------------------------------

STEPS = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)
TIES = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], dtype=torch.float64)  # between code i and i + 1


POWERS = torch.tensor([2.0 ** (i - 127) for i in range(256)], dtype=torch.float64)   # (torch.pow is a rounding off on the GPU)


def four_bits(x):
    """x [..., 64] (64 bits) -> codes uint8 [..., 64] (sign in bit 3) and exponent bytes uint8 [..., 2]."""
    blocks = x.reshape(*x.shape[:-1], 2, 32)
    bad = ~torch.isfinite(blocks).all(-1)
    top = torch.where(torch.isfinite(blocks), blocks, 0.0).abs().amax(-1)
    e = torch.full(top.shape, -100, dtype=torch.int64, device=x.device)
    for p in range(-99, 126):
        e = torch.where(top >= 7 * 2.0 ** (p - 1), p, e)
    a = (torch.where(torch.isfinite(blocks), blocks, 0.0).abs() / POWERS.to(x.device)[e + 127][..., None])
    code = torch.zeros(a.shape, dtype=torch.int64, device=x.device)
    for i, t in enumerate(TIES.tolist()):
        code += (a > t) | ((a == t) & (i % 2 == 1))      # a tie goes to the even code: i + 1 where i is odd
    code = code + 8 * torch.signbit(blocks).long()
    code = torch.where(bad[..., None], 0, code)
    return code.reshape(x.shape).to(torch.uint8), torch.where(bad, 255, e + 127).to(torch.uint8)


def packed(code):
    return code[..., 0::2] | (code[..., 1::2] << 4)


def values(codes, scales):
    """Packed codes [..., 32] and exponent bytes [..., 2] -> values in 64 bits."""
    code = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    x = STEPS.to(codes.device)[(code & 7).long()] * torch.where(code > 7, -1.0, 1.0).double()
    unit = torch.where(scales == 255, math.nan, POWERS.to(codes.device)[scales.long()])
    return x * unit.repeat_interleave(32, -1)


def rotated(x, at, cos, sin, neighbours):
    """x [n, heads, 64] in 64 bits; at [n, axes] rows of the tables.  Products of 24-bit numbers are exact in 64 bits."""
    axes, y = at.shape[1], x.clone()
    width = 64 // axes
    for axis in range(axes):
        c, s = cos.double()[at[:, axis]][:, None], sin.double()[at[:, axis]][:, None]
        i = torch.arange(width // 2, device=x.device)
        a, b = (2 * i, 2 * i + 1) if neighbours else (i, i + width // 2)
        a, b = a + axis * width, b + axis * width
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    return y
