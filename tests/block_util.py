"""Plain 64-bit forms of rotary positions with head norms and of the residual stream with its norms, with their gradients, and how far
the kernels may be from them.

Bounds.  u = 2^-24 is half a step of fp32, h half a step of the tensor that is stored (bf16 2^-8, fp32 2^-24).  `depth` is the number of
additions that a term of a sum over channels can pass through (8 or 16 in a lane, six steps over lanes, up to 16 waves: 40).
  norm     The mean is taken twice: what is left of its error is that of the sum of the centred values, depth u mean|d|, and of the subtraction,
           u |d|, u more for the second.  The sum of squares is off by (depth + 2) u of itself, its inverse root by half of that and 3 u.  With
           mean|d| <= sigma:  err(n) = u ((depth / 2 + 8) |n| + depth + 3).  An error e of z itself adds (e + mean e + |n| mean(|n| e)) / sigma.
  turn     x c + p, in fp32 with the rounding of p = o s made up for: 3 u |y|, in bf16 u |o s| more, and the operands' errors times |c| and |s|.
  back     g = dn, err(g) given:  mean g is off by mean err(g) + depth u mean|g|, mean(g n) by mean(|g| err(n) + |n| err(g)) + (depth + 1) u mean|g n|;
           dz = (g - mean g - n mean(g n)) / sigma  by the sum of these, 3 u of each term, and (depth / 2 + 4) u of itself.
  scale    and gate: dr' (n w + b) is summed as w (sum dr' n) + b (sum dr'), r is x + (s w) n + s b: the parts |n w| and |b| count each, with
           up to three roundings more.
  sums     over rows: the terms' errors, and `chain` u times the sum of their magnitudes: rows of a wave one after the other (at most a
           512th of all, those of 16 heads), rows side by side (16), workgroups (128 in a row) and eight groups of them.
"""
import math

import torch

U = 2.0 ** -24
DEPTH = 40


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


class Value:
    """A tensor in 64 bits and how far the kernel's may be from it."""
    def __init__(self, x, err=None):
        self.x = x.double()
        self.err = torch.zeros_like(self.x) if err is None else err

    def __mul__(self, o):
        x = self.x * o.x
        return Value(x, self.err * o.x.abs() + self.x.abs() * o.err + U * x.abs())

    def __add__(self, o):
        x = self.x + o.x
        return Value(x, self.err + o.err + U * x.abs())

    def stored(self, dtype):
        return self.x, self.err + half_step(dtype) * self.x.abs()


def given(t):
    return None if t is None else Value(t)


def norm(z, kind, eps):
    """-> n and 1 / sigma."""
    d = z.x - z.x.mean(-1, keepdim=True) if kind == "layer" else z.x
    inv = 1 / torch.sqrt((d * d).mean(-1, keepdim=True) + eps)
    n = d * inv
    err = U * ((DEPTH / 2 + 8) * n.abs() + DEPTH + 3) + inv * (z.err + z.err.mean(-1, keepdim=True)) + n.abs() * (n.abs() * inv * z.err).mean(-1, keepdim=True)
    return Value(n, err), inv


def norm_back(g, n, inv, kind):
    m1 = g.x.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(inv)
    m2 = (g.x * n.x).mean(-1, keepdim=True)
    e1 = g.err.mean(-1, keepdim=True) + DEPTH * U * g.x.abs().mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(inv)
    e2 = (g.x.abs() * n.err + n.x.abs() * g.err).mean(-1, keepdim=True) + (DEPTH + 1) * U * (g.x * n.x).abs().mean(-1, keepdim=True)
    x = inv * (g.x - m1 - n.x * m2)
    err = inv * (g.err + e1 + n.x.abs() * e2 + n.err * m2.abs() + 3 * U * (g.x.abs() + m1.abs() + (n.x * m2).abs())) + (DEPTH / 2 + 4) * U * x.abs()
    return Value(x, err)


def affine(n, weight, bias):
    n = n if weight is None else n * given(weight)
    return n if bias is None else n + given(bias)


def sum_rows(v, rows, size=None):
    """Over all axes but the last; rows: how many rows (of 16 heads and less) there are; size: the terms' magnitudes, where they are made
    of parts that are summed apart."""
    flat, err = v.x.reshape(-1, v.x.shape[-1]), v.err.reshape(-1, v.x.shape[-1])
    size = flat.abs() if size is None else size.reshape(flat.shape)
    return Value(flat.sum(0), err.sum(0) + (170 + 16 * rows / 512) * U * size.sum(0))


# ---- rotary ----------------------------------------------------------------------------------------------

def pair_channels(axis_pairs, pairs):
    """(first channel, second channel, axis) of every pair."""
    out, off, total = [], 0, sum(axis_pairs)
    for a, p in enumerate(axis_pairs):
        for i in range(p):
            j = off + i
            out.append({"halves": (2 * off + i, 2 * off + i + p, a), "neighbours": (2 * j, 2 * j + 1, a), "whole": (j, j + total, a)}[pairs])
        off += p
    return out


def turn(v, cos, sin, at, axis_pairs, pairs, dtype, sign=1.0):
    """v [n, heads, 64]; at [n, axes]: rows of the tables, held into them."""
    x, err = v.x.clone(), v.err.clone()
    at = at.long().clamp(0, cos.shape[0] - 1)
    for j, (a, b, axis) in enumerate(pair_channels(axis_pairs, pairs)):
        c, s = cos[at[:, axis], j].double()[:, None], sign * sin[at[:, axis], j].double()[:, None]
        x[..., a], x[..., b] = v.x[..., a] * c - v.x[..., b] * s, v.x[..., b] * c + v.x[..., a] * s
        size = v.x[..., a].abs() * c.abs() + v.x[..., b].abs() * s.abs(), v.x[..., b].abs() * c.abs() + v.x[..., a].abs() * s.abs()
        err[..., a], err[..., b] = v.err[..., a] * c.abs() + v.err[..., b] * s.abs(), v.err[..., b] * c.abs() + v.err[..., a] * s.abs()
        if dtype != torch.float32:
            err[..., a] += U * size[0]
            err[..., b] += U * size[1]
    return Value(x, err + 3 * U * x.abs())


def rotary(x, weight, bias, cos, sin, at, axis_pairs, pairs, kind, eps, d_out=None):
    """One of q and k: results and bounds by name: out, dx, d_weight, d_bias."""
    turns = cos is not None
    n, inv = norm(given(x), kind, eps) if kind else (given(x), None)
    y = affine(n, weight, bias)
    y = turn(y, cos, sin, at, axis_pairs, pairs, x.dtype) if turns else y
    r = {"out": y.stored(x.dtype)}
    if d_out is None:
        return r
    g = given(d_out)
    g = turn(g, cos, sin, at, axis_pairs, pairs, x.dtype, -1.0) if turns else g
    w_dtype = x.dtype if weight is None else weight.dtype
    if kind:
        rows = x.shape[0]
        r["d_weight"], r["d_bias"] = sum_rows(g * n, rows).stored(w_dtype), sum_rows(g, rows).stored(w_dtype)
        g = norm_back(g if weight is None else g * given(weight), n, inv, kind)
    r["dx"] = g.stored(x.dtype)
    return r


# ---- the residual stream -----------------------------------------------------------------------------------

def residual(x, f=None, kind=None, weight=None, bias=None, eps=1e-6, post=None, post_weight=None, post_bias=None, scale=None, gate=None,
             seq=None, residual_scale=1.0, d_r=None, d_y=None, dtype=None, w_dtype=None):
    """Results and bounds by name.  gate [batch, width] with seq [n], the sequence of every row.  dtype: of y and f."""
    dtype, w_dtype, rows = dtype or x.dtype, w_dtype or x.dtype, x.shape[0]
    r, width = given(x), x.shape[1]
    if f is not None:
        n_post, inv_post = norm(given(f), post, eps) if post else (given(f), None)
        u = affine(n_post, post_weight, post_bias)
        n_part = n_post.x.abs() if post_weight is None else (n_post.x * post_weight.double()).abs()
        b_part = torch.zeros_like(n_part) if post_bias is None else post_bias.double().abs().expand_as(n_part)
        u.err = u.err + 2 * U * (n_part + b_part)
        s = Value(torch.full((1, width), residual_scale, dtype=torch.float64, device=x.device))
        s = s if scale is None else s * given(scale)
        gates = None if gate is None else Value(gate[seq])
        s = s if gate is None else s * gates
        r = r + s * u
    out = {"r": r.stored(x.dtype)}
    if kind:
        n, inv = norm(r, kind, eps)
        out["y"] = affine(n, weight, bias).stored(dtype)
    if d_r is None and d_y is None:
        return out
    d = given(d_r) if d_r is not None else Value(torch.zeros_like(x, dtype=torch.float64))
    if d_y is not None:
        g = given(d_y)
        out["d_weight"], out["d_bias"] = sum_rows(g * n, rows).stored(w_dtype), sum_rows(g, rows).stored(w_dtype)
        back = norm_back(g if weight is None else g * given(weight), n, inv, kind)
        d = d + back
    out["dx"] = d.stored(x.dtype)
    if f is None:
        return out
    t, du = d * u, d * s
    t.err = t.err + 3 * U * d.x.abs() * (n_part + b_part)
    t_size = d.x.abs() * (n_part + b_part)
    few = Value(torch.full((1, 1), residual_scale, dtype=torch.float64, device=x.device))
    out["d_scale"] = (sum_rows(t if gate is None else t * gates, rows, t_size if gate is None else t_size * gates.x.abs()) * few).stored(w_dtype)
    if gate is not None:
        by_scale = few if scale is None else few * given(scale)
        parts = [sum_rows(Value(t.x[seq == b], t.err[seq == b]), rows, t_size[seq == b]) * by_scale for b in range(gate.shape[0])]
        x_, e_ = torch.cat([p.x.reshape(1, -1) for p in parts]), torch.cat([p.err.reshape(1, -1) for p in parts])
        out["d_gate"] = Value(x_, e_).stored(dtype)
    if post:
        out["d_post_weight"], out["d_post_bias"] = sum_rows(du * n_post, rows).stored(w_dtype), sum_rows(du, rows).stored(w_dtype)
        du = norm_back(du if post_weight is None else du * given(post_weight), n_post, inv_post, post)
    out["df"] = du.stored(dtype)
    return out


def check(name, got, want, floor=1e-36):
    """Every element within its bound; NaNs and infinities in the same places."""
    want, tol = want
    got, want, tol = got.double(), want.reshape(got.shape), tol.reshape(got.shape)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{name}: NaN in other places"
    wild = torch.isinf(want)
    assert torch.equal(got[wild], want[wild]), f"{name}: infinities differ"
    off = ((got - want).abs() / (tol + floor))[torch.isfinite(want)]
    worst = float(off.max()) if off.numel() else 0.0
    print(f"{name}: {worst:.3f} of its bound", flush=True)
    assert worst <= 1.0, f"{name}: off by {worst} times its bound"
