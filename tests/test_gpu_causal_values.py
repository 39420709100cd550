"""GPU tests of what causal attention makes of rare values and of keys that few rows see, against the plain 64-bit form of tests/decoder_util.py."""
import math

import pytest
import torch

from tests.decoder_util import check
from tests.test_gpu_causal import BF16, F32, gen, inputs, normal, reference, run, s3r, starts, what_rows_see  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,m,at,peaks,upto", [
    (300, 300, 130, {135: 200, 220: 400}, 256),      # the maximum rises in the unit of the infinity, and in a later one
    (300, 300, 190, {3: 200}, 256), (12, 140, 131, {5: 200}, 140),           # it was there before; other waves have it
    (4, 20000, 19998, {70: 200}, 20000), (300, 20000, 19750, {70: 200, 19800: 400}, 19828),   # other pieces have it
    (12, 80, 69, {75: 200}, 80)])
def test_an_infinity_whose_weight_underflows(s3r, dtype, n, m, at, peaks, upto):
    """A row that sees an infinite value has an infinity in that channel however small its weight (e^-200 and e^-400 of the largest: 0 in fp32), where the unit
    of 64 keys is one that not all rows of its tile see (tokens below `upto`); its other channels are as without it.  Elsewhere 0 times it may be NaN, as
    in cross attention."""
    g = gen(n + m + at)
    level = torch.zeros(m, device="cuda")
    for key, x in peaks.items():
        level[key] = x
    q, k = torch.zeros((n, 2, 64), device="cuda"), torch.zeros((m, 2, 64), device="cuda")
    q[:, :, 0], k[:, :, 0] = 8.0, level[:, None]                           # scores: the levels (scale 1 / 8)
    q, k, v = q.to(dtype), k.to(dtype), normal(g, m, 2, 64, dtype=dtype)
    want = reference(q, k, v, [(0, n, 0, m)], 1)
    bad = v.clone()
    bad[at, :, 3] = math.inf
    got = run(s3r, q, k, bad)
    check("lse", got["lse"], want["lse"], want["lse_tol"])
    others = [c for c in range(64) if c != 3]
    check("out", got["out"][..., others], want["out"][..., others], want["out_tol"][..., others])
    token = torch.arange(m - n, m, device="cuda")
    check("before", got["out"][token < at][..., 3], want["out"][token < at][..., 3], want["out_tol"][token < at][..., 3])
    here = got["out"][(token >= at) & (token < upto)][..., 3].float()
    finite = int(torch.isfinite(got["out"][token >= at][..., 3].float()).sum())
    assert here.numel() > 0 and finite == 0
    if dtype == BF16:
        wrong = int((here != math.inf).sum())
        assert wrong == 0


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,m,at", [(300, 300, 130), (12, 140, 131), (4, 20000, 70), (300, 20000, 70), (300, 20000, 19750)])
def test_a_score_that_is_none_is_seen_in_results_and_log_sums(s3r, dtype, n, m, at):
    """A row that sees a key with a NaN has NaN in all channels and its log-sum, in whichever unit, wave or piece the key is; the others do not."""
    q, k, v, _ = inputs(n + at, n, m, 2, 2, dtype)
    k[at, 0, 5] = math.nan
    got = run(s3r, q, k, v)
    sees = torch.arange(m - n, m, device="cuda") >= at
    assert torch.isnan(got["out"][sees, 0].float()).all() and torch.isnan(got["lse"][0, sees]).all()
    assert torch.isfinite(got["out"][~sees, 0].float()).all() and torch.isfinite(got["lse"][0, ~sees]).all()
    assert torch.isfinite(got["out"][:, 1].float()).all() and torch.isfinite(got["lse"][1]).all()


def attention_of_two_parts(q, k, v, seen, scale, d_out):
    """As attention() of tests/decoder_util.py, bounds where probabilities and dS of bf16 rows enter their products in two bf16 parts, off by h^2 (h = 2^-8)
    and not by h.  u = 2^-24.
      out   (d + h^2 + chain) sum P |v| and h |out| for the store.
      D     of the stored out is off by up to |d_out| err(out), which is taken out again: of dk by the fp32 sum of dS, (d + chain + 4 u) sum |dS| + sum P err(dP)
            are left; of dq by that of the parts of dS as they enter, times P k with P in one part: h (|d_out| err(out) + h^2 sum |dS|) sum P |k| as well.
      dS    P ((d + h^2 + 4 u) |dP - D| + err(D) + err(dP)), through |k| and |q|;  dv: (d + h^2) P^T |d_out|."""
    u, h = 2.0 ** -24, 2.0 ** -8
    q, k, v, g = q.double(), k.double(), v.double(), d_out.double()
    n, m = seen.shape
    s = ((q @ k.t()) * scale).masked_fill(~seen, -math.inf)
    size = (q.abs() @ k.abs().t()) * scale
    lse = torch.logsumexp(s, 1)
    p = torch.where(seen, torch.exp(s - lse[:, None]), 0.0)
    d = (64 * u * size + (torch.where(seen, s, 0.0).abs() + 4) * u).masked_fill(~seen, 0.0).amax(1, keepdim=True) * 2
    chain, pairs = (m / 8 + 64) * u, (max(n, m) / 8 + 64) * u
    out = p @ v
    out_tol = (d + h * h + chain) * (p @ v.abs()) + h * out.abs()
    dp, delta = g @ v.t(), (g * out).sum(1, keepdim=True)
    dp_err = 64 * u * (g.abs() @ v.abs().t())
    ds = p * (dp - delta)
    first = (g.abs() * out_tol).sum(1, keepdim=True) + 64 * u * (g * out).abs().sum(1, keepdim=True)
    d_err = (d + chain + 4 * u) * ds.abs().sum(1, keepdim=True) + (p * dp_err).sum(1, keepdim=True)
    err = p * ((d + h * h + 4 * u) * (dp - delta).abs() + d_err + dp_err)
    r = {"out": out, "out_tol": out_tol}
    for name, a, b, e in (("dq", ds, k, err + p * h * (first + h * h * ds.abs().sum(1, keepdim=True))), ("dk", ds.t(), q, err.t()), ("dv", p.t(), g, (p * (d + h * h)).t())):
        f = 1.0 if name == "dv" else scale
        x = f * (a @ b)
        r[name], r[name + "_tol"] = x, f * (e @ b.abs() + pairs * (a.abs() @ b.abs())) + h * x.abs()
    return r


@pytest.mark.parametrize("n,m,view,heads,kv_heads", [(700, 700, 1, 2, 2), (300, 300, 1, 4, 1), (130, 700, 1, 6, 2), (129, 129, 1, 3, 3), (500, 520, 20, 3, 1), (2500, 2500, 1, 4, 1),
                                                     (200, 200, 1, 16, 1), (640, 640, 1, 1, 1), (1000, 9000, 1, 2, 1)])
def test_last_keys_whose_gradients_have_few_terms(s3r, n, m, view, heads, kv_heads):
    """bf16 keys that up to 64 rows see, counting those of all heads that share one: their gradients are off by their own rounding and 2^-16 of the terms, as in
    sequences of so few rows (a term rounded once would be most of the error of such a sum)."""
    q, k, v, d_out = inputs(n + m + heads, n, m, heads, kv_heads, BF16)
    got = run(s3r, q, k, v, d_out, view)
    share, seen = heads // kv_heads, what_rows_see(n, m, view)
    keys = seen.sum(0) * share <= 64
    assert keys[-1] and not keys[0]
    rows = seen[:, keys].any(1)
    for kh in range(kv_heads):
        sums = {}
        for h in range(kh * share, (kh + 1) * share):
            x = attention_of_two_parts(q[rows, h], k[:, kh], v[:, kh], seen[rows], 0.125, d_out[rows, h])
            for name in ("dk", "dk_tol", "dv", "dv_tol"):
                sums[name] = sums.get(name, 0.0) + x[name][keys]
        for name in ("dk", "dv"):
            check(name, got[name][keys, kh], sums[name], sums[name + "_tol"])


def test_last_keys_of_packed_sequences(s3r):
    """The same over sequences side by side."""
    rows, keys = [300, 70, 1, 129, 500], [300, 570, 40, 1000, 500]
    q, k, v, d_out = inputs(5, sum(rows), sum(keys), 2, 1, BF16)
    a, b = starts(rows), starts(keys)
    got = run(s3r, q, k, v, d_out, q_start=a, kv_start=b)
    q0 = k0 = 0
    for n, m in zip(rows, keys):
        seen = what_rows_see(n, m, 1)
        last = seen.sum(0) * 2 <= 64
        x = [attention_of_two_parts(q[q0:q0 + n, h], k[k0:k0 + m, 0], v[k0:k0 + m, 0], seen, 0.125, d_out[q0:q0 + n, h]) for h in range(2)]
        for name in ("dk", "dv"):
            check(name, got[name][k0:k0 + m, 0][last], (x[0][name] + x[1][name])[last], (x[0][name + "_tol"] + x[1][name + "_tol"])[last])
        q0, k0 = q0 + n, k0 + m


@pytest.mark.parametrize("n,m,view,heads,kv_heads", [(700, 700, 1, 2, 2), (1500, 1500, 1, 4, 1), (300, 2000, 1, 6, 2), (900, 900, 100, 3, 3), (129, 5000, 1, 2, 2),
                                                     (500, 300, 0, 2, 1), (1374, 2748, 0, 2, 2)])
def test_two_parts_where_the_caller_asks_for_them(s3r, n, m, view, heads, kv_heads):
    """accurate_pv: results of many bf16 rows are off by their own rounding and 2^-16 of the terms, causal (view > 0) and not; without it they need not be (which
    the bounds of the other tests allow).  Rows in fp32 are as they were."""
    q, k, v, d_out = inputs(n + m, n, m, heads, kv_heads, BF16)
    share = heads // kv_heads

    def results(accurate, *t):
        if view:
            return run(s3r, *t, view, accurate_pv=accurate)
        q, k, v, d_out = t
        r = {"out": torch.empty_like(q), "lse": torch.empty((heads, n), device="cuda"), "dq": torch.empty_like(q), "dk": torch.empty_like(k), "dv": torch.empty_like(v)}
        s3r.speed3r_cross_attn(q, k, v, r["out"], lse=r["lse"], accurate_pv=accurate)
        s3r.speed3r_cross_attn_backward(q, k, v, r["out"], r["lse"], d_out, r["dq"], r["dk"], r["dv"], accurate_pv=accurate)
        return r

    got, plain = results(True, q, k, v, d_out), results(False, q, k, v, d_out)
    assert torch.equal(got["lse"], plain["lse"]) and not torch.equal(got["out"], plain["out"])
    seen = what_rows_see(n, m, view) if view else torch.ones((n, m), dtype=torch.bool, device="cuda")
    for kh in range(kv_heads):
        sums = {}
        for h in range(kh * share, (kh + 1) * share):
            x = attention_of_two_parts(q[:, h], k[:, kh], v[:, kh], seen, 0.125, d_out[:, h])
            for name in ("out", "dq"):
                check(name, got[name][:, h], x[name], x[name + "_tol"])
            for name in ("dk", "dk_tol", "dv", "dv_tol"):
                sums[name] = sums.get(name, 0.0) + x[name]
        for name in ("dk", "dv"):
            check(name, got[name][:, kh], sums[name], sums[name + "_tol"])
    f32 = [t[:200].float() for t in (q, k, v, d_out)]
    n = m = 200
    a, b = results(True, *f32), results(False, *f32)
    assert all(torch.equal(a[name], b[name]) for name in a)
