"""GPU tests of cross attention, its gradient and the 4-bit cache on values that are rare or that tell a mistake: infinities that count, scores
that are all -inf."""
import math

import pytest
import torch

from tests.decoder_util import check, cross_reference
from tests.test_gpu_decoder import BF16, F32, SCALE, compare, gen, normal, run_cross, s3r  # noqa: F401 (s3r: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,m,heads,kv_heads", [(1, 65, 1, 1), (5, 300, 2, 1), (16, 64, 2, 2), (3, 9000, 4, 2), (60, 700, 1, 1), (150, 700, 2, 2)])
def test_infinite_values_that_count(s3r, n, m, heads, kv_heads):  # noqa: F811
    """bf16: an infinity in v is one in out, in its channel, for every row that sees it, however many rows there are; two of either
    sign are NaN; log-sums, other channels and the gradient of v, which does not read v, are as without it."""
    g = gen(n + m)
    q, k, v = (normal(g, r, h, 64, dtype=BF16) for r, h in ((n, heads), (m, kv_heads), (m, kv_heads)))
    d_out = normal(g, n, heads, 64, dtype=BF16)
    v[m // 3, :, 3], v[m - 1, :, 5] = math.inf, -math.inf
    v[0, :, 40], v[m // 2, :, 40] = math.inf, -math.inf
    got = run_cross(s3r, q, k, v, d_out)
    want = cross_reference(q, k, v, [(0, n, 0, m)], None, SCALE, d_out)
    assert bool((want["out"][..., 3] == math.inf).all()) and bool((want["out"][..., 5] == -math.inf).all()) and bool(torch.isnan(want["out"][..., 40]).all())
    for name in ("out", "lse", "dv"):
        check(name, got[name], want[name], want[name + "_tol"])


@pytest.mark.parametrize("n,m,heads,kv_heads", [(1, 65, 1, 1), (8, 300, 2, 1), (64, 200, 1, 1), (3, 9000, 2, 2), (150, 700, 2, 2)])
def test_infinite_gradients_that_count(s3r, n, m, heads, kv_heads):  # noqa: F811
    """bf16: an infinity in d_out is one in dv, in its channel, for every key; other channels of dv are as without it."""
    g = gen(n + m)
    q, k, v = (normal(g, r, h, 64, dtype=BF16) for r, h in ((n, heads), (m, kv_heads), (m, kv_heads)))
    d_out = normal(g, n, heads, 64, dtype=BF16)
    d_out[0, :, 3], d_out[n - 1, :, 50] = math.inf, -math.inf
    got = run_cross(s3r, q, k, v, d_out)
    want = cross_reference(q, k, v, [(0, n, 0, m)], None, SCALE, d_out)
    assert bool((want["dv"][..., 3] == math.inf).all()) and bool((want["dv"][..., 50] == -math.inf).all())
    check("dv", got["dv"], want["dv"], want["dv_tol"])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,m", [(1, 40), (5, 700), (3, 9000), (150, 700), (150, 9000)])
def test_rows_whose_scores_are_all_minus_infinity_whatever_the_values(s3r, dtype, rows, m):  # noqa: F811
    """Such a row is 0 also where values are infinities or NaN; the other head's rows are as ever."""
    g = gen(rows + m)
    q, k, v = normal(g, rows, 2, 64, dtype=dtype).abs() + 1, normal(g, m, 2, 64, dtype=dtype), normal(g, m, 2, 64, dtype=dtype)
    k[:, 1] = -math.inf
    v[0, 1], v[m // 2, 1, ::3], v[m - 1, 1, 1::3] = math.nan, math.inf, -math.inf
    got = run_cross(s3r, q, k, v)
    assert bool((got["out"][:, 1] == 0).all()) and bool((got["lse"][1] == -math.inf).all())
    want = cross_reference(q[:, :1], k[:, :1], v[:, :1], [(0, rows, 0, m)], None, SCALE)
    compare({"out": got["out"][:, :1], "lse": got["lse"][:1]}, want)
