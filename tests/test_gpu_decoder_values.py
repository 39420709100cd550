"""GPU tests of cross attention, its gradient and the 4-bit cache on values that are rare or that tell a mistake: infinities that count."""
import math

import pytest
import torch

from tests.decoder_util import check, cross_reference
from tests.test_gpu_decoder import BF16, SCALE, gen, normal, run_cross, s3r  # noqa: F401 (s3r: the fixture)

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
