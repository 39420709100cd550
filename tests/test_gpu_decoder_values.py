"""GPU tests of cross attention, its gradient and the 4-bit cache on values that are rare or that tell a mistake: infinities that count, scores
that are all -inf, rotated rows next to a border of their rounding."""
import math

import pytest
import torch

from tests.decoder_once import next_to_ties, to_bf16_once
from tests.decoder_util import check, cross_reference, four_bits, packed, rotated
from tests.test_gpu_decoder import BF16, F32, SCALE, compare, gen, new_cache, normal, run_cross, s3r, tables_of_angles  # noqa: F401 (s3r: the fixture)

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


def append_one_sequence(s3r, k, v, page, **kw):  # noqa: F811
    """The rows as a sequence of their own; codes and exponents of the keys, row by row."""
    n, heads = k.shape[:2]
    width = (n + page - 1) // page
    cache, pt = new_cache(s3r, width, heads, page), torch.arange(width, dtype=torch.int32, device="cuda")[None]
    s3r.speed3r_cache_append(cache, k, v, pt, torch.tensor([n], dtype=torch.int32, device="cuda"), **kw)
    return tuple(t.permute(0, 2, 1, 3).reshape(width * page, heads, -1)[:n] for t in (cache.k_codes, cache.k_scales))


@pytest.mark.parametrize("axes", [1, 2])
@pytest.mark.parametrize("pairs", ["halves", "neighbours"])
@pytest.mark.parametrize("n,heads,kv_heads", [(1, 1, 1), (777, 6, 2)])
def test_rotated_bf16_queries_are_rounded_once(s3r, n, heads, kv_heads, axes, pairs):  # noqa: F811
    """Bit by bit: random rows, and powers of two whose exact results lie next to the middle of two bf16 numbers, nearer than fp32 can tell."""
    g = gen(n + axes)
    at = torch.arange(n, device="cuda")[:, None].expand(n, axes)
    kw = {"positions": at.int().contiguous(), "pairs": pairs}
    tied, cos_t, sin_t = next_to_ties(n, heads, axes, g, "cuda")
    for q, (cos, sin) in ((normal(g, n, heads, 64, dtype=BF16), tables_of_angles(n, 32 // axes)), (tied, (cos_t, sin_t))):
        k, out = normal(g, n, kv_heads, 64, dtype=BF16), torch.full_like(q, math.nan)
        append_one_sequence(s3r, k, k, 32, q=q, q_out=out, cos=cos, sin=sin, **kw)
        assert torch.equal(out, to_bf16_once(rotated(q.double(), at, cos, sin, pairs == "neighbours")))


@pytest.mark.parametrize("axes", [1, 2])
@pytest.mark.parametrize("pairs", ["halves", "neighbours"])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_codes_next_to_a_border_in_every_order_of_pairs(s3r, dtype, axes, pairs):  # noqa: F811
    """Channels at a tie of the 4-bit form or at a change of exponent, turned by cosines of 1 and sines of 2^-30 to 2^-45 (the
    exact value is off the border by less than fp32 can tell), and fp32 rows that a turn brings next to one."""
    n = 1000
    g = gen(23)
    at = torch.arange(n, device="cuda")[:, None].expand(n, axes)
    border = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0], device="cuda")
    want = border[torch.randint(0, 8, (n, 2, 64), generator=g, device="cuda")] * torch.where(torch.rand((n, 2, 64), generator=g, device="cuda") < 0.5, -1, 1)
    _, _, sin = next_to_ties(n, 1, axes, g, "cuda")
    cases = [(want.to(dtype), torch.ones_like(sin), sin)]
    if dtype == F32:
        cos, sin = tables_of_angles(n, 32 // axes)
        cases.append((rotated(want.double(), at, cos, -sin, pairs == "neighbours").float(), cos, sin))
    for k, cos, sin in cases:
        codes, scales = append_one_sequence(s3r, k, k, 64, cos=cos, sin=sin, positions=at.int().contiguous(), pairs=pairs)
        code, scale = four_bits(rotated(k.double(), at, cos, sin, pairs == "neighbours"))
        assert torch.equal(codes, packed(code)) and torch.equal(scales, scale)
