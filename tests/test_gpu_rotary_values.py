"""GPU tests of rotary positions whose products cancel, against the 64-bit form of tests/block_util.py."""
import math

import pytest
import torch

from tests.block_util import check, given, pair_channels, turn
from tests.test_gpu_block import AXES, BF16, F32, gen, nan_like, normal, s3r  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("pairs", ["halves", "neighbours", "whole"])
@pytest.mark.parametrize("axis_pairs", AXES)
def test_products_that_cancel(s3r, dtype, pairs, axis_pairs):
    """Pairs of equal channels (and of opposite ones), turned by 45 degrees: one of the results is exactly 0, as products that are rounded alike, or not at all,
    leave it.  All are within 3 * 2^-24 and their own rounding, of the result and not of its parts, in bf16 as in fp32."""
    g = gen(sum(axis_pairs))
    x = normal(g, 30, 3, 64, dtype=dtype)
    channels = pair_channels(axis_pairs, pairs)
    for j, (a, b, _) in enumerate(channels):
        x[..., b] = x[..., a] if j % 2 else -x[..., a]
    cos = torch.full((5, sum(axis_pairs)), math.sqrt(0.5), device="cuda")
    sin = cos.clone()
    at = torch.randint(0, 5, (30, len(axis_pairs)), generator=g, device="cuda").int()
    out, dq = nan_like(x), nan_like(x)
    s3r.speed3r_rotary(x, None, out, None, cos, sin, at, axis_pairs=axis_pairs, pairs=pairs)
    s3r.speed3r_rotary_backward(None, None, x, None, dq, None, cos, sin, at, axis_pairs=axis_pairs, pairs=pairs)
    for name, got, sign in (("out", out, 1.0), ("dq", dq, -1.0)):
        want = turn(given(x), cos, sin, at, axis_pairs, pairs, F32, sign)
        for j, (a, b, _) in enumerate(channels):
            none = a if (j % 2 == 1) == (sign > 0) else b
            assert not want.x[..., none].any()
        check(name, got, want.stored(dtype))
