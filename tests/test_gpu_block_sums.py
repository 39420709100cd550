"""GPU tests of the sums over rows that the gradients of weights, scales and gates are, where plain sums in fp32 would lose something: infinities,
parts that cancel, many terms of one sign.  Against the 64-bit forms of tests/block_util.py, or with bounds derived at each test."""
import math

import pytest
import torch

from tests.block_util import check, residual
from tests.test_gpu_block import BF16, F32, TYPES, gen, normal, residual_case, run_residual, s3r, starts  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("width,post", [(64, None), (1024, None), (1024, "rms"), (4096, "rms"), (8192, None)])
def test_an_infinite_gradient_without_a_post_bias(s3r, types, width, post):
    """An infinity in d_r is one in the gradients of scale, gate and post weight of its channel, whose terms are its products with finite numbers:
    a bias that there is not takes no part in them (0 times an infinite sum of d_r would make them NaN)."""
    rows = [20, 1, 16]
    c = residual_case(width, 37, width, *types, post=post, rows=rows, bias=False)
    c["d_r"][5, 3], c["d_r"][20, 9], c["d_r"][30, width - 1] = math.inf, -math.inf, math.inf
    got = run_residual(s3r, c)
    seq = torch.repeat_interleave(torch.arange(3, device="cuda"), torch.tensor(rows, device="cuda"))
    want = residual(c["x"], c["f"], "layer", c["weight"], None, 1e-6, post, c["post_weight"], None, c["scale"], c["gate"], seq, 0.75, c["d_r"], c["d_y"],
                    c["dtype"], c["w_dtype"])
    for name in ("d_scale", "d_gate") + (("d_post_weight",) if post else ()):
        assert torch.isinf(want[name][0]).any() and not torch.isnan(want[name][0]).any()
        check(name, got[name], want[name])
    # without gates, the sums of rows of which each is its own
    plain = {**c, "gate": None, "row_start": None}
    got = run_residual(s3r, plain)
    want = residual(c["x"], c["f"], "layer", c["weight"], None, 1e-6, post, c["post_weight"], None, c["scale"], None, None, 0.75, c["d_r"], c["d_y"],
                    c["dtype"], c["w_dtype"])
    check("d_scale", got["d_scale"], want["d_scale"])
