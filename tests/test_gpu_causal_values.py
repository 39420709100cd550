"""GPU tests of what causal attention makes of rare values and of rows that see few keys, against the plain 64-bit form of tests/decoder_util.py."""
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
