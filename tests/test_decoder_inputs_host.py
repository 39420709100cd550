"""The inputs that tell a lost piece, and the reference that rounds a rotated row once, do what the GPU tests need of them."""
import pytest
import torch

from tests.decoder_once import next_to_ties, to_bf16_once
from tests.decoder_util import check, rotated
from tests.pieces_util import UNIT, plant, planted_reference, planted_tokens


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("m,pieces", [(10992, 1), (10992, 40), (300_000, 256)])
def test_a_lost_unit_or_piece_is_out_of_bounds(dtype, m, pieces):
    """With 2500 planted keys at most, the longest case is as hard as one of millions of tokens."""
    g = torch.Generator().manual_seed(m)
    q, k, v = (torch.randn((n, 1, 64), generator=g).to(dtype) for n in (3, m, m))
    at = plant(q, k, v, 1)
    want = planted_reference(q[:, 0], k[:, 0], v[:, 0], 0.125, dtype, pieces)
    own = {"out": want["out"].to(dtype), "lse": want["lse"].float()}
    for name in own:
        check(name, own[name], want[name], want[name + "_tol"])
    per = (m + pieces - 1) // pieces
    first = int(at[len(at) // 2]) // UNIT * UNIT
    lost = {"a unit": torch.arange(first, min(first + UNIT, m)), "the last token": torch.tensor([m - 1]), "the first token": torch.tensor([0])}
    if pieces > 1:
        lost.update({"a piece": torch.arange(per * (pieces // 2), per * (pieces // 2 + 1)), "the last piece": torch.arange(per * (pieces - 1), m)})
    for what, tokens in lost.items():
        bad = planted_reference(q[:, 0], k[:, 0], v[:, 0], 0.125, dtype, pieces, tokens)["out"]
        with pytest.raises(AssertionError, match="times its bound"):
            check(what, bad.to(dtype), want["out"], want["out_tol"])
    with pytest.raises(AssertionError, match="times its bound"):
        check("zeros", torch.zeros_like(q[:, 0]), want["out"], want["out_tol"])


@pytest.mark.parametrize("m", [1, 63, 64, 65, 10992, 1_500_000])
def test_planted_tokens_are_in_every_so_many_units(m):
    at = planted_tokens(m, "cpu")
    assert int(at[0]) == 0 and int(at[-1]) == m - 1 and len(at) <= 2502
    units = torch.unique(at // UNIT)
    assert int((units[1:] - units[:-1]).max() if len(units) > 1 else 0) <= (m // UNIT + 2500) // 2500


def test_rounding_once_to_bf16():
    x = torch.tensor([1 + 2.0 ** -8, 1 + 3 * 2.0 ** -8, 1 + 2.0 ** -8 + 2.0 ** -40, 1 + 3 * 2.0 ** -8 - 2.0 ** -40, -1 - 2.0 ** -8 - 2.0 ** -40, 2 - 2.0 ** -8 + 2.0 ** -45,
                      0.0, 3.0], dtype=torch.float64)
    assert to_bf16_once(x).tolist() == [1.0, 1 + 2.0 ** -6, 1 + 2.0 ** -7, 1 + 2.0 ** -7, -1 - 2.0 ** -7, 2.0, 0.0, 3.0]
    y = torch.randn(100_000, generator=torch.Generator().manual_seed(1), dtype=torch.float64)
    assert torch.equal(to_bf16_once(y.float().double()), y.float().bfloat16())       # from fp32 there is one rounding in any case


@pytest.mark.parametrize("axes", [1, 2])
@pytest.mark.parametrize("neighbours", [False, True])
def test_rows_next_to_ties_tell_two_roundings_from_one(axes, neighbours):
    q, cos, sin = next_to_ties(200, 3, axes, torch.Generator().manual_seed(2), "cpu")
    x = rotated(q.double(), torch.arange(200)[:, None].expand(200, axes), cos, sin, neighbours)
    once, twice, cut = to_bf16_once(x), x.float().bfloat16(), (x.float().view(torch.int32) & -65536).view(torch.float32).bfloat16()
    assert float((once != twice).float().mean()) > 0.2 and float((once != cut).float().mean()) > 0.2
    assert bool(((once.double() - x).abs() <= 2.0 ** -8 * x.abs()).all())
