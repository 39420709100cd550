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


@pytest.mark.parametrize("x_dtype,dtype", [(F32, F32), (BF16, BF16), (F32, BF16)])
@pytest.mark.parametrize("n,width,lengths", [
    (800, 64, None), (100000, 64, None), (800, 64, [500, 1, 0, 299]), (800, 128, [800]), (800, 256, None), (800, 520, [700, 100]), (3000, 1000, None),
    (800, 1024, [500, 1, 299]), (800, 2048, [800]), (800, 4096, [1, 799]), (800, 8192, None), (800, 8192, [300, 0, 77, 423]), (1500, 64, [1] * 1500)])
def test_products_that_cancel_before_they_are_summed(s3r, x_dtype, dtype, n, width, lengths):
    """Rows of one number, so that the post-norm leaves the same nu of all, and u = nu w + b with w = 1.5, b = -w nu (1 - 2^-16): of the gradients of scale
    and gate, sums of dr' u, each part, w sum dr' nu and b sum dr', is 2^16 times the whole, and a rounding of one of them to fp32 is 2^-8 of it.

    nu is known to 6 u alone (u = 2^-24), but is the same for all rows and channels, as is the rounding of nu w + b: a gradient over the exact sum of its
    channel's d_r (y is not asked for, so that dr' is d_r) has to be the same for all channels but for the roundings of sums of terms of one sign: up to 8 rows
    of a thread, 32 rows side by side and, where sequences are single rows, 32 of these, the products with the gate and with scale, and the store: 44 u, 76 u
    for single rows, either way."""
    g = gen(width)
    exact_nu = 1.625 / math.sqrt(1.625 ** 2 + 0.3)
    f, w = torch.full((n, width), 1.625, dtype=dtype, device="cuda"), torch.full((width,), 1.5, device="cuda")
    b, scale = (-w.double() * exact_nu * (1 - 2.0 ** -16)).float(), torch.full((width,), 0.5, device="cuda")
    d_r = (1 + torch.rand((n, width), generator=g, device="cuda")).to(x_dtype)
    gate = torch.ones((len(lengths), width), dtype=dtype, device="cuda") if lengths else None
    x = torch.zeros((n, width), dtype=x_dtype, device="cuda")
    grads = {"d_scale": torch.full((width,), math.nan, device="cuda")}
    if lengths:
        grads["d_gate"] = torch.full(gate.shape, math.nan, dtype=dtype, device="cuda")
    s3r.speed3r_residual_norm_backward(x, None, torch.empty_like(x), d_r=d_r, df=torch.empty_like(f), f=f, post_norm="rms", post_weight=w, post_bias=b, scale=scale,
                                       gate=gate, row_start=starts(lengths) if lengths else None, eps=0.3, **grads)
    u = 2.0 ** -24
    nu_err = 7 * u * 2.0 ** 16                                        # of what nu w + b is, and a rounding of b

    def same(name, got, size, factor, store):
        ratio = got.double() / size / (1.5 * exact_nu * factor * 2.0 ** -16)
        mean = float(ratio.mean())
        off = float((ratio - mean).abs().max()) / mean
        bound = (76 if lengths and len(lengths) > 300 else 44) * u + store
        print(f"{name}: {mean:.6f}, {off / bound:.3f} of its bound", flush=True)
        assert abs(mean - 1) <= nu_err + store and off <= 2 * bound

    same("d_scale", grads["d_scale"], d_r.double().sum(0), 1.0, 0.0)
    if lengths:
        store = torch.finfo(dtype).eps / 2 if dtype != F32 else 0.0
        for i, part in enumerate(d_r.double().split(lengths)):
            if lengths[i] == 0:
                assert not grads["d_gate"][i].any()
            elif i < 10:
                same(f"d_gate {i}", grads["d_gate"][i], part.sum(0), 0.5, store)


ALIKE = 1 + 2.0 ** -13 + 2.0 ** -21    # 1024 to 4096 of them added in fp32, each to the sum of those before, end 2^-14 of the sum too high


def close_to(name, got, want, bound):
    off = float((got.double() / want - 1).abs().max())
    print(f"{name}: {off / bound:.3f} of its bound", flush=True)
    assert off <= bound, name


@pytest.mark.parametrize("post,lengths", [(None, None), ("rms", None), ("rms", [2 ** 26 - 5, 1, 4]), (None, [2 ** 26])])
def test_millions_of_terms_of_one_sign(s3r, post, lengths):
    """2^26 rows of eight channels, whose terms are all the same: a thread has 4096 of them.  At most 256 are added in fp32, 32 rows side by side are,
    and beyond that 64 bits: 288 u of the sum, and 8 u for n and u (the norm of ones), gate, scale and the store."""
    n, width, u = 2 ** 26, 8, 2.0 ** -24
    ones = torch.ones((n, width), device="cuda")
    d = torch.full((n, width), ALIKE, device="cuda")
    weight = torch.ones(width, device="cuda")
    names = ["d_scale", "d_post_weight", "d_post_bias"] if post else ["d_scale"]
    grads = {name: torch.full((width,), math.nan, device="cuda") for name in names}
    gate = torch.ones((len(lengths), width), device="cuda") if lengths else None
    if lengths:
        grads["d_gate"] = torch.full_like(gate, math.nan)
    s3r.speed3r_residual_norm_backward(ones, None, torch.empty_like(ones), d_r=d, f=ones.clone(), df=torch.empty_like(ones), post_norm=post, eps=2.0 ** -40,
                                       post_weight=weight if post else None, scale=weight, gate=gate, row_start=starts(lengths) if lengths else None, **grads)
    for name in names:
        close_to(name, grads[name], n * d[0, 0].double(), 296 * u)
    for b, length in enumerate(lengths or []):
        close_to(f"d_gate {b}", grads["d_gate"][b], length * d[0, 0].double(), 296 * u)
    if lengths is None:
        grads = {name: torch.full((width,), math.nan, device="cuda") for name in ("d_weight", "d_bias")}
        s3r.speed3r_residual_norm_backward(ones, d, torch.empty_like(ones), norm="rms", weight=weight, eps=2.0 ** -40, **grads,
                                           **(dict(f=torch.zeros_like(ones), df=torch.empty_like(ones), post_norm=post, post_weight=weight) if post else {}))
        for name in grads:
            close_to(name, grads[name], n * d[0, 0].double(), 296 * u)


@pytest.mark.parametrize("width", [64, 8192])
def test_many_sequences_of_a_row_in_one_workgroup(s3r, width):
    """60000 sequences of a row before a long one, so that some workgroups have hundreds of sequences (or thousands) to add up: terms that are all the
    same, as above."""
    n, u = (2 ** 23, 2.0 ** -24) if width == 64 else (2 ** 17, 2.0 ** -24)
    lengths = [1] * 60000 + [n - 60000]
    ones = torch.ones((n, width), device="cuda")
    d = torch.full((n, width), ALIKE, device="cuda")
    weight, gate = torch.ones(width, device="cuda"), torch.ones((len(lengths), width), device="cuda")
    grads = {name: torch.full((width,), math.nan, device="cuda") for name in ("d_scale", "d_post_weight", "d_post_bias")}
    grads["d_gate"] = torch.full_like(gate, math.nan)
    s3r.speed3r_residual_norm_backward(ones, None, torch.empty_like(ones), d_r=d, f=ones.clone(), df=torch.empty_like(ones), post_norm="rms", eps=2.0 ** -40,
                                       post_weight=weight, scale=weight, gate=gate, row_start=starts(lengths), **grads)
    for name in ("d_scale", "d_post_weight", "d_post_bias"):
        close_to(name, grads[name], n * d[0, 0].double(), 296 * u)
    close_to("d_gate of a row", grads["d_gate"][:60000], d[0, 0].double(), 10 * u)
    close_to("d_gate of many", grads["d_gate"][60000], lengths[-1] * d[0, 0].double(), 296 * u)


def test_millions_of_rotated_rows_of_one_sign(s3r):
    """2^26 heads of rows, whose terms are all the same in the channels that are turned (by a cosine of that value): a lane has 4096 of them.  At most the 16
    heads of a run are added in fp32, four waves at the end, with 5 u for n (the norm of ones), and three roundings: 28 u."""
    n, heads, u = 2 ** 22, 16, 2.0 ** -24
    ones = torch.ones((n, heads, 64), dtype=BF16, device="cuda")
    cos, sin = torch.full((1, 11), ALIKE, device="cuda"), torch.zeros((1, 11), device="cuda")
    weight = torch.ones(64, device="cuda")
    grads = {name: torch.full((64,), math.nan, device="cuda") for name in ("dq_weight", "dq_bias")}
    s3r.speed3r_rotary_backward(ones, None, ones, None, torch.empty_like(ones), None, cos, sin, axis_pairs=(11,), norm="rms", eps=2.0 ** -40, q_weight=weight, **grads)
    for name in grads:
        close_to(name, grads[name][:22], n * heads * cos[0, 0].double(), 28 * u)
        close_to(name + " of others", grads[name][22:], torch.tensor(float(n * heads), dtype=torch.float64, device="cuda"), 28 * u)


def multiples(g, bits, *shape):
    """Random multiples of 2^-bits in [0, 1)."""
    return torch.randint(0, 2 ** bits, shape, generator=g, device="cuda") * 2.0 ** -bits


@pytest.mark.parametrize("n,width,bits", [(2 ** 14, 64, 19), (2048, 1024, 22), (512, 8192, 24), (2 ** 23, 64, 11), (2 ** 18, 2048, 14)])
def test_workgroups_are_added_up_in_64_bits(s3r, n, width, bits):
    """Gradients of a bias whose sums are exact in fp32 within a workgroup (24 bits: 5, 2, 0, 13 and 9 for the rows of one, of which those beyond 256 for a thread
    are added in 64 bits) and take more bits together: the result is the exact sum, rounded once."""
    d = multiples(gen(n), bits, n, width)
    x = torch.ones_like(d)
    d_bias = torch.full((width,), math.nan, device="cuda")
    s3r.speed3r_residual_norm_backward(x, d, torch.empty_like(x), norm="rms", d_bias=d_bias)
    assert torch.equal(d_bias, d.sum(0, dtype=torch.float64).float())


@pytest.mark.parametrize("n,heads,bits", [(2 ** 16, 1, 19), (2 ** 16, 16, 14)])
def test_workgroups_of_rotated_rows_are_added_up_in_64_bits(s3r, n, heads, bits):
    """As above: 32 rows for a workgroup of 2048, or 512 heads of rows."""
    d = multiples(gen(n + heads), bits, n, heads, 64)
    q = torch.ones_like(d)
    dq_bias = torch.full((64,), math.nan, device="cuda")
    s3r.speed3r_rotary_backward(q, None, d, None, torch.empty_like(q), None, norm="rms", dq_bias=dq_bias)
    assert torch.equal(dq_bias, d.sum((0, 1), dtype=torch.float64).float())


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("width,n", [(64, 700), (1024, 60), (4096, 60), (8192, 60), (8192, 1500), (64, 2 ** 17 + 700)])
@pytest.mark.parametrize("gated", [False, True])
def test_each_gradient_by_itself(s3r, types, width, n, gated):
    """A gradient that is asked for alone has the bits that it has beside all others (sequences that share a workgroup; 300 of a row in one, so that a thread's
    sums go to the workspace in shares, where n is large)."""
    rows = ([1] * 300 + [n - 310, 4, 0, 6] if n > 1000 else [n // 2, 1, 0, n - n // 2 - 1]) if gated else None
    c = residual_case(n + width, n, width, *types, post="layer", rows=rows)
    want = run_residual(s3r, c)
    how = {name: c[name] for name in ("f", "norm", "weight", "post_norm", "post_weight", "post_bias", "scale", "gate", "row_start")}
    for name in ("d_weight", "d_bias", "d_post_weight", "d_post_bias", "d_scale", "d_gate"):
        if name not in want:
            continue
        got = torch.full_like(want[name], math.nan)
        dx, df = torch.empty_like(c["x"]), torch.empty_like(c["f"])
        s3r.speed3r_residual_norm_backward(c["x"], c["d_y"], dx, d_r=c["d_r"], df=df, eps=1e-6, residual_scale=0.75, **{name: got}, **how)
        assert torch.equal(got, want[name]), name
        assert torch.equal(dx, want["dx"]) and torch.equal(df, want["df"]), name


@pytest.mark.parametrize("width,n", [(64, 2 ** 17 + 700), (8192, 1500)])
def test_shares_replay_from_a_graph(s3r, width, n):
    """Sums that go to the workspace in shares, replayed with other contents and sequences between eager calls: the bits of an eager call (places of the
    workspace are written before they are added to)."""
    c = residual_case(n, n, width, rows=[1] * 300 + [n - 310, 4, 0, 6], post="layer")
    names = ("d_weight", "d_bias", "d_post_weight", "d_post_bias", "d_scale", "d_gate")
    want = run_residual(s3r, c)
    out = {name: torch.zeros_like(want[name]) for name in (*names, "dx", "df")}

    def step():
        how = {name: c[name] for name in ("f", "norm", "weight", "post_norm", "post_weight", "post_bias", "scale", "gate", "row_start")}
        s3r.speed3r_residual_norm_backward(c["x"], c["d_y"], out["dx"], d_r=c["d_r"], df=out["df"], eps=1e-6, residual_scale=0.75,
                                           **{name: out[name] for name in names}, **how)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(3):
        g = gen(turn)
        for t in (c["x"], c["d_y"], c["gate"]):
            t.copy_(normal(g, *t.shape, dtype=t.dtype))
        c["row_start"].copy_(starts([[1] * 300 + [n - 310, 4, 0, 6], [0] * 303 + [n], [2] * 300 + [0, n - 600, 0, 0]][turn]))
        for t in out.values():
            t.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        want = run_residual(s3r, c)
        assert all(torch.equal(out[name], want[name]) for name in out), turn
