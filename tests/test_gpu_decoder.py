"""GPU tests of cross attention, its gradient and the 4-bit cache through the binding, against plain 64-bit forms
(tests/decoder_util.py, which derives the bounds)."""
import math

import pytest
import torch

from tests.decoder_util import attention, check, cross_reference, four_bits, packed, rotated, values

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
SCALE = 0.125


@pytest.fixture(scope="module")
def s3r():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2603_08055_amd import speed3r
    speed3r.load()
    return speed3r


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, *shape, dtype=F32, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def starts(lengths, first=0):
    s = [first]
    for n in lengths:
        s.append(s[-1] + n)
    return torch.tensor(s, dtype=torch.int32, device="cuda")


def nan_like(t, dtype=None):
    return torch.full(t.shape, math.nan, dtype=dtype or t.dtype, device=t.device)


def run_cross(s3r, q, k, v, d_out=None, **kw):
    """Forward (and gradient) into buffers full of NaN."""
    r = {"out": nan_like(q), "lse": torch.full((q.shape[1], q.shape[0]), math.nan, device="cuda")}
    s3r.speed3r_cross_attn(q, k, v, r["out"], lse=r["lse"], **kw)
    if d_out is not None:
        r.update(dq=torch.full(q.shape, math.nan, dtype=q.dtype, device="cuda"), dk=torch.full(k.shape, math.nan, dtype=q.dtype, device="cuda"),
                 dv=torch.full(k.shape, math.nan, dtype=q.dtype, device="cuda"))
        s3r.speed3r_cross_attn_backward(q, k, v, r["out"], r["lse"], d_out, r["dq"], r["dk"], r["dv"], **kw)
    torch.cuda.synchronize()
    return r


def compare(got, want):
    for name in got:
        check(name, got[name], want[name], want[name + "_tol"])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,m,heads,kv_heads", [
    (1, 1, 1, 1), (1, 64, 2, 1), (2, 63, 3, 3), (31, 65, 4, 2), (32, 129, 1, 1), (33, 200, 2, 2), (127, 64, 2, 2),
    (128, 1, 1, 1), (129, 500, 6, 2), (300, 700, 8, 1), (1, 5000, 2, 2), (3, 3001, 16, 2), (700, 2, 3, 1), (5, 0, 2, 1), (64, 4097, 1, 1),
])
def test_cross_and_its_gradient(s3r, dtype, n, m, heads, kv_heads):
    g = gen(n * 1000 + m)
    q, k, v = normal(g, n, heads, 64, dtype=dtype, scale=2.0), normal(g, m, kv_heads, 64, dtype=dtype), normal(g, m, kv_heads, 64, dtype=dtype)
    d_out = normal(g, n, heads, 64, dtype=dtype)
    got = run_cross(s3r, q, k, v, d_out)
    compare(got, cross_reference(q, k, v, [(0, n, 0, m)], None, SCALE, d_out))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,m,heads,kv_heads", [(0, 70, 4, 2), (0, 0, 1, 1), (1, 700, 32, 1), (2, 90, 16, 1), (300, 9000, 32, 32)])
def test_cross_without_rows_with_many_heads_and_many_pieces(s3r, dtype, n, m, heads, kv_heads):
    g = gen(n + m + heads)
    q, k, v = (normal(g, r, h, 64, dtype=dtype) for r, h in ((n, heads), (m, kv_heads), (m, kv_heads)))
    d_out = normal(g, n, heads, 64, dtype=dtype)
    compare(run_cross(s3r, q, k, v, d_out), cross_reference(q, k, v, [(0, n, 0, m)], None, SCALE, d_out))


BATCHES = {"130 of few rows": ([1, 2, 3] * 43 + [1], 40), "one long among many": ([1] * 70 + [300] + [1] * 30, 100), "100 single rows": ([1] * 100, 150)}


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("which", list(BATCHES))
def test_cross_batches_of_more_than_a_wave(s3r, dtype, which):
    rows, most = BATCHES[which]
    g = gen(len(rows))
    keys = torch.randint(0, most, (len(rows),), generator=g, device="cuda").tolist()
    q, k, v = normal(g, sum(rows), 4, 64, dtype=dtype), normal(g, sum(keys), 2, 64, dtype=dtype), normal(g, sum(keys), 2, 64, dtype=dtype)
    d_out = normal(g, sum(rows), 4, 64, dtype=dtype)
    a, b = starts(rows), starts(keys)
    spans = [(int(x), r, int(y), c) for x, y, r, c in zip(a, b, rows, keys)]
    compare(run_cross(s3r, q, k, v, d_out, q_start=a, kv_start=b), cross_reference(q, k, v, spans, None, SCALE, d_out))


@pytest.mark.parametrize("stride", [1 << 22, 1 << 24])
def test_rows_far_apart(s3r, stride):
    """Rows of k and v further than 2^32 bytes from the first, and further apart than a 32-bit offset within a unit reaches."""
    g = gen(77)
    m = (5 << 30) // (2 * stride)
    room = torch.zeros(m * stride, dtype=BF16, device="cuda")
    k, v = (room.as_strided((m, 1, 64), (stride, 64, 1), at) for at in (0, 64))
    k.copy_(normal(g, m, 1, 64, dtype=BF16)), v.copy_(normal(g, m, 1, 64, dtype=BF16))
    for n in (1, 100):
        q, d_out = normal(g, n, 1, 64, dtype=BF16), normal(g, n, 1, 64, dtype=BF16)
        got = {"out": nan_like(q), "lse": torch.empty((1, n), device="cuda"), "dq": nan_like(q),
               "dk": torch.empty((m, 1, 64), dtype=BF16, device="cuda"), "dv": torch.empty((m, 1, 64), dtype=BF16, device="cuda")}
        s3r.speed3r_cross_attn(q, k, v, got["out"], lse=got["lse"])
        s3r.speed3r_cross_attn_backward(q, k, v, got["out"], got["lse"], d_out, got["dq"], got["dk"], got["dv"])
        compare(got, cross_reference(q, k, v, [(0, n, 0, m)], None, SCALE, d_out))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads,kv_heads", [(2, 2), (6, 2)])
def test_ragged_batches_masks_and_what_must_not_matter(s3r, dtype, heads, kv_heads):
    """Sequences without rows or keys, a sequence whose keys are all masked, rows before the first and behind the last
    sequence, NaN and infinities in masked and outside rows."""
    g = gen(7)
    rows, keys = [40, 0, 1, 150, 33, 7], [100, 64, 0, 333, 65, 20]
    n, m, q0, k0 = sum(rows) + 12, sum(keys) + 9, 5, 4
    q, k, v = normal(g, n, heads, 64, dtype=dtype), normal(g, m, kv_heads, 64, dtype=dtype), normal(g, m, kv_heads, 64, dtype=dtype)
    d_out = normal(g, n, heads, 64, dtype=dtype)
    mask = torch.rand(m, generator=g, device="cuda") < 0.7
    spans, a, b = [], q0, k0
    for r, c in zip(rows, keys):
        spans.append((a, r, b, c))
        a, b = a + r, b + c
    mask[spans[4][2]:spans[4][2] + 65] = False
    inside = torch.zeros(m, dtype=torch.bool, device="cuda")
    inside[k0:k0 + sum(keys)] = True
    for t, x in ((k, math.nan), (v, math.inf)):
        t[~mask | ~inside] = x
    k[~mask & (torch.arange(m, device="cuda") % 2 == 0)] = -math.inf
    v[~mask & (torch.arange(m, device="cuda") % 3 == 0)] = math.nan
    status = torch.full((1,), -1, dtype=torch.int32, device="cuda")
    kw = {"q_start": starts(rows, q0), "kv_start": starts(keys, k0), "key_mask": mask, "status": status}
    got = run_cross(s3r, q, k, v, d_out, **kw)
    assert int(status) == 0
    compare(got, cross_reference(q, k, v, spans, mask, SCALE, d_out))
    assert torch.equal(got["dk"][mask.logical_not() & inside], torch.zeros_like(got["dk"][mask.logical_not() & inside]))
    again = run_cross(s3r, q, k, v, d_out, **kw)
    for name in got:
        assert torch.equal(torch.nan_to_num(got[name].float()), torch.nan_to_num(again[name].float())), name


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,m", [(17, 300), (260, 130), (1, 4000)])
def test_strided_views(s3r, dtype, n, m):
    """q out of a packed projection, k and v out of one [m, kv_heads, 2, 64] tensor and head-major storage."""
    g = gen(3)
    q = normal(g, n, 3, 4, 64, dtype=dtype)[:, 1]
    kv = normal(g, m, 2, 2, 64, dtype=dtype)
    d_out = normal(g, n, 4, 64, dtype=dtype)
    got = run_cross(s3r, q, kv[:, :, 0], kv[:, :, 1], d_out)
    compare(got, cross_reference(q, kv[:, :, 0], kv[:, :, 1], [(0, n, 0, m)], None, SCALE, d_out))
    k, v = (normal(g, 2, m, 64, dtype=dtype).transpose(0, 1) for _ in range(2))
    got = run_cross(s3r, q, k, v, d_out, softmax_scale=0.3)
    compare(got, cross_reference(q, k, v, [(0, n, 0, m)], None, 0.3, d_out))


@pytest.mark.parametrize("n,m,heads,kv_heads", [(1, 64, 4, 1), (16, 300, 8, 2), (60, 2000, 2, 2)])
def test_key_gradients_of_few_rows_are_rounded_once(s3r, n, m, heads, kv_heads):
    """bf16, up to 64 rows of the heads that share one: P and dS enter in two bf16 parts (2^-16 and 2^-17 for the part that is
    left out and for its truncation: 2^-15 covers both), D is what the dS lack of 0, and one rounding is left, that of dk and dv."""
    g = gen(21)
    q, k, v, d_out = (normal(g, x, h, 64, dtype=BF16) for x, h in ((n, heads), (m, kv_heads), (m, kv_heads), (n, heads)))
    got = run_cross(s3r, q, k, v, d_out)
    share, u, h = heads // kv_heads, 2.0 ** -24, 2.0 ** -8
    chain = (m / 8 + 64 + share * n) * u
    for kv in range(kv_heads):
        dk, dv, dk_tol, dv_tol = 0.0, 0.0, 0.0, 0.0
        for head in range(kv * share, (kv + 1) * share):
            x, y, gd, vd = q[:, head].double(), k[:, kv].double(), d_out[:, head].double(), v[:, kv].double()
            s = x @ y.t() * SCALE
            p = torch.softmax(s, 1)
            err = 2 * (64 * u * (x.abs() @ y.abs().t()) * SCALE + (s.abs() + 8) * u).amax(1, keepdim=True) + chain        # of P, relative
            dp, out = gd @ vd.t(), p @ vd
            ds = p * (dp - (gd * out).sum(1, keepdim=True))
            size = (dp.abs() + (gd.abs() * out.abs()).sum(1, keepdim=True)) * (1 + h)
            off_d = (chain + err) * (p * size).sum(1, keepdim=True) + 64 * u * (gd.abs() @ vd.abs().t()).amax(1, keepdim=True)
            ds_tol = (err + 2.0 ** -15) * p * size + p * off_d + p * 64 * u * (gd.abs() @ vd.abs().t())
            dk, dv = dk + SCALE * ds.t() @ x, dv + p.t() @ gd
            dk_tol = dk_tol + SCALE * (ds_tol + chain * ds.abs()).t() @ x.abs()
            dv_tol = dv_tol + (p * (err + 2.0 ** -15 + chain)).t() @ gd.abs()
        check("dk", got["dk"][:, kv], dk, dk_tol + h * dk.abs())
        check("dv", got["dv"][:, kv], dv, dv_tol + h * dv.abs())


def test_gradient_against_differences(s3r):
    """fp32: (f(x + t d) - f(x - t d)) / 2 t of f = sum(out * d_out), computed by the forward kernel in fp32 and summed in
    64 bits, against the gradient's product with d.  Cancellation leaves err(out) sqrt(n) / t; the cubic term is t^2: with t = 2^-4
    and directions of norm 1 the two are below 1e-4 and 4e-3 of the gradient's norm."""
    g = gen(11)
    n, m, H, KH = 37, 90, 4, 2
    q, k, v, d_out = (normal(g, *s, 64) for s in ((n, H), (m, KH), (m, KH), (n, H)))
    r = run_cross(s3r, q, k, v, d_out)

    def f(*x):
        out = torch.empty_like(q)
        s3r.speed3r_cross_attn(*x, out)
        return float((out.double() * d_out.double()).sum())
    for i, name in enumerate(("dq", "dk", "dv")):
        d = r[name] / r[name].norm()
        t, x = 2.0 ** -4, [q, k, v]
        up, down = list(x), list(x)
        up[i], down[i] = x[i] + t * d, x[i] - t * d
        slope, want = (f(*up) - f(*down)) / (2 * t), float(r[name].double().norm())
        print(name, slope, want, flush=True)
        assert abs(slope - want) <= 5e-3 * want


def test_large_scores_and_outliers(s3r):
    """Scores of hundreds: one key takes all of a row; a maximum that rises unit by unit."""
    g = gen(5)
    for dtype in (BF16, F32):
        q, k, v = normal(g, 70, 2, 64, dtype=dtype), normal(g, 900, 2, 64, dtype=dtype), normal(g, 900, 2, 64, dtype=dtype)
        k = (k.float() * torch.linspace(0, 30, 900, device="cuda")[:, None, None]).to(dtype)
        d_out = normal(g, 70, 2, 64, dtype=dtype)
        compare(run_cross(s3r, q, k, v, d_out), cross_reference(q, k, v, [(0, 70, 0, 900)], None, SCALE, d_out))


def test_infinities_and_nan_that_count(s3r):
    """A NaN in a key reaches the rows of its head and nothing else; -inf scores weigh nothing."""
    g = gen(6)
    q, k, v = (normal(g, n, 2, 64) for n in (40, 100, 100))
    k[17, 0, 3] = math.nan
    got = run_cross(s3r, q, k, v)
    assert torch.isnan(got["out"][:, 0]).all() and torch.isfinite(got["out"][:, 1]).all()
    q, k = q.abs(), normal(g, 100, 2, 64)
    k[17:90] = -math.inf
    keep = torch.ones(100, dtype=torch.bool, device="cuda")
    keep[17:90] = False
    compare(run_cross(s3r, q, k, v), cross_reference(q, k, v, [(0, 40, 0, 100)], keep, SCALE))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows", [5, 150])
def test_rows_whose_scores_are_all_minus_infinity(s3r, dtype, rows):
    g = gen(7)
    q, k, v = normal(g, rows, 2, 64, dtype=dtype).abs() + 1, normal(g, 700, 2, 64, dtype=dtype), normal(g, 700, 2, 64, dtype=dtype)
    k[:, 1] = -math.inf
    got = run_cross(s3r, q, k, v)
    assert bool((got["out"][:, 1] == 0).all()) and bool((got["lse"][1] == -math.inf).all())
    assert torch.isfinite(got["out"][:, 0]).all() and torch.isfinite(got["lse"][0]).all()


def test_broken_starts_are_reported_and_stay_in_range(s3r):
    g = gen(8)
    q, k, v = (normal(g, n, 1, 64, dtype=BF16) for n in (50, 80, 80))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for qs, ks in (([0, 60, 50], [0, 40, 80]), ([0, 20, 50], [0, 90, 80]), ([-3, 20, 50], [0, 40, 80]), ([0, 20, 50], [50, 40, 80])):
        kw = {"q_start": torch.tensor(qs, dtype=torch.int32, device="cuda"), "kv_start": torch.tensor(ks, dtype=torch.int32, device="cuda")}
        run_cross(s3r, q, k, v, q.clone(), status=status, **kw)
        assert int(status) == s3r.S3R_DIAG_SPANS


# ---- the cache ------------------------------------------------------------------------------------------

def new_cache(s3r, n_pages, kv_heads, page):
    cache = s3r.PagedCache.empty(n_pages, kv_heads, page)
    for t in cache:
        t.fill_(0xEE)
    return cache


def table(g, batch, width, n_pages):
    return torch.randperm(n_pages, generator=g, device="cuda")[:batch * width].reshape(batch, width).int()


def tables_of_angles(places, pairs):
    angle = torch.arange(places, device="cuda").double()[:, None] * 10000.0 ** (-torch.arange(pairs, device="cuda").double() / pairs)
    return torch.cos(angle).float(), torch.sin(angle).float()


def where(page_table, lengths, rows, page):
    """Page, token in it, and token number of every row."""
    pages, offsets, tokens = [], [], []
    for b, (n, r) in enumerate(zip(lengths, rows)):
        t = torch.arange(n - r, n, device="cuda")
        pages.append(page_table[b].long()[t // page])
        offsets.append(t % page)
        tokens.append(t)
    return torch.cat(pages), torch.cat(offsets), torch.cat(tokens)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("page,axes,neighbours,heads,kv_heads", [(16, 1, False, 4, 2), (32, 1, True, 3, 3), (64, 2, False, 5, 1),
                                                                (128, 2, True, 2, 2), (16, 0, False, 0, 3)])
def test_append_and_read(s3r, dtype, page, axes, neighbours, heads, kv_heads):
    """Codes and exponents are those of the exact rotated values, byte for byte; other slots stay as they were."""
    g = gen(page + axes)
    rows, lengths = [1, 70, 0, 17, 300], [1, 130, 9, 17, 777]
    n, width = sum(rows), max(lengths) // page + 2
    k, v = (normal(g, n, kv_heads, 64) * torch.exp(3 * normal(g, n, kv_heads, 1)) for _ in range(2))
    v[3] = 0.0
    v[4, 0] = 1e-35
    v[5, 0, :7] = torch.tensor([3.5, 0.25, 0.75, 1.25, 1.75, 2.5, 5.0])          # ties in units of 1
    v[6, 0] = -3.0e38
    v[7, 0, 40] = math.nan
    k[8, 0, 5] = math.inf
    k[9] = 0.0
    k, v = k.to(dtype), v.to(dtype)
    cache, pt = new_cache(s3r, 5 * width + 2, kv_heads, page), table(g, 5, width, 5 * width + 2)
    before = [t.clone() for t in cache]
    kv_len, kw = torch.tensor(lengths, dtype=torch.int32, device="cuda"), {}
    pages, offsets, tokens = where(pt, lengths, rows, page)
    want_k = k.double()
    if axes:
        cos, sin = tables_of_angles(800, 32 // axes)
        at = tokens[:, None]
        if axes == 2:
            at = torch.randint(0, 800, (n, 2), generator=g, device="cuda")
            kw["positions"] = at.int()
        q = normal(g, n, heads, 64, dtype=dtype)
        kw.update(cos=cos, sin=sin, pairs="neighbours" if neighbours else "halves", q=q, q_out=nan_like(q))
        want_k = rotated(want_k, at, cos, sin, neighbours)
    status = torch.full((1,), -1, dtype=torch.int32, device="cuda")
    s3r.speed3r_cache_append(cache, k, v, pt, kv_len, starts(rows), status=status, **kw)
    assert int(status) == 0
    for t, old, (code, scale), is_code in ((cache.k_codes, before[0], four_bits(want_k), True), (cache.v_codes, before[1], four_bits(v.double()), True),
                                           (cache.k_scales, before[2], four_bits(want_k), False), (cache.v_scales, before[3], four_bits(v.double()), False)):
        want = old.clone()
        want[pages, :, offsets] = packed(code) if is_code else scale
        assert torch.equal(t, want)
    if axes:
        want_q = rotated(q.double(), at, cos, sin, neighbours)
        check("q", kw["q_out"], want_q, want_q.abs() * torch.finfo(dtype).eps / 2)
        assert torch.equal(kw["q_out"], want_q.to(dtype) if dtype == F32 else kw["q_out"])
    ko, vo = nan_like(k), nan_like(v)
    ko.zero_(), vo.zero_()
    s3r.speed3r_cache_read(cache, ko, vo, pt, kv_len, starts(rows), status=status)
    assert int(status) == 0
    for got, t, s in ((ko, cache.k_codes, cache.k_scales), (vo, cache.v_codes, cache.v_scales)):
        want = values(t[pages, :, offsets], s[pages, :, offsets])
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.nan_to_num(got.double()), torch.nan_to_num(want))


def test_rounding_next_to_a_border(s3r):
    """fp32 rows whose rotated channels lie within one step of fp32 of a tie or of a change of exponent: the code is that of the
    exact value, which fp32 arithmetic would not tell."""
    n = 4096
    g = gen(21)
    cos, sin = tables_of_angles(n, 32)
    border = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0], device="cuda").double()
    want = border[torch.randint(0, 8, (n, 1, 64), generator=g, device="cuda")] * torch.where(torch.rand((n, 1, 64), generator=g, device="cuda") < 0.5, -1, 1)
    k = rotated(want, torch.arange(n, device="cuda")[:, None], cos, -sin, False).float()      # back by the angle, rounded to fp32
    cache, pt = new_cache(s3r, n // 64, 1, 64), torch.arange(n // 64, dtype=torch.int32, device="cuda")[None]
    s3r.speed3r_cache_append(cache, k, k, pt, torch.tensor([n], dtype=torch.int32, device="cuda"), cos=cos, sin=sin)
    code, scale = four_bits(rotated(k.double(), torch.arange(n, device="cuda")[:, None], cos, sin, False))
    assert torch.equal(cache.k_codes.permute(0, 2, 1, 3).reshape(n, 1, 32), packed(code))
    assert torch.equal(cache.k_scales.permute(0, 2, 1, 3).reshape(n, 1, 2), scale)


def filled_cache(s3r, g, n_pages, kv_heads, page):
    cache = s3r.PagedCache.empty(n_pages, kv_heads, page)
    for codes, scales in ((cache.k_codes, cache.k_scales), (cache.v_codes, cache.v_scales)):
        code, scale = four_bits(normal(g, n_pages, kv_heads, page, 64).double())
        codes.copy_(packed(code))
        scales.copy_(scale)
    return cache


def cached(cache, pt, b, length, kv_head):
    """k, v of a sequence's tokens in 64 bits."""
    page = cache.k_codes.shape[2]
    t = torch.arange(length, device="cuda")
    at = pt[b].long()[t // page], kv_head, t % page
    return values(cache.k_codes[at], cache.k_scales[at]), values(cache.v_codes[at], cache.v_scales[at])


def attend_reference(cache, q, pt, lengths, rows, causal, scale=SCALE):
    H, KH = q.shape[1], cache.k_codes.shape[1]
    r = {"out": nan_like(q, torch.float64), "lse": torch.full((H, q.shape[0]), math.nan, dtype=torch.float64, device="cuda")}
    r["out_tol"], r["lse_tol"] = torch.zeros_like(r["out"]), torch.zeros_like(r["lse"])
    first = 0
    for b, (length, n) in enumerate(zip(lengths, rows)):
        for h in range(H):
            k, v = cached(cache, pt, b, length, h // (H // KH))
            last = torch.arange(length - n, length, device="cuda") if causal else torch.full((n,), length - 1, device="cuda")
            seen = torch.arange(length, device="cuda")[None] <= last[:, None]
            x = attention(q[first:first + n, h], k, v, seen, scale, q.dtype)
            s = slice(first, first + n)
            r["out"][s, h], r["lse"][h, s], r["out_tol"][s, h], r["lse_tol"][h, s] = x["out"], x["lse"], x["out_tol"], x["lse_tol"]
        first += n
    return r


def run_attend(s3r, cache, q, pt, lengths, rows, causal, **kw):
    out, lse = nan_like(q), torch.full((q.shape[1], q.shape[0]), math.nan, device="cuda")
    status = torch.full((1,), -1, dtype=torch.int32, device="cuda")
    s3r.speed3r_cache_attn(cache, q, out, pt, torch.tensor(lengths, dtype=torch.int32, device="cuda"), starts(rows), causal=causal, lse=lse,
                           status=status, **kw)
    assert int(status) == 0
    return {"out": out, "lse": lse}


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("page,heads,kv_heads,rows,lengths", [
    (16, 4, 2, [1], [1]), (16, 8, 1, [1, 1, 1], [17, 64, 1000]), (32, 2, 2, [40], [40]), (64, 3, 3, [130, 1, 0, 65], [130, 700, 33, 128]),
    (128, 6, 2, [31, 200], [31, 1500]), (64, 2, 1, [1], [9000]), (128, 1, 1, [3], [5000]), (16, 5, 5, [100, 7], [50, 0]),
])
def test_cache_attention(s3r, dtype, causal, page, heads, kv_heads, rows, lengths):
    """From one token to thousands; sequences with more rows than tokens, whose first rows see nothing (causal), and none at all."""
    g = gen(page * 7 + heads)
    width = max(lengths) // page + 1
    cache = filled_cache(s3r, g, width * len(rows) + 1, kv_heads, page)
    pt = table(g, len(rows), width, width * len(rows) + 1)
    q = normal(g, sum(rows) + 3, heads, 64, dtype=dtype, scale=2.0)
    got = run_attend(s3r, cache, q, pt, lengths, rows, causal)
    compare(got, attend_reference(cache, q, pt, lengths, rows, causal))
    assert torch.isnan(got["out"][sum(rows):]).all()                               # rows behind the last sequence


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("which", list(BATCHES))
def test_cache_batches_of_more_than_a_wave(s3r, dtype, page, which):
    rows, most = BATCHES[which]
    g = gen(len(rows) + page)
    lengths = [r + int(x) for r, x in zip(rows, torch.randint(0, 2 * most, (len(rows),), generator=g, device="cuda"))]
    width = max(lengths) // page + 1
    cache = filled_cache(s3r, g, width * len(rows), 2, page)
    pt = table(g, len(rows), width, width * len(rows))
    q = normal(g, sum(rows), 4, 64, dtype=dtype)
    for causal in (True, False):
        compare(run_attend(s3r, cache, q, pt, lengths, rows, causal), attend_reference(cache, q, pt, lengths, rows, causal))


@pytest.mark.parametrize("rows", [2, 150])
def test_pages_that_sequences_share(s3r, rows):
    """Two sequences with the same first pages, one that has a page twice: the same as with pages of their own."""
    g = gen(32)
    page, lengths = 64, [300, 290, 200]
    cache = filled_cache(s3r, g, 24, 2, page)
    shared = torch.tensor([[3, 7, 5, 2, 11], [3, 7, 5, 9, 0], [6, 6, 4, 6, 1]], dtype=torch.int32, device="cuda")
    own = s3r.PagedCache(*(t[shared.flatten().long()].contiguous() for t in cache))
    apart = torch.arange(15, dtype=torch.int32, device="cuda").reshape(3, 5)
    q = normal(g, 3 * rows, 4, 64, dtype=BF16)
    for causal in (True, False):
        a, b = (run_attend(s3r, c, q, pt, lengths, [rows] * 3, causal) for c, pt in ((cache, shared), (own, apart)))
        assert torch.equal(a["out"], b["out"]) and torch.equal(a["lse"], b["lse"])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_cache_rows_in_larger_tensors(s3r, dtype):
    """k, v and q as slices of one projection; rows read back into slices, and what lies between them left alone."""
    g = gen(91)
    n, page = 50, 32
    packed_rows = normal(g, n, 8, 64, dtype=dtype)
    q, k, v = packed_rows[:, :4], packed_rows[:, 4:6], packed_rows[:, 6:]
    cos, sin = tables_of_angles(n, 32)
    pt, kv_len = table(g, 1, 2, 3), torch.tensor([n], dtype=torch.int32, device="cuda")
    one, two = s3r.PagedCache.empty(3, 2, page), s3r.PagedCache.empty(3, 2, page)
    turned, again = torch.empty((n, 4, 64), dtype=dtype, device="cuda"), torch.empty((n, 4, 64), dtype=dtype, device="cuda")
    s3r.speed3r_cache_append(one, k, v, pt, kv_len, q=q, q_out=turned, cos=cos, sin=sin)
    s3r.speed3r_cache_append(two, k.contiguous(), v.contiguous(), pt, kv_len, q=q.contiguous(), q_out=again, cos=cos, sin=sin)
    assert torch.equal(turned, again) and all(torch.equal(a, b) for a, b in zip(one, two))
    room = torch.full((n, 3, 2, 64), 7.0, dtype=dtype, device="cuda")
    s3r.speed3r_cache_read(one, room[:, 0], room[:, 2], pt, kv_len)
    ko, vo = torch.empty((n, 2, 64), dtype=dtype, device="cuda"), torch.empty((n, 2, 64), dtype=dtype, device="cuda")
    s3r.speed3r_cache_read(one, ko, vo, pt, kv_len)
    assert torch.equal(room[:, 0], ko) and torch.equal(room[:, 2], vo) and bool((room[:, 1] == 7.0).all())
    wide = torch.empty((n, 2, 4, 64), dtype=dtype, device="cuda")
    wide[:, 1] = turned
    a, b = torch.empty_like(turned), torch.empty_like(turned)
    s3r.speed3r_cache_attn(one, wide[:, 1], a, pt, kv_len)
    s3r.speed3r_cache_attn(one, turned, b, pt, kv_len)
    assert torch.equal(a, b)


def test_no_rows_at_all(s3r):
    cache, pt = s3r.PagedCache.empty(2, 1, 16), torch.zeros((1, 2), dtype=torch.int32, device="cuda")
    kv_len, none = torch.tensor([5], dtype=torch.int32, device="cuda"), torch.empty((0, 1, 64), dtype=BF16, device="cuda")
    status = torch.full((1,), -1, dtype=torch.int32, device="cuda")
    s3r.speed3r_cache_append(cache, none, none, pt, kv_len, status=status)
    s3r.speed3r_cache_read(cache, none, none.clone(), pt, kv_len)
    s3r.speed3r_cache_attn(cache, none, none.clone(), pt, kv_len)
    assert int(status) == 0 and all(int(t.max()) == 0 for t in cache)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows", [3, 200])
def test_nan_in_the_cache_reaches_only_rows_that_see_it(s3r, dtype, rows):
    g = gen(31)
    length, page = 333, 32
    cache, pt = filled_cache(s3r, g, 12, 2, page), table(g, 1, 11, 12)
    for token, head, half, of_v in ((length - 2, 0, 1, True), (length - 1, 1, 0, False)):
        (cache.v_scales if of_v else cache.k_scales)[pt[0, token // page].long(), head, token % page, half] = 255
    tail = length % page                                                            # behind the sequence's end: what another left
    cache.v_scales[pt[0, length // page].long(), :, tail:] = 255
    cache.k_scales[pt[0, length // page].long(), :, tail:] = 255
    q = normal(g, rows, 2, 64, dtype=dtype)
    out = run_attend(s3r, cache, q, pt, [length], [rows], True)["out"]
    nan = torch.isnan(out)
    assert nan[-2:, 0, 32:].all() and not nan[:-2].any() and not nan[:, 0, :32].any() and nan[-1, 1].all() and not nan[-2, 1].any()
    assert torch.isnan(run_attend(s3r, cache, q, pt, [length], [rows], False)["out"][:, 0, 32:]).all()


@pytest.mark.parametrize("rows", [3, 200])
def test_nan_that_a_row_sees_counts_however_little_it_weighs(s3r, rows):
    """A value of NaN under a weight of e^-512, which is 0 in 32 bits; with few rows it is in a piece of its own that weighs e^-256."""
    length, page = 2000, 64
    cache, pt = s3r.PagedCache.empty(32, 1, page), torch.arange(32, dtype=torch.int32, device="cuda")[None]
    k, v = torch.zeros((length, 1, 64), dtype=BF16, device="cuda"), torch.ones((length, 1, 64), dtype=BF16, device="cuda")
    k[5], k[1900], v[5, 0, 40] = -4.0, 4.0, math.nan
    kv_len = torch.tensor([length], dtype=torch.int32, device="cuda")
    s3r.speed3r_cache_append(cache, k, v, pt, kv_len)
    out = run_attend(s3r, cache, torch.full((rows, 1, 64), 8.0, dtype=BF16, device="cuda"), pt, [length], [rows], False)["out"]
    assert torch.isnan(out[:, 0, 32:]).all() and bool((out[:, 0, :32] == 1).all())


def test_broken_lists_are_reported_and_stay_in_range(s3r):
    g = gen(41)
    page, batch, width = 16, 3, 4
    rows, lengths = [5, 5, 5], [40, 64, 33]
    good = {"pt": table(g, batch, width, 12), "len": torch.tensor(lengths, dtype=torch.int32, device="cuda"), "start": starts(rows)}

    def run(**change):
        x = dict(good, **change)
        cache = filled_cache(s3r, gen(42), 12, 2, page)
        old = [t.clone() for t in cache]
        k = normal(gen(43), 15, 2, 64, dtype=BF16)
        cos, sin = tables_of_angles(64, 32)
        status = torch.full((3,), -1, dtype=torch.int32, device="cuda")
        s3r.speed3r_cache_append(cache, k, k, x["pt"], x["len"], x["start"], cos=x.get("cos", cos), sin=x.get("sin", sin), positions=x.get("pos"),
                                 status=status[0:1])
        ko, vo, out = torch.empty_like(k), torch.empty_like(k), torch.zeros_like(k)
        s3r.speed3r_cache_read(cache, ko, vo, x["pt"], x["len"], x["start"], status=status[1:2])
        s3r.speed3r_cache_attn(cache, k, out, x["pt"], x["len"], x["start"], status=status[2:3])
        return status.tolist(), cache, old, ko, out

    assert run()[0] == [0, 0, 0]
    pt = good["pt"].clone()
    pt[1, 3] = 12                                             # the page of sequence 1's last 16 tokens
    s, cache, old, ko, out = run(pt=pt)
    assert s == [s3r.S3R_DIAG_PAGE] * 3 and float(ko[5:10].abs().max()) == 0.0 and torch.isfinite(out.float()).all()
    pt[1, 3] = -1
    assert run(pt=pt)[0] == [s3r.S3R_DIAG_PAGE] * 3
    assert run(len=torch.tensor([40, 65, 33], dtype=torch.int32, device="cuda"))[0] == [s3r.S3R_DIAG_LENGTH] * 3
    assert run(len=torch.tensor([40, -1, 33], dtype=torch.int32, device="cuda"))[0][0] & s3r.S3R_DIAG_LENGTH
    assert run(len=torch.tensor([40, 3, 33], dtype=torch.int32, device="cuda"))[0] == [s3r.S3R_DIAG_LENGTH, s3r.S3R_DIAG_LENGTH, 0]
    assert run(start=torch.tensor([0, 5, 4, 15], dtype=torch.int32, device="cuda"))[0] == [s3r.S3R_DIAG_SPANS] * 3
    assert run(start=torch.tensor([0, 5, 10, 16], dtype=torch.int32, device="cuda"))[0] == [s3r.S3R_DIAG_SPANS] * 3
    assert run(pos=torch.tensor([0] * 14 + [64], dtype=torch.int32, device="cuda"))[0] == [s3r.S3R_DIAG_POSITION, 0, 0]
    assert run(pos=torch.tensor([0] * 14 + [-1], dtype=torch.int32, device="cuda"))[0] == [s3r.S3R_DIAG_POSITION, 0, 0]
    cos, sin = tables_of_angles(63, 32)
    assert run(cos=cos, sin=sin)[0] == [s3r.S3R_DIAG_POSITION, 0, 0]


def test_offsets_past_32_bits(s3r):
    """Pages that lie more than 2^32 bytes into the arrays."""
    g = gen(51)
    page, kv_heads = 128, 8
    n_pages = (1 << 32) // (page * kv_heads * 32) + 40                              # 4.3 GB of codes, twice
    cache = s3r.PagedCache.empty(n_pages, kv_heads, page)
    pt = torch.arange(n_pages - 12, n_pages, dtype=torch.int32, device="cuda").flip(0)[None].contiguous()
    k, v = normal(g, 1500, kv_heads, 64, dtype=BF16), normal(g, 1500, kv_heads, 64, dtype=BF16)
    kv_len = torch.tensor([1500], dtype=torch.int32, device="cuda")
    s3r.speed3r_cache_append(cache, k, v, pt, kv_len)
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    s3r.speed3r_cache_read(cache, ko, vo, pt, kv_len)
    for got, x in ((ko, k), (vo, v)):
        code, scale = four_bits(x.double())
        assert torch.equal(got.double(), values(packed(code), scale))
    for rows in (1, 200):
        q = normal(g, rows, 16, 64, dtype=BF16)
        compare(run_attend(s3r, cache, q, pt, [1500], [rows], True), attend_reference(cache, q, pt, [1500], [rows], True))
    assert int(cache.k_codes[: n_pages - 12].max()) == 0


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows", [1, 20, 100])
def test_millions_of_tokens(s3r, dtype, rows):
    """A sequence that is divided into as many pieces as can be joined."""
    g = gen(53)
    page, length = 128, 1_500_000
    n_pages = (length + page - 1) // page
    cache, pt = filled_cache(s3r, g, n_pages, 1, page), torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)[None].contiguous()
    q = normal(g, rows, 1, 64, dtype=dtype)
    compare(run_attend(s3r, cache, q, pt, [length], [rows], True), attend_reference(cache, q, pt, [length], [rows], True))
    k, v = normal(g, 400_000, 1, 64, dtype=dtype), normal(g, 400_000, 1, 64, dtype=dtype)
    compare(run_cross(s3r, q, k, v), cross_reference(q, k, v, [(0, rows, 0, 400_000)], None, SCALE))


def test_more_than_2_to_the_31_elements(s3r):
    """Rows whose offset in q, out and the gradients passes 32 bits, in elements and in bytes: the last ones, and a whole head."""
    g = gen(52)
    n, m, heads = 600_000, 70, 64
    q, d_out = (torch.empty((n, heads, 64), dtype=BF16, device="cuda").normal_(generator=g) for _ in range(2))
    k, v = normal(g, m, heads, 64, dtype=BF16), normal(g, m, heads, 64, dtype=BF16)
    got = run_cross(s3r, q, k, v, d_out)
    tail = slice(n - 300, n)
    for h in range(heads):
        want = attention(q[tail, h], k[:, h], v[:, h], torch.ones((1, m), dtype=torch.bool, device="cuda"), SCALE, BF16, d_out[tail, h])
        for name in ("out", "dq"):
            check(name, got[name][tail, h], want[name], want[name + "_tol"])
        check("lse", got["lse"][h, tail], want["lse"], want["lse_tol"])
    want = attention(q[:, 63], k[:, 63], v[:, 63], torch.ones((1, m), dtype=torch.bool, device="cuda"), SCALE, BF16, d_out[:, 63])
    for name in ("out", "dq", "dk", "dv"):
        check(name, got[name][:, 63], want[name], want[name + "_tol"])


# ---- as they are used -------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,batch", [(BF16, 3), (F32, 3), (BF16, 100)])
def test_a_decoder_over_a_scene_captured_and_replayed(s3r, dtype, batch):
    """Sparse global attention gives a scene's states; a decoder layer appends a token at a time, attends its cache and the scene.  The
    step is captured once (lengths and tokens in device memory) and replayed with the program's own work between; every
    replay equals the eager call, and two graphs with workspaces of their own do not disturb each other."""
    g = gen(61)
    views, tokens, H, KH, page, width = 2, 300, 4, 2, 16, 14
    n = views * tokens
    q, k, v = (normal(g, n, H, 64, dtype=BF16) for _ in range(3))
    states = torch.empty_like(q)
    s3r.speed3r_sparse_global_attn(q, k, v, states, 64, 4)
    states = states.to(dtype)
    scene_k, scene_v = states[:, :KH], states[:, KH:]
    kv_start = starts([n] + [0] * (batch - 1))                                       # the first sequence has the scene, the others none
    cos, sin = tables_of_angles(256, 32)

    class Step:
        def __init__(self):
            self.cache = s3r.PagedCache.empty(batch * width, KH, page)
            self.pt = torch.arange(batch * width, dtype=torch.int32, device="cuda").reshape(batch, width)
            self.len = torch.tensor(([1, 5, 200] * batch)[:batch], dtype=torch.int32, device="cuda")
            self.start = starts([1] * batch)
            self.q, self.k, self.v = (torch.zeros((batch, h, 64), dtype=dtype, device="cuda") for h in (H, KH, KH))
            self.turned, self.own, self.out = (torch.zeros_like(self.q) for _ in range(3))
            dt = s3r.S3R_BF16 if dtype == BF16 else s3r.S3R_F32
            need = max(s3r.speed3r_cache_workspace_bytes(self.cache, batch, H, dt, batch, width),
                       s3r.speed3r_cross_workspace_bytes(self.q, scene_k, q_start=self.start), 1)
            self.ws = torch.empty(need, dtype=torch.uint8, device="cuda")

        def __call__(self):
            s3r.speed3r_cache_append(self.cache, self.k, self.v, self.pt, self.len, self.start, q=self.q, q_out=self.turned, cos=cos, sin=sin)
            s3r.speed3r_cache_attn(self.cache, self.turned, self.own, self.pt, self.len, self.start, workspace=self.ws)
            s3r.speed3r_cross_attn(self.own, scene_k, scene_v, self.out, q_start=self.start, kv_start=kv_start, workspace=self.ws)

        def feed(self, i):
            x = gen(100 + i)
            for t in (self.q, self.k, self.v):
                t.copy_(normal(x, *t.shape, dtype=dtype))

    eager, one, two = Step(), Step(), Step()
    side = torch.cuda.Stream()
    graphs = []
    for step in (one, two):
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        graphs.append(graph)
    for t in (*one.cache, *two.cache):
        t.zero_()
    for i in range(8):
        for step in (eager, one, two):
            step.feed(i)
        eager()
        torch.cuda.synchronize()
        for step, graph in ((one, graphs[0]), (two, graphs[1])):
            graph.replay()
        float(eager.out.float().sum())                                               # the program's own work in between
        for step in (one, two):
            assert torch.equal(step.own, eager.own) and torch.equal(step.out, eager.out), i
            for a, b in zip(step.cache, eager.cache):
                assert torch.equal(a, b)
        for step in (eager, one, two):
            step.len += 1
    assert float(eager.out[1:].abs().max()) == 0.0                                   # no scene: zeros


def test_views_one_after_another_match_all_at_once(s3r):
    """Appending a scene view by view leaves the same cache as all rows at once, and the rows read back feed the sparse path."""
    g = gen(71)
    views, tokens, H, page = 4, 333, 2, 64
    n = views * tokens
    k, v = normal(g, n, H, 64, dtype=BF16), normal(g, n, H, 64, dtype=BF16)
    width = n // page + 1
    pt = table(g, 1, width, width)
    whole, parts = new_cache(s3r, width, H, page), new_cache(s3r, width, H, page)

    def length(m):
        return torch.tensor([m], dtype=torch.int32, device="cuda")
    s3r.speed3r_cache_append(whole, k, v, pt, length(n))
    for i in range(views):
        s = slice(i * tokens, (i + 1) * tokens)
        s3r.speed3r_cache_append(parts, k[s], v[s], pt, length((i + 1) * tokens))
    assert all(torch.equal(a, b) for a, b in zip(whole, parts))
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    s3r.speed3r_cache_read(whole, ko, vo, pt, length(n))
    out, dense = torch.empty_like(k), torch.empty_like(k)
    s3r.speed3r_sparse_global_attn(ko, ko, vo, out, 64, n // 64 + 1)                 # every block: dense, merged half and half
    s3r.speed3r_dense_attn(ko, ko, vo, dense)
    attended = run_attend(s3r, whole, ko, pt, [n], [n], False)["out"]
    crossed = run_cross(s3r, ko, ko, vo)["out"]
    want = cross_reference(ko, ko, vo, [(0, n, 0, n)], None, SCALE)
    for name, got in (("cache", attended), ("cross", crossed), ("dense", dense)):
        check(name, got, want["out"], want["out_tol"])
    assert torch.isfinite(out.float()).all()


def test_gradient_captured_and_replayed(s3r):
    """A training step's calls in a graph, with the inputs changed and the program's own work between replays."""
    g = gen(101)
    q, k, v, d_out = (normal(g, n, 4, 64, dtype=BF16) for n in (200, 900, 900, 200))
    names = ("out", "lse", "dq", "dk", "dv")
    buffers = (torch.empty_like(q), torch.empty((4, 200), device="cuda"), torch.empty_like(q), torch.empty_like(k), torch.empty_like(v))
    ws = torch.empty(max(s3r.speed3r_cross_workspace_bytes(q, k), s3r.speed3r_cross_workspace_bytes(q, k, backward=True)), dtype=torch.uint8, device="cuda")

    def step():
        out, lse, dq, dk, dv = buffers
        s3r.speed3r_cross_attn(q, k, v, out, lse=lse, workspace=ws)
        s3r.speed3r_cross_attn_backward(q, k, v, out, lse, d_out, dq, dk, dv, workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        for t in (q, k, v, d_out):
            t.copy_(normal(g, *t.shape, dtype=BF16))
        want = run_cross(s3r, q, k, v, d_out)
        graph.replay()
        torch.cuda.synchronize()
        for name, t in zip(names, buffers):
            assert torch.equal(t, want[name]), (i, name)


def test_another_stream(s3r):
    g = gen(81)
    q, k, v = (normal(g, n, 2, 64, dtype=BF16) for n in (100, 500, 500))
    want, got = torch.empty_like(q), torch.zeros_like(q)
    s3r.speed3r_cross_attn(q, k, v, want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    s3r.speed3r_cross_attn(q, k, v, got, stream=side)
    side.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("raw", [False, True])
def test_workspace_belongs_to_the_stream_of_the_call(s3r, raw):
    """What a call allocates for itself must not go to the program's own stream while the call's may still be at work."""
    g = gen(82)
    q, k, v = normal(g, 8, 2, 64, dtype=BF16), normal(g, 4000, 2, 64, dtype=BF16), normal(g, 4000, 2, 64, dtype=BF16)
    out, side = torch.empty_like(q), torch.cuda.Stream()
    torch.cuda.synchronize()
    workspace = s3r.speed3r_cross_attn(q, k, v, out, stream=side.cuda_stream if raw else side)
    place, size = workspace.data_ptr(), workspace.numel()
    del workspace
    mine = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(3)]
    assert place not in [t.data_ptr() for t in mine]
    side.synchronize()
    want = torch.empty_like(q)
    s3r.speed3r_cross_attn(q, k, v, want)
    assert torch.equal(out, want)


def test_two_calls_at_once(s3r):
    """Calls of two streams that overlap, each with a workspace that the binding allocates."""
    g = gen(83)
    work = []
    for n, m in ((700, 5000), (3, 20000)):
        q, k, v, d_out = (normal(g, x, 4, 64, dtype=BF16) for x in (n, m, m, n))
        work.append((torch.cuda.Stream(), (q, k, v, d_out), run_cross(s3r, q, k, v, d_out)))
    results = []
    for _ in range(6):
        for stream, (q, k, v, d_out), want in work:
            out, lse, dq, dk, dv = (torch.empty_like(want[x]) for x in ("out", "lse", "dq", "dk", "dv"))
            stream.wait_stream(torch.cuda.current_stream())
            s3r.speed3r_cross_attn(q, k, v, out, lse=lse, stream=stream)
            s3r.speed3r_cross_attn_backward(q, k, v, out, lse, d_out, dq, dk, dv, stream=stream)
            results.append((want, dict(out=out, lse=lse, dq=dq, dk=dk, dv=dv)))
    torch.cuda.synchronize()
    for want, got in results:
        for name in got:
            assert torch.equal(got[name], want[name]), name
