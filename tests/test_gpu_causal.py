"""GPU tests of causal attention of packed sequences and its gradient, against the plain 64-bit form of tests/decoder_util.py (which derives
the bounds; what a row does not see is a mask there)."""
import math

import pytest
import torch

from tests.decoder_util import attention, check

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


def nan_like(t):
    return torch.full(t.shape, math.nan, dtype=t.dtype, device="cuda")


def run(s3r, q, k, v, d_out=None, view=1, **kw):
    r = {"out": nan_like(q), "lse": torch.full((q.shape[1], q.shape[0]), math.nan, device="cuda")}
    s3r.speed3r_causal_attn(q, k, v, r["out"], lse=r["lse"], tokens_per_view=view, **kw)
    if d_out is not None:
        r.update(dq=nan_like(d_out), dk=torch.full(k.shape, math.nan, dtype=q.dtype, device="cuda"),
                 dv=torch.full(k.shape, math.nan, dtype=q.dtype, device="cuda"))
        s3r.speed3r_causal_attn_backward(q, k, v, r["out"], r["lse"], d_out, r["dq"], r["dk"], r["dv"], tokens_per_view=view, **kw)
    torch.cuda.synchronize()
    return r


def what_rows_see(n, m, view):
    token, key = torch.arange(m - n, m, device="cuda"), torch.arange(m, device="cuda")
    return (torch.div(key, view, rounding_mode="floor") <= torch.div(token, view, rounding_mode="floor")[:, None]) & (token >= 0)[:, None]


def reference(q, k, v, spans, view, d_out=None, mask=None, scale=SCALE):
    """spans: (first row, rows, first key, keys).  Rows outside stay NaN."""
    H, KH = q.shape[1], k.shape[1]
    like = {"out": q, "lse": q[:, :, 0].t(), **({} if d_out is None else {"dq": q, "dk": k, "dv": v})}
    r = {}
    for name, t in like.items():
        r[name], r[name + "_tol"] = (torch.full(t.shape, x, dtype=torch.float64, device="cuda") for x in (math.nan, 0.0))
    for q0, n, k0, m in spans:
        seen = what_rows_see(n, m, view)
        if mask is not None:
            seen = seen & (mask[k0:k0 + m] != 0)[None]
        if d_out is not None:
            r["dk"][k0:k0 + m] = r["dv"][k0:k0 + m] = 0.0
        for h in range(H):
            kh = h // (H // KH)
            x = attention(q[q0:q0 + n, h], k[k0:k0 + m, kh], v[k0:k0 + m, kh], seen, scale, q.dtype, None if d_out is None else d_out[q0:q0 + n, h])
            for name in ("out", "out_tol", "dq", "dq_tol"):
                if name in r:
                    r[name][q0:q0 + n, h] = x[name]
            for name in ("lse", "lse_tol"):
                r[name][h, q0:q0 + n] = x[name]
            for name in ("dk", "dk_tol", "dv", "dv_tol"):
                if name in r:
                    r[name][k0:k0 + m, kh] += x[name]
    return r


def compare(got, want):
    for name in got:
        check(name, got[name], want[name], want[name + "_tol"])


def inputs(seed, n, m, heads, kv_heads, dtype):
    g = gen(seed)
    return (normal(g, n, heads, 64, dtype=dtype, scale=2.0), normal(g, m, kv_heads, 64, dtype=dtype), normal(g, m, kv_heads, 64, dtype=dtype),
            normal(g, n, heads, 64, dtype=dtype))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,m,heads,kv_heads", [
    (1, 1, 1, 1), (2, 2, 2, 1), (1, 64, 4, 2), (16, 16, 1, 1), (17, 64, 3, 3), (33, 65, 2, 2), (64, 64, 4, 1), (65, 65, 1, 1), (100, 129, 6, 2),
    (128, 128, 2, 2), (129, 300, 8, 2), (300, 300, 3, 1), (700, 700, 4, 4), (4, 3001, 8, 2), (40, 5000, 2, 2), (200, 4097, 2, 1), (1000, 1000, 12, 2),
    (50, 20, 2, 1), (300, 64, 2, 2), (5, 0, 2, 1), (70, 1, 1, 1)])
def test_causal_by_token(s3r, dtype, n, m, heads, kv_heads):
    q, k, v, d_out = inputs(n * 1000 + m, n, m, heads, kv_heads, dtype)
    compare(run(s3r, q, k, v, d_out), reference(q, k, v, [(0, n, 0, m)], 1, d_out))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,m,view", [(300, 300, 7), (300, 300, 64), (260, 260, 100), (500, 500, 128), (700, 700, 233), (300, 300, 300), (300, 300, 299),
                                      (300, 300, 2 ** 31 - 1), (10, 300, 60), (64, 700, 90), (129, 2000, 1000), (200, 130, 50), (16, 30, 8)])
def test_causal_by_view(s3r, dtype, n, m, view):
    q, k, v, d_out = inputs(n + m + view % 1000, n, m, 4, 2, dtype)
    compare(run(s3r, q, k, v, d_out, view), reference(q, k, v, [(0, n, 0, m)], view, d_out))


BATCHES = {"prompts": ([130, 1, 64, 300, 33, 0, 200], None), "with earlier tokens": ([4, 70, 1, 0, 16, 130], [300, 70, 514, 9, 900, 2000]),
           "single rows": ([1] * 100, [1 + 17 * i % 300 for i in range(100)]), "of few rows": ([1, 2, 3, 4] * 30, [40] * 120),
           "more rows than keys": ([30, 5, 200], [10, 5, 64]), "one long among many": ([1] * 70 + [600] + [1] * 30, None)}


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("view", [1, 50])
@pytest.mark.parametrize("which", list(BATCHES))
def test_packed_sequences_and_masks(s3r, dtype, which, view):
    """Rows before the first and behind the last sequence are left as they were; masked keys and what is outside hold NaN."""
    rows, keys = BATCHES[which]
    keys = keys or rows
    q0, k0 = 3, 5
    n, m = sum(rows) + 7, sum(keys) + 9
    q, k, v, d_out = inputs(len(rows), n, m, 4, 2, dtype)
    a, b = starts(rows, q0), starts(keys, k0)
    spans = [(int(x), r, int(y), c) for x, y, r, c in zip(a, b, rows, keys)]
    for mask in (None, torch.rand(m, generator=gen(9), device="cuda") < 0.6):
        outside = torch.ones(m, dtype=torch.bool, device="cuda")
        outside[k0:k0 + sum(keys)] = False
        bad = outside if mask is None else outside | ~mask
        k[bad], v[bad] = math.nan, math.inf
        status = torch.full((1,), -1, dtype=torch.int32, device="cuda")
        got = run(s3r, q, k, v, d_out, view, q_start=a, kv_start=b, key_mask=mask, status=status)
        assert int(status) == 0
        compare(got, reference(q, k, v, spans, view, d_out, mask))


def lengths(seed, count, lo, hi):
    return torch.randint(lo, hi, (count,), generator=torch.Generator().manual_seed(seed)).tolist()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("view", [1, 90])
@pytest.mark.parametrize("count,lo,hi,earlier,heads,kv_heads", [
    (70, 70, 150, 0, 2, 2),          # more sequences than a wave has lanes, 128 rows and fewer in each
    (64, 1, 300, 0, 3, 1), (65, 40, 200, 300, 2, 1), (5, 300, 1200, 0, 2, 1), (3, 129, 700, 2000, 4, 4), (2, 1, 2, 5000, 8, 1), (40, 0, 400, 100, 1, 1)])
def test_many_rows_of_many_sequences(s3r, dtype, view, count, lo, hi, earlier, heads, kv_heads):
    """Tiles by their lengths over all sequences, in one piece and in several."""
    rows = lengths(count, count, lo, hi)
    keys = [r + x for r, x in zip(rows, lengths(count + 1, count, 0, earlier + 1))]
    q, k, v, d_out = inputs(count + view, sum(rows), sum(keys), heads, kv_heads, dtype)
    a, b = starts(rows), starts(keys)
    spans = [(int(x), r, int(y), c) for x, y, r, c in zip(a, b, rows, keys)]
    compare(run(s3r, q, k, v, d_out, view, q_start=a, kv_start=b), reference(q, k, v, spans, view, d_out))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("seed", range(12))
def test_batches_with_a_long_sequence(s3r, dtype, seed):
    """Batches whose tiles take more pieces than the mean length asks for: all launches of a call find the same number."""
    g = torch.Generator().manual_seed(seed)
    pick = lambda lo, hi: int(torch.randint(lo, hi + 1, (1,), generator=g))
    count, heads = (2, 5, 17, 40, 64, 65)[seed % 6], (1, 2, 4, 8)[pick(0, 3)]
    kv_heads = heads // (1, 2, 4, 8)[pick(0, (1, 2, 4, 8).index(heads))]
    rows = [max(1, int(2 ** (pick(0, 80) / 10))) for _ in range(count)]
    keys = [r + (int(2 ** (pick(0, 90) / 10)) if pick(0, 2) == 0 else 0) for r in rows]
    rows[seed % count], keys[seed % count] = (700, 700) if seed % 3 == 0 else (150, 2500 + 100 * seed)
    q, k, v, d_out = inputs(seed, sum(rows), sum(keys), heads, kv_heads, dtype)
    a, b = starts(rows), starts(keys)
    spans = [(int(x), r, int(y), c) for x, y, r, c in zip(a, b, rows, keys)]
    view = (1, 1, 37)[pick(0, 2)]
    got = run(s3r, q, k, v, d_out, view, q_start=a, kv_start=b)
    compare(got, reference(q, k, v, spans, view, d_out))
    again = run(s3r, q, k, v, d_out, view, q_start=a, kv_start=b)
    assert all(torch.equal(got[name], again[name]) for name in got)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,m,view,heads,kv_heads", [(300, 300, 1, 2, 1), (300, 300, 100, 2, 2), (12, 80, 1, 2, 2), (30, 30, 1, 4, 1), (700, 900, 1, 4, 4)])
def test_what_is_not_seen_may_hold_anything(s3r, dtype, n, m, view, heads, kv_heads):
    """Infinities and NaN in keys and values of later tokens do not reach earlier rows, nor those of earlier rows later keys; who does see them
    has an infinity or NaN in that channel.  The others are within their bounds of the exact results, as without such numbers, but need not
    have the same bits: 32 rows decide together when they look for a larger maximum, and the probabilities, to which it is the unit, are
    rounded to bf16 by up to half a step either way, which the bounds count."""
    q, k, v, d_out = inputs(n + view, n, m, heads, kv_heads, dtype)
    want = reference(q, k, v, [(0, n, 0, m)], view, d_out)
    seen = what_rows_see(n, m, view)
    share = heads // kv_heads

    def within(got, name, *at):
        check(name, got[name][at], want[name][at], want[name + "_tol"][at])

    for at in (m - 1, m - n // 2, m - n + 5):
        row_sees = seen[:, at]
        for what, x in (("v", math.inf), ("v", math.nan), ("k", math.nan), ("k", math.inf)):
            bad_k, bad_v = k.clone(), v.clone()
            (bad_v if what == "v" else bad_k)[at, 0, 3] = x
            got = run(s3r, q, bad_k, bad_v, d_out, view)
            print(what, x, at, flush=True)
            for name in ("out", "dq"):
                within(got, name, ~row_sees)
                within(got, name, slice(None), slice(share, None))
            if what == "v":
                out = got["out"][row_sees][:, :share, 3].float()
                # (of fp32 rows an infinity may come out as NaN, as in speed3r_cross_attn: 0 times it in the products of parts)
                assert (torch.isinf(out) if x == math.inf and dtype == BF16 else ~torch.isfinite(out)).all()
                within(got, "out", slice(None), slice(None), slice(4, None))
            elif math.isnan(x):
                assert torch.isnan(got["out"][row_sees][:, :share].float()).all()
    for row in (0, n // 2, n - 1):
        key_seen = seen[row]
        for what, x in (("q", math.nan), ("d_out", math.nan), ("d_out", math.inf)):
            bad_q, bad_d = q.clone(), d_out.clone()
            (bad_q if what == "q" else bad_d)[row, 0, 3] = x
            got = run(s3r, bad_q, k, v, bad_d, view)
            print(what, x, row, flush=True)
            for name in ("dk", "dv"):
                within(got, name, ~key_seen)
                within(got, name, slice(None), slice(1, None))
            assert not torch.isfinite(got["dv"][key_seen][:, 0, 3].float()).any()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_strides_scale_and_sums_of_shared_heads(s3r, dtype):
    g = gen(3)
    n, m = 150, 260
    q, kv, d_out = normal(g, n, 3, 6, 64, dtype=dtype)[:, 1], normal(g, m, 2, 2, 64, dtype=dtype), normal(g, n, 6, 64, dtype=dtype)
    got = run(s3r, q, kv[:, :, 0], kv[:, :, 1], d_out, 3, softmax_scale=0.3)
    compare(got, reference(q, kv[:, :, 0], kv[:, :, 1], [(0, n, 0, m)], 3, d_out, scale=0.3))
    k, v = (normal(g, 2, m, 64, dtype=dtype).transpose(0, 1) for _ in range(2))
    compare(run(s3r, q, k, v, d_out), reference(q, k, v, [(0, n, 0, m)], 1, d_out))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", ["projection", "head by head", "far heads", "far rows"])
@pytest.mark.parametrize("heads,kv_heads", [(8, 2), (6, 2), (64, 1)])
def test_layouts_of_shared_heads(s3r, dtype, layout, heads, kv_heads):
    """Rows of q anywhere give the bits of packed ones, by token and in cross attention: units of whole rows (64 is a multiple of the heads that
    share one) and others, rows and heads near enough for offsets of 32 bits and not."""
    n, m = 150, 200
    q, k, v, d_out = inputs(heads, n, m, heads, kv_heads, dtype)
    if layout == "projection":
        there = torch.zeros((n, heads + 5, 64), dtype=dtype, device="cuda")[:, 3:3 + heads]
    elif layout == "head by head":
        there = torch.zeros((heads, n, 64), dtype=dtype, device="cuda").transpose(0, 1)
    else:
        far = 2 ** 23 + 64                                       # elements; room for the last row of the last head, no more
        row, head = (64, far) if layout == "far heads" else (far, 64)
        there = torch.zeros((n - 1) * row + (heads - 1) * head + 64, dtype=dtype, device="cuda").as_strided((n, heads, 64), (row, head, 1))
    there.copy_(q)
    got, want = run(s3r, there, k, v, d_out), run(s3r, q, k, v, d_out)
    assert all(torch.equal(got[name], want[name]) for name in want)
    results = []
    for x in (there, q):
        out, lse, dq, dk, dv = torch.empty_like(d_out), torch.empty((heads, n), device="cuda"), torch.empty_like(d_out), torch.empty_like(k), torch.empty_like(v)
        s3r.speed3r_cross_attn(x, k, v, out, lse=lse)
        s3r.speed3r_cross_attn_backward(x, k, v, out, lse, d_out, dq, dk, dv)
        results.append((out, lse, dq, dk, dv))
    assert all(torch.equal(a, b) for a, b in zip(*results))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,m", [(0, 200), (0, 0), (90, 0)])
def test_calls_without_rows_or_keys(s3r, dtype, n, m):
    """Keys that no row sees have gradients of 0."""
    q, k, v, d_out = inputs(n + m, n, m, 4, 2, dtype)
    got = run(s3r, q, k, v, d_out)
    assert not got["dk"].any() and not got["dv"].any() and not got["dq"].any() and not got["out"].any()
    assert (got["lse"] == -math.inf).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_view_of_all_tokens_is_cross_attention(s3r, dtype):
    """And the last token alone sees all."""
    q, k, v, d_out = inputs(5, 200, 200, 4, 2, dtype)
    got = run(s3r, q, k, v, d_out, 200)
    seen = torch.ones((200, 200), dtype=torch.bool, device="cuda")
    assert torch.equal(what_rows_see(200, 200, 200), seen)
    compare(got, reference(q, k, v, [(0, 200, 0, 200)], 200, d_out))
    one, cross = run(s3r, q[-1:], k, v), torch.empty_like(q[-1:])
    s3r.speed3r_cross_attn(q[-1:], k, v, cross)
    assert torch.equal(one["out"], cross)


def test_a_view_longer_than_32_bits_hold(s3r):
    q, k, v, d_out = inputs(6, 200, 200, 4, 2, torch.bfloat16)
    want = run(s3r, q, k, v, d_out, 200)
    for view in (2 ** 31 - 1, 2 ** 32 + 1):
        got = run(s3r, q, k, v, d_out, view)
        assert all(torch.equal(got[name], want[name]) for name in want)


def test_the_cache_gives_the_same(s3r):
    """A prompt over itself by the cache (keys and values that 4 bits hold exactly) and without it, in fp32."""
    g = gen(6)
    n, KH = 300, 2
    steps = torch.tensor([0, 0.5, 1, 1.5, 2, 3, -0.5, -1, -1.5, -2, -3], device="cuda")
    k, v = (steps[torch.randint(0, len(steps), (n, KH, 64), generator=g, device="cuda")].contiguous() for _ in range(2))
    k[..., ::32] = v[..., ::32] = 6.0
    q = normal(g, n, 4, 64)
    cache = s3r.PagedCache.empty(n_pages=10, kv_heads=KH, page=32)
    pages, length = torch.arange(10, dtype=torch.int32, device="cuda")[None], torch.tensor([n], dtype=torch.int32, device="cuda")
    s3r.speed3r_cache_append(cache, k, v, pages, length)
    want, lse = torch.empty_like(q), torch.empty((4, n), device="cuda")
    s3r.speed3r_cache_attn(cache, q, want, pages, length, causal=True, lse=lse)
    got = run(s3r, q, k, v)
    r = reference(q, k, v, [(0, n, 0, n)], 1)
    check("cache", want, r["out"], r["out_tol"])
    compare(got, r)


def test_gradient_against_differences(s3r):
    """fp32: (f(x + t d) - f(x - t d)) / 2 t of f = sum(out * d_out) against the gradient's product with d: t = 2^-4 and directions of
    norm 1 leave 1e-4 by cancellation and 4e-3 by the cubic term."""
    q, k, v, d_out = inputs(11, 57, 90, 4, 2, F32)
    q = q / 2
    r = run(s3r, q, k, v, d_out, 4)

    def f(*x):
        out = torch.empty_like(q)
        s3r.speed3r_causal_attn(*x, out, tokens_per_view=4)
        return float((out.double() * d_out.double()).sum())
    for i, name in enumerate(("dq", "dk", "dv")):
        d = r[name] / r[name].norm()
        t, x = 2.0 ** -4, [q, k, v]
        up, down = list(x), list(x)
        up[i], down[i] = x[i] + t * d, x[i] - t * d
        slope, want = (f(*up) - f(*down)) / (2 * t), float(r[name].double().norm())
        print(name, slope, want, flush=True)
        assert abs(slope - want) <= 5e-3 * want


def test_rows_past_2_31_elements(s3r):
    """Keys whose rows lie further than 2^32 bytes apart, and rows of q that start past 2^31 elements."""
    g = gen(21)
    n, m, H = 150, 400, 2
    stride = (5 << 30) // (2 * m) // 8 * 8
    room = torch.zeros(m * stride, dtype=BF16, device="cuda")
    k, v = (room.as_strided((m, 1, 64), (stride, 64, 1), at) for at in (0, 64))
    q = room.as_strided((n, H, 64), (stride, 64, 1), room.numel() - (n - 1) * stride - 64 * H - 128)
    for t in (k, v, q):
        t.copy_(normal(g, *t.shape, dtype=BF16))
    d_out = normal(g, n, H, 64, dtype=BF16)
    got = {"out": torch.full((n, H, 64), math.nan, dtype=BF16, device="cuda"), "lse": torch.empty((H, n), device="cuda")}
    s3r.speed3r_causal_attn(q, k, v, got["out"], lse=got["lse"])
    got.update(dq=nan_like(d_out), dk=torch.full((m, 1, 64), math.nan, dtype=BF16, device="cuda"), dv=torch.full((m, 1, 64), math.nan, dtype=BF16, device="cuda"))
    s3r.speed3r_causal_attn_backward(q, k, v, got["out"], got["lse"], d_out, got["dq"], got["dk"], got["dv"])
    compare(got, reference(q.contiguous(), k.contiguous(), v.contiguous(), [(0, n, 0, m)], 1, d_out))


def test_keys_that_are_their_own_values(s3r):
    q, k, _, d_out = inputs(22, 300, 300, 2, 2, BF16)
    compare(run(s3r, q, k, k, d_out), reference(q, k, k, [(0, 300, 0, 300)], 1, d_out))


def test_large_scores_and_rising_maxima(s3r):
    g = gen(5)
    for dtype in (BF16, F32):
        q, k, v = normal(g, 500, 2, 64, dtype=dtype), normal(g, 500, 2, 64, dtype=dtype), normal(g, 500, 2, 64, dtype=dtype)
        k = (k.float() * torch.linspace(0, 30, 500, device="cuda")[:, None, None]).to(dtype)
        d_out = normal(g, 500, 2, 64, dtype=dtype)
        compare(run(s3r, q, k, v, d_out), reference(q, k, v, [(0, 500, 0, 500)], 1, d_out))


def test_long_sequences_in_pieces(s3r):
    """Few and many rows over keys that are divided; bf16 against fp32 rows of the reference at both ends and in the middle."""
    for n, m, heads in ((3, 70000, 2), (300, 40000, 2), (9000, 9000, 1)):
        q, k, v, d_out = inputs(n, n, m, heads, 1, BF16)
        got = run(s3r, q, k, v, d_out)
        for h in range(heads):
            for r0 in (0, n // 2, max(0, n - 100)):
                rows = slice(r0, min(n, r0 + 100))
                seen = what_rows_see(n, m, 1)[rows]
                x = attention(q[rows, h], k[:, 0], v[:, 0], seen, SCALE, BF16, d_out[rows, h])
                for name in ("out", "dq"):
                    check(name, got[name][rows, h], x[name], x[name + "_tol"])
                check("lse", got["lse"][h, rows], x["lse"], x["lse_tol"])
        want = reference(q, k, v, [(0, n, 0, m)], 1, d_out)
        for name in ("dk", "dv"):
            check(name, got[name], want[name], want[name + "_tol"])


def test_broken_starts_are_reported_and_stay_in_range(s3r):
    q, k, v, d_out = inputs(8, 50, 80, 1, 1, BF16)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for view in (1, 30):
        for qs, ks in (([0, 60, 50], [0, 40, 80]), ([0, 20, 50], [0, 90, 80]), ([-3, 20, 50], [0, 40, 80]), ([0, 20, 50], [50, 40, 80])):
            kw = {"q_start": torch.tensor(qs, dtype=torch.int32, device="cuda"), "kv_start": torch.tensor(ks, dtype=torch.int32, device="cuda")}
            run(s3r, q, k, v, d_out, view, status=status, **kw)
            assert int(status) == s3r.S3R_DIAG_SPANS


def test_calls_repeat_overlap_and_replay(s3r):
    """The same bits on every call, on two streams at once, and from a graph replayed with other contents between eager calls."""
    rows = [700, 300, 24]
    q, k, v, d_out = inputs(12, 1024, 1024, 4, 2, BF16)
    a = starts(rows)
    want = run(s3r, q, k, v, d_out, q_start=a, kv_start=a)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        got = []
        for s in streams:
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                got.append(run(s3r, q, k, v, d_out, q_start=a, kv_start=a))
        torch.cuda.synchronize()
        assert all(torch.equal(r[n], want[n]) for r in got for n in want)
    out = {n: torch.zeros_like(t) for n, t in want.items()}

    def step():
        s3r.speed3r_causal_attn(q, k, v, out["out"], lse=out["lse"], q_start=a, kv_start=a)
        s3r.speed3r_causal_attn_backward(q, k, v, out["out"], out["lse"], d_out, out["dq"], out["dk"], out["dv"], q_start=a, kv_start=a)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(4):
        g = gen(50 + turn)
        for t in (q, k, v, d_out):
            t.copy_(normal(g, *t.shape, dtype=BF16))
        a.copy_(starts([[700, 300, 24], [1024, 0, 0], [1, 1, 1022], [0, 500, 524]][turn]))
        for t in out.values():
            t.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        want = run(s3r, q, k, v, d_out, q_start=a, kv_start=a)
        assert all(torch.equal(out[n], want[n]) for n in want), turn


def test_a_block_by_these_calls(s3r):
    """Norm, projection, rotation, causal attention, projection, residual: a block's forward pass and its gradient with these calls in turn,
    against autograd in 64 bits.  Everything is fp32: errors of 2^-24 through a dozen operations of conditions below a hundred, 1e-4 of each gradient's
    norm leaves ten times that."""
    g = gen(13)
    lengths, C, H = [90, 60], 256, 4
    n, a = sum(lengths), starts(lengths)
    x, weight, bias = normal(g, n, C), normal(g, C) * 0.1 + 1, normal(g, C) * 0.1
    wqkv, wo, scale, gate = normal(g, C, 3 * C) / 16, normal(g, C, C) / 16, normal(g, C), normal(g, 2, C)
    qw, kw = normal(g, 64) * 0.1 + 1, normal(g, 64) * 0.1 + 1
    angle = torch.rand((40, 32), generator=g, device="cuda").double() * 6
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    at = torch.randint(0, 40, (n, 2), generator=g, device="cuda").int()
    d_r, d_y = normal(g, n, C), normal(g, n, C)
    rot = dict(axis_pairs=(16, 16), norm="rms", q_weight=qw, k_weight=kw)
    res = dict(norm="layer", weight=weight, scale=scale, gate=gate, row_start=a)

    y0 = torch.empty_like(x)
    s3r.speed3r_residual_norm(x, y0, norm="layer", weight=weight, bias=bias)
    qkv = (y0 @ wqkv).view(n, 3, H, 64)
    q, k, o = (torch.empty((n, H, 64), device="cuda") for _ in range(3))
    lse = torch.empty((H, n), device="cuda")
    s3r.speed3r_rotary(qkv[:, 0], qkv[:, 1], q, k, cos, sin, at, **rot)
    v = qkv[:, 2].contiguous()
    s3r.speed3r_causal_attn(q, k, v, o, lse=lse, q_start=a, kv_start=a)
    f = o.view(n, C) @ wo
    r, y = torch.empty_like(x), torch.empty_like(x)
    s3r.speed3r_residual_norm(x, y, f=f, r=r, bias=bias, **res)

    grads = {name: torch.empty_like(t) for name, t in (("d_weight", weight), ("d_bias", bias), ("d_scale", scale), ("d_gate", gate))}
    dx, df = torch.empty_like(x), torch.empty_like(x)
    s3r.speed3r_residual_norm_backward(x, d_y, dx, f=f, d_r=d_r, df=df, **grads, **res)
    d_o = (df @ wo.t()).view(n, H, 64).contiguous()
    dq, dk, dqkv = torch.empty_like(q), torch.empty_like(k), torch.empty((n, 3, H, 64), device="cuda")
    dv = torch.empty_like(v)
    s3r.speed3r_causal_attn_backward(q, k, v, o, lse, d_o, dq, dk, dv, q_start=a, kv_start=a)
    dqw, dkw = torch.empty_like(qw), torch.empty_like(kw)
    s3r.speed3r_rotary_backward(qkv[:, 0], qkv[:, 1], dq, dk, dqkv[:, 0], dqkv[:, 1], cos, sin, at, dq_weight=dqw, dk_weight=dkw, **rot)
    dqkv[:, 2] = dv
    d_y0, d_x0 = dqkv.view(n, 3 * C) @ wqkv.t(), torch.empty_like(x)
    d_w0, d_b0 = torch.empty_like(weight), torch.empty_like(bias)
    s3r.speed3r_residual_norm_backward(x, d_y0, d_x0, norm="layer", weight=weight, d_weight=d_w0, d_bias=d_b0)
    got = {"x": dx + d_x0, "weight": grads["d_weight"] + d_w0, "bias": grads["d_bias"] + d_b0, "scale": grads["d_scale"], "gate": grads["d_gate"],
           "wqkv": y0.t() @ dqkv.view(n, 3 * C), "wo": o.view(n, C).t() @ df, "qw": dqw, "kw": dkw}

    t = {name: x.double().requires_grad_() for name, x in dict(x=x, weight=weight, bias=bias, scale=scale, gate=gate, wqkv=wqkv, wo=wo, qw=qw, kw=kw).items()}

    def layer(z):
        d = z - z.mean(-1, keepdim=True)
        return d / torch.sqrt((d * d).mean(-1, keepdim=True) + 1e-6) * t["weight"] + t["bias"]

    def head(z, w):
        z = z / torch.sqrt((z * z).mean(-1, keepdim=True) + 1e-6) * w
        parts = []
        for axis in range(2):
            c, s = (tab.double()[at[:, axis].long(), 16 * axis:16 * axis + 16][:, None] for tab in (cos, sin))
            lo, hi = z[..., 32 * axis:32 * axis + 16], z[..., 32 * axis + 16:32 * axis + 32]
            parts += [lo * c - hi * s, hi * c + lo * s]
        return torch.cat(parts, -1)

    p = (layer(t["x"]) @ t["wqkv"]).view(n, 3, H, 64)
    qq, kk, outs, b0 = head(p[:, 0], t["qw"]), head(p[:, 1], t["kw"]), [], 0
    for m in lengths:
        rows = slice(b0, b0 + m)
        s = torch.stack([qq[rows, i] @ kk[rows, i].t() for i in range(H)]) * SCALE
        s = torch.softmax(s.masked_fill(~what_rows_see(m, m, 1), -math.inf), -1)
        outs.append(torch.stack([s[i] @ p[rows, 2, i] for i in range(H)], 1))
        b0 += m
    u = torch.cat(outs).reshape(n, C) @ t["wo"] * t["scale"] * torch.cat([t["gate"][i].expand(m, C) for i, m in enumerate(lengths)])
    rr = t["x"] + u
    yy = layer(rr)
    want = dict(zip(t, torch.autograd.grad((rr, yy), list(t.values()), (d_r.double(), d_y.double()))))
    for name, a_, b_ in [("r", r, rr), ("y", y, yy)] + [(name, got[name], want[name]) for name in t]:
        off = float((a_.double() - b_.detach()).norm() / b_.detach().norm())
        print(name, off, flush=True)
        assert off <= 1e-4, name
