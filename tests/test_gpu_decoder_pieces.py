"""GPU tests that every piece of a long sequence counts, once: inputs of tests/pieces_util.py, from keys of one workgroup to 256 pieces."""
import pytest
import torch

from tests.decoder_util import attention, check
from tests.pieces_util import UNIT, plant, planted_reference
from tests.test_gpu_decoder import BF16, F32, SCALE, cached, gen, normal, run_attend, run_cross, s3r, starts, table  # noqa: F401 (s3r: the fixture)

pytestmark = pytest.mark.gpu


def pieces_of(need, rows, heads):
    """Pieces by the workspace: partial results of 64 channels and a log-sum of every row of a head for each (padded to 256 bytes)."""
    return max(1, need // (rows * heads * 65 * 4))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,m,heads,kv_heads", [
    (1, 10992, 2, 2), (16, 10992, 1, 1), (3, 10993, 4, 1), (40, 3000, 2, 2), (100, 10992, 4, 2), (1374, 5000, 1, 1), (300, 27480, 1, 1),
    (1, 400_001, 1, 1), (20, 400_001, 1, 1), (100, 400_001, 1, 1),
])
def test_every_piece_of_the_keys_counts(s3r, dtype, n, m, heads, kv_heads):  # noqa: F811
    g = gen(n + m)
    q, k, v = (normal(g, r, h, 64, dtype=dtype) for r, h in ((n, heads), (m, kv_heads), (m, kv_heads)))
    plant(q, k, v, heads // kv_heads)
    got = run_cross(s3r, q, k, v)
    pieces = pieces_of(s3r.speed3r_cross_workspace_bytes(q, k), n, heads)
    for h in range(heads):
        kv = h // (heads // kv_heads)
        want = planted_reference(q[:, h], k[:, kv], v[:, kv], SCALE, dtype, pieces)
        for name, x in (("out", got["out"][:, h]), ("lse", got["lse"][h])):
            check(name, x, want[name], want[name + "_tol"])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,m,heads,kv_heads,page", [
    (1, 3000, 4, 2, 16), (1, 137_400, 2, 2, 64), (20, 20_001, 2, 1, 32), (100, 10_992, 2, 2, 128), (1374, 5000, 1, 1, 64), (300, 41_220, 1, 1, 16),
    (1, 1_500_001, 1, 1, 128), (20, 1_500_001, 1, 1, 64), (100, 1_500_001, 1, 1, 128),
])
def test_every_piece_of_the_cache_counts(s3r, dtype, n, m, heads, kv_heads, page):  # noqa: F811
    g = gen(n + m + page)
    q, k, v = (normal(g, r, h, 64, dtype=BF16) for r, h in ((n, heads), (m, kv_heads), (m, kv_heads)))
    plant(q, k, v, heads // kv_heads)
    width = (m + page - 1) // page
    cache, pt = s3r.PagedCache.empty(width, kv_heads, page), torch.randperm(width, generator=g, device="cuda").int()[None].contiguous()
    s3r.speed3r_cache_append(cache, k, v, pt, torch.tensor([m], dtype=torch.int32, device="cuda"))
    q = q.to(dtype)
    need = s3r.speed3r_cache_workspace_bytes(cache, n, heads, s3r.S3R_BF16 if dtype == BF16 else s3r.S3R_F32, 1, width)
    got = run_attend(s3r, cache, q, pt, [m], [n], False)
    for h in range(heads):
        kc, vc = cached(cache, pt, 0, m, h // (heads // kv_heads))
        # (the workspace is that of causal rows or others, whichever is more: they may have half as many pieces)
        want = planted_reference(q[:, h], kc, vc, SCALE, dtype, max(1, pieces_of(need, n, heads) // 2))
        for name, x in (("out", got["out"][:, h]), ("lse", got["lse"][h])):
            check(name, x, want[name], want[name + "_tol"])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,m,heads,kv_heads", [(2, 10992, 2, 2), (300, 9000, 2, 1), (9000, 200, 1, 1), (4000, 700, 4, 2)])
def test_every_piece_of_a_gradient_counts(s3r, dtype, n, m, heads, kv_heads):  # noqa: F811
    """One key of every unit of 64 has a channel of its own in k, and the others 0, so that a channel of dq is a sum over some units; one row
    of every 64 (of the heads that share a head of keys) has one in q and d_out, and the others 0, so that one of dk and dv is."""
    g = gen(n + m)
    share = heads // kv_heads
    q, k, d_out = (torch.zeros((r, h, 64), device="cuda") for r, h in ((n, heads), (m, kv_heads), (n, heads)))
    rows, keys = torch.arange(0, n, max(1, UNIT // share), device="cuda"), torch.arange(0, m, UNIT, device="cuda")
    for h in range(heads):
        q[rows, h, torch.arange(len(rows), device="cuda") % 64] = 2.0
        d_out[rows, h, (torch.arange(len(rows), device="cuda") + 7 * h) % 64] = 2.0
    for h in range(kv_heads):
        k[keys, h, (torch.arange(len(keys), device="cuda") + 3 * h) % 64] = 1.0
    q, k, v, d_out = q.to(dtype), k.to(dtype), normal(g, m, kv_heads, 64, dtype=dtype), d_out.to(dtype)
    got = run_cross(s3r, q, k, v, d_out)
    seen = torch.ones((1, m), dtype=torch.bool, device="cuda")
    for kv in range(kv_heads):
        sums = {"dk": 0.0, "dv": 0.0, "dk_tol": 0.0, "dv_tol": 0.0}
        for h in range(kv * share, (kv + 1) * share):
            want = attention(q[:, h], k[:, kv], v[:, kv], seen, SCALE, dtype, d_out[:, h])
            check("dq", got["dq"][:, h], want["dq"], want["dq_tol"])
            for name in sums:
                sums[name] = sums[name] + want[name]
        for name in ("dk", "dv"):
            check(name, got[name][:, kv], sums[name], sums[name + "_tol"])


RAGGED = {"few rows": ([3, 1, 2, 5], [9000, 65, 1, 30_000]), "many rows": ([300, 40, 1, 129], [9000, 700, 20_000, 64]),
          "single rows, one long": ([1] * 20, [500] * 19 + [40_000])}


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("which", list(RAGGED))
def test_every_piece_of_ragged_keys_counts(s3r, dtype, which):  # noqa: F811
    rows, keys = RAGGED[which]
    g = gen(len(rows))
    q, k, v = (normal(g, r, h, 64, dtype=dtype) for r, h in ((sum(rows), 4), (sum(keys), 2), (sum(keys), 2)))
    at = [(sum(rows[:b]), n, sum(keys[:b]), m) for b, (n, m) in enumerate(zip(rows, keys))]
    for q0, n, k0, m in at:
        plant(q[q0:q0 + n], k[k0:k0 + m], v[k0:k0 + m], 2)
    got = run_cross(s3r, q, k, v, q_start=starts(rows), kv_start=starts(keys))
    for q0, n, k0, m in at:
        for h in range(4):
            want = planted_reference(q[q0:q0 + n, h], k[k0:k0 + m, h // 2], v[k0:k0 + m, h // 2], SCALE, dtype, 1)
            for name, x in (("out", got["out"][q0:q0 + n, h]), ("lse", got["lse"][h, q0:q0 + n])):
                check(name, x, want[name], want[name + "_tol"])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("which", list(RAGGED))
@pytest.mark.parametrize("page", [16, 128])
def test_every_piece_of_a_ragged_cache_counts(s3r, dtype, causal, which, page):  # noqa: F811
    rows, keys = RAGGED[which]
    keys = [max(n, m) for n, m in zip(rows, keys)]
    g = gen(len(rows) + page)
    q, k, v = (normal(g, r, h, 64, dtype=BF16) for r, h in ((sum(rows), 4), (sum(keys), 2), (sum(keys), 2)))
    at = [(sum(rows[:b]), n, sum(keys[:b]), m) for b, (n, m) in enumerate(zip(rows, keys))]
    for q0, n, k0, m in at:
        plant(q[q0:q0 + n], k[k0:k0 + m], v[k0:k0 + m], 2)
    width = max((m + page - 1) // page for m in keys)
    cache, pt = s3r.PagedCache.empty(width * len(keys), 2, page), table(g, len(keys), width, width * len(keys))
    s3r.speed3r_cache_append(cache, k, v, pt, torch.tensor(keys, dtype=torch.int32, device="cuda"), starts(keys))
    q = q.to(dtype)
    got = run_attend(s3r, cache, q, pt, keys, rows, causal)
    for b, (q0, n, k0, m) in enumerate(at):
        last = torch.arange(m - n, m, device="cuda") if causal else torch.full((n,), m - 1, device="cuda")
        seen = torch.arange(m, device="cuda")[None] <= last[:, None]
        for h in range(4):
            kc, vc = cached(cache, pt, b, m, h // 2)
            want = planted_reference(q[q0:q0 + n, h], kc, vc, SCALE, dtype, 1, seen=seen)
            for name, x in (("out", got["out"][q0:q0 + n, h]), ("lse", got["lse"][h, q0:q0 + n])):
                check(name, x, want[name], want[name + "_tol"])
