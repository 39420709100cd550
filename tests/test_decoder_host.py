"""Host-only checks of cross attention and the 4-bit cache: the structures of the header and of the binding agree, refusals come before any
device work with the documented status, and the 64-bit forms that the GPU tests compare with are right themselves."""
import ctypes
import math
import os
import re
import shutil
import subprocess

import pytest
import torch

from tests.decoder_util import attention, four_bits, packed, rotated, values

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "speed3r.h")
P = 0x10000     # an aligned address that is never dereferenced


@pytest.fixture(scope="module")
def s3r():
    from paper_2603_08055_amd import speed3r
    if not os.path.exists(speed3r.LIB_PATH):
        from paper_2603_08055_amd import build
        build.build_library()
    speed3r.load()
    return speed3r


@pytest.mark.parametrize("name", ["s3r_cross_params", "s3r_cache_params"])
def test_structures_match_the_header(s3r, name, tmp_path):
    cls = getattr(s3r, name)
    body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (name, name), open(HEADER).read(), flags=re.S).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    fields = [re.findall(r"[A-Za-z_][A-Za-z0-9_]*", n)[-1] for decl in body.split(";") if decl.strip() for n in decl.split(",")]
    assert fields == [f[0] for f in cls._fields_]
    if shutil.which("gcc") is None:
        pytest.skip("no gcc")
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "speed3r.h"\nint main(void) {\n  printf("%zu\\n", sizeof(' + name + '));\n'
                   + "".join(f'  printf("%zu\\n", offsetof({name}, {f}));\n' for f in fields) + "  return 0; }\n")
    exe = str(tmp_path / "layout")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), str(src), "-o", exe], check=True,
                   capture_output=True, text=True)
    got = [int(x) for x in subprocess.run([exe], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [ctypes.sizeof(cls)] + [getattr(cls, f).offset for f in fields]


def cross(s3r, **change):
    p = s3r.s3r_cross_params()
    for f in ("q", "k", "v"):
        setattr(p, f, P)
    p.out, p.lse, p.d_out, p.dq, p.dk, p.dv = 0x20000, 0x30000, 0x40000, 0x50000, 0x60000, 0x70000
    p.n_q, p.n_kv, p.batch, p.heads, p.kv_heads, p.head_dim, p.dtype = 10, 20, 1, 4, 2, 64, s3r.S3R_BF16
    for f, x in change.items():
        setattr(p, f, x)
    return p


INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3


@pytest.mark.parametrize("change,status,word", [
    (dict(head_dim=128), UNSUPPORTED, "head_dim"), (dict(dtype=2), UNSUPPORTED, "dtype"), (dict(heads=3), INVALID, "multiple"),
    (dict(heads=0), INVALID, "heads"), (dict(kv_heads=0), INVALID, "kv_heads"), (dict(n_q=-1), INVALID, "n_q"),
    (dict(n_kv=-1), INVALID, "n_kv"), (dict(batch=2), INVALID, "batch"), (dict(batch=-1), INVALID, "batch"),
    (dict(q_start=P), INVALID, "together"), (dict(q_start=P, kv_start=P, batch=0), INVALID, "batch"),
    (dict(q_start=P, kv_start=P, batch=65537), UNSUPPORTED, "65536"), (dict(q_start=P, kv_start=P, batch=32769, heads=16, kv_heads=16), UNSUPPORTED, "2^19"),
    (dict(n_q=1 << 27), UNSUPPORTED, "2^28"), (dict(n_kv=1 << 40), UNSUPPORTED, "2^28"), (dict(heads=1 << 17, kv_heads=1), UNSUPPORTED, "heads"),
    (dict(q=None), INVALID, "null"), (dict(out=None), INVALID, "null"), (dict(k=None), INVALID, "null"), (dict(v=None), INVALID, "null"),
    (dict(q=P + 2), INVALID, "aligned"), (dict(out=0x20008), INVALID, "aligned"), (dict(lse=0x30002), INVALID, "aligned"),
    (dict(out=P), INVALID, "alias"), (dict(q_stride_tok=-8), INVALID, "stride"), (dict(kv_stride_head=4), INVALID, "stride"),
])
def test_cross_refusals(s3r, change, status, word):
    p = cross(s3r, **change)
    for fn in (s3r.load().speed3r_cross_attn, s3r.load().speed3r_cross_attn_backward):
        assert fn(ctypes.byref(p)) == status and word in s3r.speed3r_last_error()


@pytest.mark.parametrize("change,status,word", [
    (dict(lse=None), INVALID, "null"), (dict(d_out=None), INVALID, "null"), (dict(dq=None), INVALID, "null"), (dict(dk=None), INVALID, "null"),
    (dict(dv=None), INVALID, "null"), (dict(dq=0x50004), INVALID, "aligned"), (dict(dk=P), INVALID, "alias"), (dict(dq=0x40000), INVALID, "alias"),
    (dict(dv=0x60000), INVALID, "alias"), (dict(), WORKSPACE, "workspace"), (dict(workspace=0x80010, workspace_bytes=1 << 30), INVALID, "256"),
])
def test_cross_backward_refusals(s3r, change, status, word):
    p = cross(s3r, **change)
    assert s3r.load().speed3r_cross_attn_backward(ctypes.byref(p)) == status and word in s3r.speed3r_last_error()


def test_null_parameters(s3r):
    lib = s3r.load()
    for fn in (lib.speed3r_cross_attn, lib.speed3r_cross_attn_backward, lib.speed3r_cache_append, lib.speed3r_cache_read, lib.speed3r_cache_attn):
        assert fn(None) == INVALID and "null" in s3r.speed3r_last_error()
    assert lib.speed3r_cross_workspace_bytes(None, 0) == lib.speed3r_cache_workspace_bytes(None) == 2 ** 64 - 1


def cache(s3r, **change):
    p = s3r.s3r_cache_params()
    p.k_codes, p.v_codes, p.k_scales, p.v_scales, p.page_table, p.kv_len = (P * (i + 1) for i in range(6))
    p.q, p.k, p.v, p.out = 0x100000, 0x200000, 0x300000, 0x400000
    p.n_pages, p.n_rows, p.page, p.max_pages, p.batch, p.heads, p.kv_heads, p.head_dim, p.dtype = 8, 4, 16, 4, 1, 4, 2, 64, s3r.S3R_BF16
    p.cos, p.sin, p.n_positions, p.rot_axes = 0x500000, 0x600000, 100, 1
    for f, x in change.items():
        setattr(p, f, x)
    return p


@pytest.mark.parametrize("change,status,word", [
    (dict(head_dim=32), UNSUPPORTED, "head_dim"), (dict(dtype=-1), UNSUPPORTED, "dtype"), (dict(heads=5), INVALID, "multiple"),
    (dict(page=48), UNSUPPORTED, "page"), (dict(page=256), UNSUPPORTED, "page"), (dict(n_pages=0), INVALID, "n_pages"),
    (dict(max_pages=0), INVALID, "max_pages"), (dict(batch=0), INVALID, "batch"), (dict(batch=2), INVALID, "row_start"),
    (dict(n_rows=-1), INVALID, "n_rows"), (dict(max_pages=1 << 27), UNSUPPORTED, "max_pages"), (dict(n_rows=1 << 30), UNSUPPORTED, "2^28"),
    (dict(n_pages=1 << 31), UNSUPPORTED, "n_pages"), (dict(k_codes=None), INVALID, "null"), (dict(v_scales=None), INVALID, "null"),
    (dict(page_table=None), INVALID, "null"), (dict(kv_len=None), INVALID, "null"), (dict(v_codes=P + 8), INVALID, "aligned"),
    (dict(k_scales=P + 1), INVALID, "aligned"), (dict(out=0x400008), INVALID, "aligned"), (dict(kv_stride_tok=12), INVALID, "stride"),
    (dict(q_stride_head=-8), INVALID, "stride"), (dict(row_start=P, batch=65537), UNSUPPORTED, "65536"),
    (dict(row_start=P, batch=32769, heads=16, kv_heads=16), UNSUPPORTED, "2^19"),
])
def test_cache_refusals(s3r, change, status, word):
    p, lib = cache(s3r, **change), s3r.load()
    for fn in (lib.speed3r_cache_append, lib.speed3r_cache_read, lib.speed3r_cache_attn):
        assert fn(ctypes.byref(p)) == status and word in s3r.speed3r_last_error()


@pytest.mark.parametrize("fn,change,status,word", [
    ("append", dict(k=None), INVALID, "null"), ("append", dict(cos=None), INVALID, "together"), ("append", dict(out=None), INVALID, "together"),
    ("append", dict(cos=None, sin=None), INVALID, "rotated"), ("append", dict(rot_axes=3), INVALID, "rot_axes"),
    ("append", dict(rot_axes=2), INVALID, "positions"), ("append", dict(rot_neighbours=2), INVALID, "rot_neighbours"),
    ("append", dict(v_codes=P), INVALID, "share"), ("append", dict(v_scales=P * 3), INVALID, "share"),
    ("append", dict(n_positions=0), INVALID, "n_positions"), ("append", dict(out=0x100000), INVALID, "alias"),
    ("read", dict(v=None), INVALID, "null"), ("read", dict(v=0x200000), INVALID, "apart"),
    ("attn", dict(q=None), INVALID, "null"), ("attn", dict(out=0x100000), INVALID, "alias"), ("attn", dict(causal=2), INVALID, "causal"),
    ("attn", dict(max_pages=1000), WORKSPACE, "workspace"), ("attn", dict(max_pages=1000, workspace=P + 16, workspace_bytes=1 << 40), INVALID, "256"),
])
def test_cache_refusals_of_one_call(s3r, fn, change, status, word):
    p = cache(s3r, **change)
    assert getattr(s3r.load(), "speed3r_cache_" + fn)(ctypes.byref(p)) == status and word in s3r.speed3r_last_error()


@pytest.mark.parametrize("where", ["q", "k", "v"])
def test_rotated_queries_do_not_go_where_an_input_is(s3r, where):
    """Waves that have a row's keys or values may still be about to read what another, with its queries, would write over."""
    p = cache(s3r, heads=2, kv_heads=2)                                       # rows of q, k and v alike, so that the shapes fit
    p.out = getattr(p, where)
    assert s3r.load().speed3r_cache_append(ctypes.byref(p)) == INVALID and "alias" in s3r.speed3r_last_error()


def test_workspaces(s3r):
    q, kv = torch.empty((1, 16, 64), dtype=torch.bfloat16, device="meta"), torch.empty((100000, 16, 64), dtype=torch.bfloat16, device="meta")
    assert s3r.speed3r_cross_workspace_bytes(q, kv) > 0                               # one row over many keys: split along them
    assert s3r.speed3r_cross_workspace_bytes(kv, kv) == 0
    assert s3r.speed3r_cross_workspace_bytes(kv, kv, backward=True) == 100000 * 16 * 8
    assert s3r.speed3r_cross_workspace_bytes(q[:0], kv) == 0
    with pytest.raises(s3r.Speed3rError):
        s3r.speed3r_cross_workspace_bytes(q, kv[:, :3])
    c = s3r.PagedCache.empty(10, 4, 16, device="meta")
    assert s3r.speed3r_cache_workspace_bytes(c, 1, 16, s3r.S3R_BF16, 1, 10000) > s3r.speed3r_cache_workspace_bytes(c, 1, 16, s3r.S3R_BF16, 1, 4) == 0
    with pytest.raises(s3r.Speed3rError):
        s3r.speed3r_cache_workspace_bytes(c, 1, 6, s3r.S3R_BF16, 1, 4)


@pytest.mark.parametrize("rows", [0, 1, 40, 100, 1374, 8192])
@pytest.mark.parametrize("batch", [1, 3])
@pytest.mark.parametrize("dtype", [0, 1])
def test_cache_workspace_serves_causal_rows_and_others(s3r, rows, batch, dtype):
    need = []
    for causal in (0, 1):
        p = cache(s3r, n_rows=rows, batch=batch, row_start=P, max_pages=700, page=64, causal=causal, dtype=dtype)
        need.append(s3r.load().speed3r_cache_workspace_bytes(ctypes.byref(p)))
        if need[-1] and rows:
            p.workspace, p.workspace_bytes = 0x1000000 + 16, need[-1]      # refused for its alignment, and not for its size
            assert s3r.load().speed3r_cache_attn(ctypes.byref(p)) == INVALID and "256" in s3r.speed3r_last_error()
    assert need[0] == need[1] < 1 << 40


@pytest.mark.parametrize("rows", [1, 16, 200])
@pytest.mark.parametrize("dtype", [0, 1])
def test_pieces_of_very_long_sequences_are_as_many_as_can_be_joined(s3r, rows, dtype):
    most = 256 * rows * 65 * 4 + 2 * 256                                     # partial results and log-sums of 256 pieces
    for heads in (1, 2, 3, 7):
        for pages in (10_000, 100_000, 1_000_000, 16_000_000):
            p = cache(s3r, n_rows=rows, max_pages=pages, page=128, n_pages=1 << 20, heads=heads, kv_heads=heads, dtype=dtype)
            assert 0 < s3r.load().speed3r_cache_workspace_bytes(ctypes.byref(p)) <= most * heads
        for keys in (1_000_000, 30_000_000):
            p = cross(s3r, n_q=rows, n_kv=keys, heads=heads, kv_heads=heads, batch=1, dtype=dtype)
            assert 0 < s3r.load().speed3r_cross_workspace_bytes(ctypes.byref(p), 0) <= most * heads


@pytest.mark.parametrize("n_q,n_kv", [(0, 0), (0, 5000), (5000, 0), (1, 1), (1 << 20, 1 << 20)])
@pytest.mark.parametrize("batch", [1, 7])
@pytest.mark.parametrize("dtype", [0, 1])
def test_cross_workspace_of_any_size(s3r, n_q, n_kv, batch, dtype):
    p = cross(s3r, n_q=n_q, n_kv=n_kv, batch=batch, q_start=P, kv_start=P, dtype=dtype)
    for backward in (0, 1):
        assert s3r.load().speed3r_cross_workspace_bytes(ctypes.byref(p), backward) < 1 << 40


def test_binding_refuses_what_it_can_see(s3r):
    q, kv = torch.zeros((4, 2, 64), dtype=torch.bfloat16), torch.zeros((8, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(TypeError, match="GPU"):
        s3r.speed3r_cross_attn(q, kv, kv, q.clone(), stream=0)
    c, lists = s3r.PagedCache.empty(4, 2, 16, device="cpu"), torch.zeros((1, 4), dtype=torch.int32)
    with pytest.raises(TypeError, match="GPU"):
        s3r.speed3r_cache_attn(c, q, q.clone(), lists, lists[0, :1], stream=0)
    m = torch.zeros((4, 2, 64), dtype=torch.bfloat16)                  # on the CPU: index -1, for the checks that need no GPU
    with pytest.raises(TypeError, match="contiguous"):
        s3r._rows_arg(m.transpose(1, 2), "q", -1, m.dtype, (4, 64, 2))
    with pytest.raises(TypeError, match="broadcast"):
        s3r._rows_arg(m[:1].expand(4, 2, 64), "q", -1, m.dtype, (4, 2, 64))
    with pytest.raises(TypeError, match="share"):
        s3r._kv_arg(m, torch.zeros((4, 4, 64), dtype=m.dtype)[:, ::2], -1, m.dtype, (4, 2, 64))
    with pytest.raises(TypeError, match="GPU 0"):
        s3r._rows_arg(m, "q", 0, m.dtype, (4, 2, 64))
    with pytest.raises(ValueError, match="shape"):
        s3r._arg(m, "out", -1, m.dtype, (4, 3, 64))
    with pytest.raises(TypeError, match="dtype"):
        s3r._arg(m, "out", -1, torch.float32, (4, 2, 64))
    with pytest.raises(TypeError, match="contiguous"):
        s3r._arg(m[:, :1], "out", -1, m.dtype, (4, 1, 64))
    assert s3r._rows_arg(m, "q", -1, m.dtype, (4, 2, 64))[1:] == (128, 64)
    assert s3r._rows_arg(m[:, 1:], "q", -1, m.dtype, (4, 1, 64))[1:] == (128, 64)
    assert s3r._arg(None, "lse", -1, torch.float32, (1,)) is None


# ---- the 64-bit forms themselves ------------------------------------------------------------------------

def test_reference_gradients_are_those_of_autograd():
    g = torch.Generator().manual_seed(1)
    q, k, v, d = (torch.randn((n, 64), generator=g, dtype=torch.float64) for n in (7, 12, 12, 7))
    seen = torch.rand((7, 12), generator=g) < 0.6
    seen[3] = False
    x = [t.clone().requires_grad_() for t in (q, k, v)]
    s = (x[0] @ x[1].t() * 0.125).masked_fill(~seen, -math.inf)
    p = torch.where(seen, torch.softmax(torch.where(seen.any(1, keepdim=True), s, 0.0), 1), 0.0)
    out = p @ x[2]
    out.backward(d)
    r = attention(q, k, v, seen, 0.125, torch.float32, d)
    assert torch.allclose(r["out"], out.detach(), atol=1e-13) and float(r["out"][3].abs().max()) == 0 and r["lse"][3] == -math.inf
    for name, t in zip(("dq", "dk", "dv"), x):
        assert torch.allclose(r[name], t.grad, atol=1e-12), name


def test_reference_four_bits():
    """By distance to the eight steps, and the block's power of two by its definition."""
    g = torch.Generator().manual_seed(2)
    x = torch.randn((50, 3, 64), generator=g, dtype=torch.float64) * torch.exp(5 * torch.randn((50, 3, 1), generator=g, dtype=torch.float64))
    x[0, 0, :32] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.5] * 4)
    code, scale = four_bits(x)
    unit = torch.tensor([2.0 ** (int(s) - 127) for s in scale.flatten()], dtype=torch.float64).reshape(50, 3, 2)
    top = x.reshape(50, 3, 2, 32).abs().amax(-1)
    assert bool((top < 7 * unit).all()) and bool((top >= 3.5 * unit).all())
    got = values(packed(code), scale)
    assert bool(((got - x).abs() <= unit.repeat_interleave(32, -1)).all())
    assert got[0, 0, :8].tolist() == [0, 1, 1, 2, 2, 4, 4, 6]
    bad = x.clone()
    bad[1, 1, 40] = math.inf
    read = values(*(lambda c, s: (packed(c), s))(*four_bits(bad)))
    assert bool(torch.isnan(read[1, 1, 32:]).all()) and torch.equal(read[1, 1, :32], got[1, 1, :32])


@pytest.mark.parametrize("axes", [1, 2])
@pytest.mark.parametrize("neighbours", [False, True])
def test_reference_rotation_keeps_lengths_and_adds_up(axes, neighbours):
    g = torch.Generator().manual_seed(3)
    x = torch.randn((9, 2, 64), generator=g, dtype=torch.float64)
    angle = torch.rand((20, 32 // axes), generator=g, dtype=torch.float64)
    at = torch.randint(0, 20, (9, axes), generator=g)
    y = rotated(x, at, torch.cos(angle), torch.sin(angle), neighbours)
    assert torch.allclose(y.norm(dim=-1), x.norm(dim=-1))
    assert torch.allclose(rotated(y, at, torch.cos(angle), -torch.sin(angle), neighbours), x)
