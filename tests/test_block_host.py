"""Host-only checks of rotary positions and the residual stream: structures, refusals with the documented status before any device work,
and the 64-bit forms that the GPU tests compare with, against torch's autograd and differences."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest
import torch

from tests.block_util import pair_channels, residual, rotary

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "speed3r.h")
P = 0x10000     # an aligned address that is never dereferenced
INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3


@pytest.fixture(scope="module")
def s3r():
    from paper_2603_08055_amd import speed3r
    if not os.path.exists(speed3r.LIB_PATH):
        from paper_2603_08055_amd import build
        build.build_library()
    speed3r.load()
    return speed3r


@pytest.mark.parametrize("name", ["s3r_rotary_params", "s3r_residual_params"])
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
                   + "".join(f'  printf("%zu\\n", offsetof({name}, {f}));\n' for f in fields)
                   + '  printf("%d %d %d %d %d %d\\n", S3R_NORM_NONE, S3R_NORM_RMS, S3R_NORM_LAYER, S3R_PAIRS_HALVES, S3R_PAIRS_NEIGHBOURS, '
                     "S3R_PAIRS_WHOLE);\n  return 0; }\n")
    exe = str(tmp_path / "layout")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), str(src), "-o", exe], check=True,
                   capture_output=True, text=True)
    got = [int(x) for x in subprocess.run([exe], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [ctypes.sizeof(cls)] + [getattr(cls, f).offset for f in fields] + [
        s3r.S3R_NORM_NONE, s3r.S3R_NORM_RMS, s3r.S3R_NORM_LAYER, s3r.S3R_PAIRS_HALVES, s3r.S3R_PAIRS_NEIGHBOURS, s3r.S3R_PAIRS_WHOLE]


def fill(p, names):
    for i, name in enumerate(names):
        setattr(p, name, P * (i + 1))
    return p


def rotary_params(s3r, **change):
    p = fill(s3r.s3r_rotary_params(), ("q", "k", "q_out", "k_out", "d_q_out", "d_k_out", "dq", "dk", "q_weight", "q_bias", "k_weight", "k_bias",
                                       "dq_weight", "dq_bias", "dk_weight", "dk_bias", "cos", "sin", "positions"))
    p.n_rows, p.n_positions, p.heads, p.kv_heads, p.head_dim, p.dtype, p.weight_dtype = 10, 100, 4, 2, 64, s3r.S3R_BF16, s3r.S3R_F32
    p.axes, p.axis_pairs[0], p.axis_pairs[1], p.norm, p.eps = 2, 16, 16, s3r.S3R_NORM_LAYER, 1e-6
    p.workspace, p.workspace_bytes = 0x900000, 1 << 30
    for f, x in change.items():
        if f == "axis_pairs":
            for i, n in enumerate(x):
                p.axis_pairs[i] = n
        else:
            setattr(p, f, x)
    return p


@pytest.mark.parametrize("change,status,word", [
    (dict(head_dim=128), UNSUPPORTED, "head_dim"), (dict(dtype=2), UNSUPPORTED, "dtype"), (dict(weight_dtype=-1), UNSUPPORTED, "weight_dtype"),
    (dict(heads=-1), INVALID, "heads"), (dict(heads=0, kv_heads=0), INVALID, "both 0"), (dict(heads=65536), UNSUPPORTED, "heads"),
    (dict(n_rows=-1), INVALID, "n_rows"), (dict(n_rows=1 << 27), UNSUPPORTED, "2^28"), (dict(norm=3), INVALID, "norm"),
    (dict(axes=4), INVALID, "axes"), (dict(axes=-1), INVALID, "axes"), (dict(axes=0), INVALID, "together"), (dict(cos=None), INVALID, "together"),
    (dict(sin=None), INVALID, "together"), (dict(axis_pairs=(0, 16)), INVALID, "axis_pairs"), (dict(axis_pairs=(33, 16)), INVALID, "axis_pairs"),
    (dict(axis_pairs=(16, 17)), INVALID, "32 pairs"), (dict(axis_pairs=(16, -1)), INVALID, "axis_pairs"), (dict(pairs=3), INVALID, "pairs"),
    (dict(eps=0.0), INVALID, "eps"), (dict(eps=-1.0), INVALID, "eps"), (dict(eps=float("nan")), INVALID, "eps"), (dict(eps=float("inf")), INVALID, "eps"),
    (dict(eps=1e-42), INVALID, "eps"), (dict(norm=0), INVALID, "norm"), (dict(axes=0, cos=None, sin=None, norm=0), INVALID, "nothing to do"),
    (dict(axes=0, cos=None, sin=None), INVALID, "positions"), (dict(n_positions=0), INVALID, "n_positions"), (dict(positions=None), INVALID, "positions"),
    (dict(q=P + 8), INVALID, "aligned"), (dict(cos=P + 4), INVALID, "aligned"), (dict(positions=P + 2), INVALID, "aligned"),
    (dict(q_weight=P + 4), INVALID, "aligned"), (dict(q_stride_tok=12), INVALID, "stride"), (dict(k_stride_head=-8), INVALID, "stride"),
    (dict(dq_stride_tok=4), INVALID, "stride"), (dict(dk_stride_head=4), INVALID, "stride"),
])
def test_rotary_refusals(s3r, change, status, word):
    p = rotary_params(s3r, **change)
    for fn in (s3r.load().speed3r_rotary, s3r.load().speed3r_rotary_backward):
        assert fn(ctypes.byref(p)) == status and word in s3r.speed3r_last_error()


@pytest.mark.parametrize("fn,change,status,word", [
    ("", dict(q=None), INVALID, "null"), ("", dict(k_out=None), INVALID, "null"), ("", dict(q_out=P), INVALID, "alias"), ("", dict(k_out=P), INVALID, "alias"),
    ("", dict(k_out=3 * P), INVALID, "alias"), ("_backward", dict(q=None), INVALID, "null"), ("_backward", dict(dk=None), INVALID, "null"),
    ("_backward", dict(d_q_out=None), INVALID, "null"), ("_backward", dict(dq=5 * P), INVALID, "alias"), ("_backward", dict(dk=P), INVALID, "alias"),
    ("_backward", dict(dk=7 * P), INVALID, "alias"), ("_backward", dict(workspace=None), WORKSPACE, "workspace"),
    ("_backward", dict(workspace_bytes=100), WORKSPACE, "workspace"), ("_backward", dict(workspace=P + 16), INVALID, "256"),
])
def test_rotary_refusals_of_one_call(s3r, fn, change, status, word):
    p = rotary_params(s3r, **change)
    assert getattr(s3r.load(), "speed3r_rotary" + fn)(ctypes.byref(p)) == status and word in s3r.speed3r_last_error()


def residual_params(s3r, **change):
    p = fill(s3r.s3r_residual_params(), ("x", "f", "r", "y", "weight", "bias", "post_weight", "post_bias", "scale", "gate", "row_start", "d_r", "d_y", "dx",
                                         "df", "d_weight", "d_bias", "d_post_weight", "d_post_bias", "d_scale", "d_gate"))
    p.n_rows, p.width, p.batch, p.x_dtype, p.dtype, p.weight_dtype = 10, 64, 3, s3r.S3R_F32, s3r.S3R_BF16, s3r.S3R_F32
    p.norm, p.post_norm, p.eps, p.residual_scale, p.workspace, p.workspace_bytes = s3r.S3R_NORM_LAYER, s3r.S3R_NORM_RMS, 1e-6, 1.0, 0x900000, 1 << 30
    for f, x in change.items():
        setattr(p, f, x)
    return p


@pytest.mark.parametrize("change,status,word", [
    (dict(width=0), UNSUPPORTED, "width"), (dict(width=12), UNSUPPORTED, "width"), (dict(width=8200), UNSUPPORTED, "width"), (dict(width=-8), UNSUPPORTED, "width"),
    (dict(n_rows=-1), INVALID, "n_rows"), (dict(n_rows=(1 << 28) + 1), UNSUPPORTED, "2^28"), (dict(dtype=2), UNSUPPORTED, "dtype"),
    (dict(x_dtype=1, dtype=0), UNSUPPORTED, "x_dtype"), (dict(weight_dtype=7), UNSUPPORTED, "weight_dtype"), (dict(batch=-1), INVALID, "batch"),
    (dict(batch=0), INVALID, "batch"), (dict(row_start=None), INVALID, "batch"), (dict(gate=None), INVALID, "gate"), (dict(batch=65537), UNSUPPORTED, "65536"),
    (dict(norm=-1), INVALID, "norm"), (dict(post_norm=3), INVALID, "post_norm"), (dict(eps=0.0), INVALID, "eps"), (dict(residual_scale=float("inf")), INVALID, "finite"),
    (dict(norm=0), INVALID, "norm"), (dict(post_norm=0), INVALID, "post_norm"), (dict(f=None), INVALID, "need f"), (dict(x=None), INVALID, "null"),
    (dict(gate=None, row_start=None, batch=1), INVALID, "gate"),
    (dict(x=P + 8), INVALID, "aligned"), (dict(weight=P + 4), INVALID, "aligned"), (dict(row_start=P + 2), INVALID, "aligned"),
    (dict(x_stride=12), INVALID, "stride"), (dict(gate_stride=-8), INVALID, "stride"),
])
def test_residual_refusals(s3r, change, status, word):
    p = residual_params(s3r, **change)
    for fn in (s3r.load().speed3r_residual_norm, s3r.load().speed3r_residual_norm_backward):
        assert fn(ctypes.byref(p)) == status and word in s3r.speed3r_last_error()


@pytest.mark.parametrize("fn,change,status,word", [
    ("", dict(r=None, y=None), INVALID, "both"), ("", dict(norm=0, weight=None, bias=None, d_weight=None, d_bias=None), INVALID, "norm"),
    ("", dict(y=P), INVALID, "alias"), ("", dict(r=2 * P), INVALID, "alias"), ("", dict(r=4 * P), INVALID, "alias"), ("", dict(r=P, x_stride=128), INVALID, "alias"),
    ("_backward", dict(dx=None), INVALID, "null"), ("_backward", dict(df=None), INVALID, "together"), ("_backward", dict(d_r=None, d_y=None), INVALID, "both"),
    ("_backward", dict(dx=P), INVALID, "alias"), ("_backward", dict(df=14 * P), INVALID, "alias"), ("_backward", dict(df=13 * P), INVALID, "alias"),
    ("_backward", dict(workspace=None), WORKSPACE, "workspace"), ("_backward", dict(workspace=P + 16), INVALID, "256"),
    ("_backward", dict(norm=0, weight=None, bias=None, d_weight=None, d_bias=None), INVALID, "norm"),
])
def test_residual_refusals_of_one_call(s3r, fn, change, status, word):
    p = residual_params(s3r, **change)
    assert getattr(s3r.load(), "speed3r_residual_norm" + fn)(ctypes.byref(p)) == status and word in s3r.speed3r_last_error()


def test_workspaces_and_null_parameters(s3r):
    lib, most = s3r.load(), 2 ** 64 - 1
    for fn in (lib.speed3r_rotary, lib.speed3r_rotary_backward, lib.speed3r_residual_norm, lib.speed3r_residual_norm_backward):
        assert fn(None) == INVALID and "null" in s3r.speed3r_last_error()
    assert lib.speed3r_rotary_workspace_bytes(None) == lib.speed3r_residual_workspace_bytes(None) == most
    assert lib.speed3r_rotary_workspace_bytes(ctypes.byref(rotary_params(s3r, head_dim=32))) == most
    assert lib.speed3r_residual_workspace_bytes(ctypes.byref(residual_params(s3r, width=4))) == most
    assert 0 < lib.speed3r_rotary_workspace_bytes(ctypes.byref(rotary_params(s3r))) < 1 << 24
    none = {w: None for w in ("dq_weight", "dq_bias", "dk_weight", "dk_bias")}
    assert lib.speed3r_rotary_workspace_bytes(ctypes.byref(rotary_params(s3r, **none))) == 0
    none = {w: None for w in ("d_weight", "d_bias", "d_post_weight", "d_post_bias", "d_scale", "d_gate")}
    assert lib.speed3r_residual_workspace_bytes(ctypes.byref(residual_params(s3r, **none))) == 0
    assert 0 < lib.speed3r_residual_workspace_bytes(ctypes.byref(residual_params(s3r, n_rows=1 << 28, width=8192))) < 1 << 30


def causal_params(s3r, **change):
    p = fill(s3r.s3r_cross_params(), ("q", "k", "v", "out", "lse", "d_out", "dq", "dk", "dv"))
    p.n_q, p.n_kv, p.batch, p.heads, p.kv_heads, p.head_dim, p.dtype = 10, 20, 1, 4, 2, 64, s3r.S3R_BF16
    for f, x in change.items():
        setattr(p, f, x)
    return p


@pytest.mark.parametrize("change,view,status,word", [
    (dict(), 0, INVALID, "tokens_per_view"), (dict(), -5, INVALID, "tokens_per_view"), (dict(head_dim=32), 1, UNSUPPORTED, "head_dim"),
    (dict(n_kv=-1), 1, INVALID, "n_kv"), (dict(n_kv=1 << 40), 7, UNSUPPORTED, "2^28"), (dict(heads=3), 1, INVALID, "multiple"),
    (dict(q_start=P), 1, INVALID, "together"), (dict(q=None), 1, INVALID, "null"), (dict(out=P), 1, INVALID, "alias"), (dict(k=P + 2), 1, INVALID, "aligned"),
])
def test_causal_refusals(s3r, change, view, status, word):
    lib, p = s3r.load(), causal_params(s3r, **change)
    for fn in (lib.speed3r_causal_attn, lib.speed3r_causal_attn_backward):
        assert fn(ctypes.byref(p), view) == status and word in s3r.speed3r_last_error()
        assert fn(None, 1) == INVALID and "null" in s3r.speed3r_last_error()
    assert lib.speed3r_causal_workspace_bytes(None, 1, 0) == 2 ** 64 - 1
    assert lib.speed3r_causal_workspace_bytes(ctypes.byref(causal_params(s3r)), 0, 0) == 2 ** 64 - 1
    p = causal_params(s3r)
    assert lib.speed3r_causal_attn_backward(ctypes.byref(p), 1) == WORKSPACE and "workspace" in s3r.speed3r_last_error()


def test_workspaces_by_the_binding(s3r):
    q = torch.empty((10000, 4, 64), dtype=torch.bfloat16, device="meta")
    assert s3r.speed3r_causal_workspace_bytes(q, q, backward=True) >= 10000 * 4 * 8
    with pytest.raises(s3r.Speed3rError, match="tokens_per_view"):
        s3r.speed3r_causal_workspace_bytes(q, q, tokens_per_view=0)
    assert s3r.speed3r_rotary_workspace_bytes(False) == 0 < s3r.speed3r_rotary_workspace_bytes()
    plain, gates = s3r.speed3r_residual_workspace_bytes(1000, 512), s3r.speed3r_residual_workspace_bytes(1000, 512, batch=7, gate_gradients=True)
    assert 0 < plain < gates and s3r.speed3r_residual_workspace_bytes(1000, 512, weight_gradients=False) == 0
    with pytest.raises(s3r.Speed3rError, match="width"):
        s3r.speed3r_residual_workspace_bytes(10, 12)


def test_a_view_longer_than_32_bits_hold(s3r):
    """It is held to what they do, and not cut down to another one."""
    q = torch.empty((10000, 4, 64), dtype=torch.bfloat16, device="meta")
    largest = s3r.speed3r_causal_workspace_bytes(q, q, tokens_per_view=2 ** 31 - 1, backward=True)
    assert largest != s3r.speed3r_causal_workspace_bytes(q, q, tokens_per_view=1, backward=True)
    for view in (2 ** 31, 2 ** 32 + 1, 2 ** 63 - 1):
        assert s3r.speed3r_causal_workspace_bytes(q, q, tokens_per_view=view, backward=True) == largest
    with pytest.raises(s3r.Speed3rError, match="tokens_per_view"):
        s3r.speed3r_causal_workspace_bytes(q, q, tokens_per_view=1 - 2 ** 32)


def test_the_binding_refuses(s3r):
    x = torch.zeros((4, 2, 64))
    with pytest.raises(TypeError, match="GPU"):
        s3r.speed3r_rotary(x, x, x, x)
    with pytest.raises(TypeError, match="GPU"):
        s3r.speed3r_residual_norm(torch.zeros((4, 64)))


# ---- the 64-bit forms ---------------------------------------------------------------------------------------

def norm_by_torch(x, kind, weight, bias, eps):
    if kind == "layer":
        return torch.nn.functional.layer_norm(x, x.shape[-1:], weight, bias, eps)
    if kind == "rms":
        x = torch.nn.functional.rms_norm(x, x.shape[-1:], weight, eps)
        return x if bias is None else x + bias
    return x


@pytest.mark.parametrize("pairs", ["halves", "neighbours", "whole"])
@pytest.mark.parametrize("axis_pairs", [(32,), (16, 16), (10, 11, 11), (3, 1, 5)])
def test_pairs_cover_each_channel_once(pairs, axis_pairs):
    got = pair_channels(axis_pairs, pairs)
    channels = [c for a, b, _ in got for c in (a, b)]
    assert sorted(channels) == list(range(2 * sum(axis_pairs))) and [x for _, _, x in got] == [a for a, p in enumerate(axis_pairs) for _ in range(p)]


@pytest.mark.parametrize("kind", [None, "rms", "layer"])
@pytest.mark.parametrize("pairs", ["halves", "neighbours", "whole"])
def test_rotary_reference(kind, pairs):
    g = torch.Generator().manual_seed(3)
    x, d_out = (torch.randn((5, 3, 64), generator=g, dtype=torch.float64) for _ in range(2))
    w, b = (torch.randn(64, generator=g, dtype=torch.float64) if kind else None for _ in range(2))
    axis_pairs, at = (10, 11, 5), torch.randint(0, 7, (5, 3), generator=g)
    angle = torch.randn((7, 26), generator=g, dtype=torch.float64)
    cos, sin = torch.cos(angle), torch.sin(angle)
    leaves = [t.clone().requires_grad_() for t in (x, w, b) if t is not None]
    n = norm_by_torch(leaves[0], kind, *(leaves[1:] if kind else (None, None)), 1e-3)
    turns = torch.eye(64, dtype=torch.float64).repeat(5, 1, 1)          # a rotation matrix for every row
    for j, (a, c, axis) in enumerate(pair_channels(axis_pairs, pairs)):
        turns[:, a, a] = turns[:, c, c] = cos[at[:, axis], j]
        turns[:, a, c], turns[:, c, a] = -sin[at[:, axis], j], sin[at[:, axis], j]
    y = torch.matmul(turns[:, None], n[..., None])[..., 0]
    r = rotary(x, w, b, cos, sin, at, axis_pairs, pairs, kind, 1e-3, d_out)
    grads = torch.autograd.grad(y, leaves, d_out)
    for name, want in zip(("out", "dx", "d_weight", "d_bias"), (y.detach(),) + grads):
        assert torch.allclose(r[name][0], want, rtol=1e-11, atol=1e-11), name


@pytest.mark.parametrize("kind,post,with_f,gates,dr,dy", [
    ("layer", None, True, False, True, True), ("rms", "layer", True, True, True, True), ("layer", "rms", True, True, False, True),
    (None, "rms", True, True, True, False), ("rms", None, False, False, True, True), ("layer", None, False, False, False, True),
])
def test_residual_reference(kind, post, with_f, gates, dr, dy):
    """Against autograd, and the gradients of x and f against differences."""
    g = torch.Generator().manual_seed(4)
    n, C = 6, 24
    normal = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)
    t = {"x": normal(n, C), "f": normal(n, C) if with_f else None, "weight": normal(C) if kind else None, "bias": normal(C) if kind else None,
         "post_weight": normal(C) if post else None, "post_bias": normal(C) if post else None, "scale": normal(C) if with_f else None,
         "gate": normal(3, C) if gates else None}
    seq = torch.tensor([0, 0, 0, 2, 2, 2])
    d_r, d_y = normal(n, C) if dr else None, normal(n, C) if dy else None

    def formula(t):
        r = t["x"]
        if with_f:
            u = 0.7 * t["scale"] * norm_by_torch(t["f"], post, t["post_weight"], t["post_bias"], 1e-3)
            r = r + (u * t["gate"][seq] if gates else u)
        return r, norm_by_torch(r, kind, t["weight"], t["bias"], 1e-3) if kind else None

    def loss(t):
        r, y = formula(t)
        return (0 if d_r is None else (r * d_r).sum()) + (0 if d_y is None else (y * d_y).sum())

    leaves = {k: v.clone().requires_grad_() for k, v in t.items() if v is not None}
    total = loss({**t, **leaves})
    grads = dict(zip(leaves, torch.autograd.grad(total, list(leaves.values()), allow_unused=True)))
    got = residual(t["x"], t["f"], kind, t["weight"], t["bias"], 1e-3, post, t["post_weight"], t["post_bias"], t["scale"], t["gate"], seq, 0.7, d_r, d_y)
    r, y = formula(t)
    assert torch.allclose(got["r"][0], r) and (y is None or torch.allclose(got["y"][0], y))
    names = {"x": "dx", "f": "df"}
    for k, want in grads.items():
        if want is not None:
            assert torch.allclose(got[names.get(k, "d_" + k)][0].reshape(want.shape), want, rtol=1e-10, atol=1e-10), k
    for k in ("x", "f") if with_f else ("x",):
        for at in ((0, 0), (5, 23), (3, 7)):
            step = torch.zeros_like(t["x"])
            step[at] = 1e-6
            slope = (loss({**t, k: t[k] + step}) - loss({**t, k: t[k] - step})) / 2e-6
            assert abs(float(slope - got[names[k]][0][at])) < 1e-7
