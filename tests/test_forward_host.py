"""Host-side checks of the forward pass's operators that need no GPU: argument
checks return the documented codes before anything touches a device, workspace
sizes, and the layout of mezo_attention_t in the binding."""
import os
import subprocess

import numpy as np
import pytest

import f8_ref
from paper_2306_10015_amd import build, mezo

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
L = mezo.lib

# device addresses that no call below may get as far as using
A, B, C, D, E, W = (0x7F0000000000 + i * 0x100000000 for i in range(6))


def test_forward_kernels_do_not_spill():
    path = build.BUILD_DIR / "forward_resources.txt"
    if not path.exists():
        pytest.skip("no in-tree build record (run python -m paper_2306_10015_amd.build)")
    rows = [line.split() for line in path.read_text().splitlines() if line.strip()]
    assert {r[0] for r in rows} == set(build.FORWARD_UNITS)
    assert all(dict(kv.split("=") for kv in r[2:])["scratch"] == "0" for r in rows)


def test_attention_struct_layout(tmp_path):
    """The binding packs mezo_attention_t as the C compiler lays it out."""
    names = ["q", "k", "v", "out", "lse", "docs", "slopes", "q_tokens", "k_tokens", "q_token", "q_head", "k_token",
             "k_head", "v_token", "v_head", "o_token", "o_head", "max_q", "max_k", "n_docs", "heads", "kv_heads",
             "dim", "dtype", "causal", "scale", "softcap"]
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "mezo.h"\nint main(void) {\n'
                   + "".join(f'  printf("%zu\\n", offsetof(mezo_attention_t, {n}));\n' for n in names)
                   + '  printf("%zu\\n", sizeof(mezo_attention_t));\n  return 0;\n}\n')
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    want = [8 * i for i in range(19)] + [152 + 4 * i for i in range(8)]
    assert got == want + [mezo._ATTENTION.size]


# ---- 8-bit storage ----------------------------------------------------------------

def quantize(src=A, dtype=mezo.F32, rows=4, cols=256, ld=256, codes=B, scales=C):
    return L.mezo_f8_quantize(src, dtype, rows, cols, ld, codes, scales, None)


def test_quantize_refusals():
    for bad in (dict(src=None), dict(codes=None), dict(scales=None), dict(rows=0), dict(cols=0), dict(ld=255),
                dict(src=A + 2), dict(codes=B + 8), dict(scales=C + 2), dict(cols=(1 << 23) + 1),
                dict(rows=(1 << 30) + 1), dict(rows=1 << 30, cols=1 << 20, ld=1 << 20), dict(ld=1 << 63)):
        assert quantize(**bad) == mezo.EINVAL, bad
    assert quantize(dtype=mezo.NF4) == mezo.EDTYPE
    assert quantize(dtype=9) == mezo.EDTYPE
    assert quantize(codes=A + 16) == mezo.EOVERLAP
    assert quantize(scales=A + 4 * 256 * 4 - 4) == mezo.EOVERLAP
    assert quantize(scales=B + 1020) == mezo.EOVERLAP


def matmul(x=A, xs=B, w=C, ws=D, m=4, n=8, k=256, c=E, dtype=mezo.F32, ldc=8, work=None, size=0):
    return L.mezo_f8_matmul(x, xs, w, ws, m, n, k, c, dtype, ldc, work, size, None)


def test_matmul_refusals():
    for bad in (dict(x=None), dict(xs=None), dict(w=None), dict(ws=None), dict(c=None), dict(m=0), dict(n=0),
                dict(k=0), dict(ldc=7), dict(x=A + 8), dict(w=C + 4), dict(xs=B + 1), dict(ws=D + 2), dict(c=E + 2),
                dict(m=1 << 25, n=1 << 25, k=128, ldc=1 << 25)):
        assert matmul(**bad) == mezo.EINVAL, bad
    assert matmul(dtype=mezo.NF4) == mezo.EDTYPE
    assert matmul(c=C + 128) == mezo.EOVERLAP
    assert matmul(c=B) == mezo.EOVERLAP
    # a product whose k is split needs its workspace
    need = L.mezo_f8_matmul_workspace(4, 64, 1 << 15, mezo.F32)
    assert need > 0 and need % (4 * 64 * 4) == 0
    big = dict(m=4, n=64, k=1 << 15, ldc=64)
    assert matmul(**big) == mezo.EINVAL
    assert matmul(**big, work=W, size=need - 1) == mezo.EINVAL
    assert matmul(**big, work=W + 8, size=need) == mezo.EINVAL
    assert matmul(**big, work=E, size=need) == mezo.EOVERLAP
    assert L.mezo_f8_matmul_workspace(0, 64, 128, mezo.F32) == 0
    assert L.mezo_f8_matmul_workspace(4, 64, 128, 7) == 0


def linear(x=A, x_dtype=mezo.BF16, ldx=256, w=C, ws=D, m=4, n=8, k=256, c=E, dtype=mezo.F32, ldc=8, work=W, size=None):
    size = L.mezo_f8_linear_workspace(m, n, k, dtype) if size is None else size
    return L.mezo_f8_linear(x, x_dtype, ldx, w, ws, m, n, k, c, dtype, ldc, work, size, None)


def test_linear_refusals():
    assert L.mezo_f8_linear_workspace(4, 8, 256, mezo.F32) >= 4 * 256 + 4 * 4
    for bad in (dict(x=None), dict(w=None), dict(ws=None), dict(c=None), dict(work=None), dict(work=W + 4),
                dict(size=1000), dict(m=0), dict(k=0), dict(n=0), dict(ldx=255), dict(ldc=7), dict(x=A + 1)):
        assert linear(**bad) == mezo.EINVAL, bad
    assert linear(x_dtype=mezo.NF4) == mezo.EDTYPE
    assert linear(dtype=5) == mezo.EDTYPE
    assert linear(c=A) == mezo.EOVERLAP
    assert linear(work=A) == mezo.EOVERLAP
    assert linear(work=C) == mezo.EOVERLAP
    assert linear(c=D) == mezo.EOVERLAP


# ---- attention ----------------------------------------------------------------------

BASE = dict(q=A, k=B, v=C, out=D, lse=E, docs=W, slopes=0, q_tokens=10, k_tokens=20, q_token=128, q_head=64,
            k_token=64, k_head=64, v_token=64, v_head=64, o_token=128, o_head=64, max_q=10, max_k=20, n_docs=1,
            heads=2, kv_heads=1, dim=64, dtype=mezo.F32, causal=1, scale=0.125, softcap=0.0)


def attend(work=None, size=0, **kw):
    return L.mezo_attention(mezo._ATTENTION.pack(*{**BASE, **kw}.values()), work, size, None)


def workspace(**kw):
    return L.mezo_attention_workspace(mezo._ATTENTION.pack(*{**BASE, **kw}.values()))


def test_attention_refusals():
    assert L.mezo_attention(None, None, 0, None) == mezo.EINVAL
    for bad in (dict(q=0), dict(k=0), dict(v=0), dict(out=0), dict(docs=0), dict(heads=0), dict(kv_heads=0),
                dict(heads=3, kv_heads=2), dict(dim=0), dict(dim=4), dict(dim=60), dict(dim=136), dict(q=A + 8),
                dict(k=B + 4), dict(v=C + 8), dict(out=D + 8), dict(lse=E + 2), dict(docs=W + 4), dict(slopes=A + 1),
                dict(q_token=130), dict(k_head=2), dict(o_token=126), dict(heads=70000),
                dict(q_token=1 << 62), dict(k_token=1 << 25), dict(q_tokens=1 << 35),
                dict(max_q=1 << 24, q_tokens=1 << 24), dict(k_tokens=1 << 32, max_k=1 << 32)):
        assert attend(**bad) == mezo.EINVAL, bad
    assert attend(dtype=mezo.NF4) == mezo.EDTYPE
    inf, nan = float("inf"), float("nan")
    for bad in (dict(scale=inf), dict(scale=nan), dict(softcap=-1.0), dict(softcap=inf), dict(softcap=nan)):
        assert attend(**bad) == mezo.ERANGE, bad
    for bad in (dict(out=A), dict(out=B + 256), dict(lse=D), dict(out=W), dict(o_head=0), dict(o_token=64),
                dict(o_token=0, o_head=64), dict(slopes=D + 64), dict(lse=A + 64)):
        assert attend(**bad) == mezo.EOVERLAP, bad
    # nothing to do
    for empty in (dict(n_docs=0), dict(max_q=0), dict(q_tokens=0)):
        assert attend(**empty) == mezo.OK


def test_attention_workspace():
    assert workspace() == 0
    long = dict(q_tokens=1, max_q=1, k_tokens=1 << 20, max_k=1 << 20)
    need = workspace(**long)
    assert need > 0
    splits = -(-need // (2 * (8 + 64 * 4)))
    assert 2 <= splits <= 64
    assert attend(**long) == mezo.EINVAL
    assert attend(**long, work=0x7E0000000000, size=need - 1) == mezo.EINVAL
    assert attend(**long, work=D, size=need) == mezo.EOVERLAP
    assert workspace(dim=60) == 0 and workspace(heads=0) == 0 and L.mezo_attention_workspace(None) == 0


# ---- the token loss -------------------------------------------------------------------

def loss(logits=A, dtype=mezo.F32, rows=4, vocab=100, ld=100, targets=B, losses=C, mean=D, work=None, size=0):
    return L.mezo_token_loss(logits, dtype, rows, vocab, ld, targets, losses, mean, work, size, None)


def test_token_loss_refusals():
    for bad in (dict(logits=None), dict(targets=None), dict(losses=None), dict(rows=0), dict(vocab=0), dict(ld=99),
                dict(logits=A + 2), dict(targets=B + 4), dict(losses=C + 2), dict(mean=D + 1),
                dict(rows=(1 << 23) + 1), dict(ld=1 << 62)):
        assert loss(**bad) == mezo.EINVAL, bad
    assert loss(dtype=mezo.NF4) == mezo.EDTYPE
    for bad in (dict(losses=A + 400), dict(losses=B + 8), dict(mean=C + 4), dict(mean=A)):
        assert loss(**bad) == mezo.EOVERLAP, bad
    need = L.mezo_token_loss_workspace(8, 50272)
    assert need > 0
    assert loss(rows=8, vocab=50272, ld=50272) == mezo.EINVAL
    assert loss(rows=8, vocab=50272, ld=50272, work=A, size=need) == mezo.EOVERLAP
    assert L.mezo_token_loss_workspace(0, 10) == 0 and L.mezo_token_loss_workspace(1, 50272) == 0


# ---- the reference of 8-bit storage (what the GPU tests compare with) ---------------

def test_reference_of_e4m3():
    """The published format: 448 the largest, 2^-9 the smallest, 126 positive values."""
    v = f8_ref.VALUES
    assert v[0x7E] == 448.0 and v[1] == 2.0 ** -9 and v[0x38] == 1.0 and np.isnan(v[0x7F]) and np.isnan(v[0xFF])
    assert np.all(np.diff(v[:127]) > 0) and np.array_equal(v[128:255], -v[:127])
    import torch
    assert np.array_equal(torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy(), v, True)


def test_reference_quantizer():
    """Values of the format are kept, everything else goes to the nearest one."""
    rng = np.random.Generator(np.random.PCG64(5))
    w = rng.normal(0, 1, (3, 300)).astype(np.float32)
    codes, scales = f8_ref.quantize(w)
    back = f8_ref.dequantize(codes, scales, 300)
    again, s2 = f8_ref.quantize(back.astype(np.float32))
    assert np.array_equal(again, codes) and np.array_equal(s2, scales)
    e = scales[:, :3].astype(int) - 127
    for r in range(3):
        for b in range(3):
            part = w[r, 128 * b:128 * b + 128].astype(np.float64)
            top = np.abs(part).max()
            assert top <= 448 * 2.0 ** e[r, b] and top > 448 * 2.0 ** (e[r, b] - 1)
            grid = np.concatenate([-f8_ref.VALUES[:127], f8_ref.VALUES[:127]]) * 2.0 ** e[r, b]
            near = np.abs(part[:, None] - grid[None]).min(axis=1)
            assert np.array_equal(np.abs(part - back[r, 128 * b:128 * b + 128]), near)
