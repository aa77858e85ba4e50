"""Host-side checks of the operators of generation that need no GPU: argument
checks return the documented codes before anything touches a device, workspace
sizes, the layouts of the structures in the binding, and trees of drafted tokens."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2306_10015_amd import mezo

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
L = mezo.lib

# device addresses that no call below may get as far as using
Q, K, V, O, KC, VC, T, P, F, S, W, E = (0x7F0000000000 + i * 0x100000000 for i in range(12))


def offsets(tmp_path, struct, names):
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "mezo.h"\nint main(void) {\n'
                   + "".join(f'  printf("%zu\\n", offsetof({struct}, {n}));\n' for n in names)
                   + f'  printf("%zu\\n", sizeof({struct}));\n  return 0;\n}}\n')
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    return [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]


APPEND = ["q", "k", "v", "q_out", "k_cache", "v_cache", "docs", "pages", "freqs", "positions", "tokens", "n_pages",
          "n_entries", "max_q", "q_token", "q_head", "k_token", "k_head", "v_token", "v_head", "o_token", "o_head",
          "kc_page", "kc_row", "kc_head", "vc_page", "vc_row", "vc_head", "n_docs", "heads", "kv_heads", "dim",
          "page_rows", "rot", "interleaved", "dtype"]
PAGES = ["list", "tree", "n_entries", "n_pages", "k_page", "v_page", "rows", "tree_words"]


def test_struct_layouts(tmp_path):
    want = [8 * i for i in range(28)] + [224 + 4 * i for i in range(8)]
    assert offsets(tmp_path, "mezo_append_t", APPEND) == want + [mezo._APPEND.size]
    assert offsets(tmp_path, "mezo_pages_t", PAGES) == [8 * i for i in range(6)] + [48, 52] + [mezo._PAGES.size]


def append(**kw):
    a = dict(q=Q, k=K, v=V, q_out=O, k_cache=KC, v_cache=VC, docs=T, pages=P, freqs=F, positions=S, tokens=10,
             n_pages=6, n_entries=5, max_q=10, q_token=256, q_head=64, k_token=128, k_head=64, v_token=128, v_head=64,
             o_token=256, o_head=64, kc_page=2048, kc_row=128, kc_head=64, vc_page=2048, vc_row=128, vc_head=64,
             n_docs=3, heads=4, kv_heads=2, dim=64, page_rows=16, rot=64, interleaved=0, dtype=mezo.BF16)
    a.update(kw)
    return L.mezo_cache_append(mezo._APPEND.pack(*(a[n] or 0 for n in APPEND)), None)


def test_append_refusals():
    for bad in (dict(k=0), dict(v=0), dict(docs=0), dict(k_cache=0), dict(v_cache=0), dict(pages=0), dict(q_out=0),
                dict(freqs=0), dict(heads=0), dict(kv_heads=0), dict(heads=65537), dict(kv_heads=65537), dict(dim=0),
                dict(dim=60), dict(dim=136), dict(rot=66), dict(rot=63), dict(page_rows=4), dict(page_rows=24),
                dict(page_rows=1 << 17), dict(page_rows=0), dict(q=Q + 8), dict(k=K + 2), dict(v=V + 8),
                dict(q_out=O + 8), dict(k_cache=KC + 8), dict(v_cache=VC + 4), dict(docs=T + 4), dict(pages=P + 2),
                dict(freqs=F + 2), dict(positions=S + 4), dict(q_token=260), dict(k_head=4), dict(v_token=1),
                dict(o_head=12), dict(kc_page=2044), dict(vc_row=129), dict(n_pages=1 << 32), dict(tokens=1 << 35),
                dict(n_docs=1 << 27, tokens=1 << 20, max_q=1 << 20), dict(n_entries=1 << 35),
                dict(kc_page=1 << 62), dict(k_token=1 << 62), dict(q_token=1 << 60)):
        assert append(**bad) == mezo.EINVAL, bad
    assert append(dtype=mezo.NF4) == mezo.EDTYPE
    assert append(dtype=7) == mezo.EDTYPE
    assert L.mezo_cache_append(None, None) == mezo.EINVAL


def test_append_overlaps():
    for bad in (dict(k_cache=K), dict(v_cache=K + 128), dict(k_cache=VC), dict(k_cache=VC + 16), dict(q_out=K), dict(q_out=Q + 128),
                dict(q_out=Q, o_token=264), dict(q_out=KC), dict(q_out=T), dict(k_cache=P - 4096), dict(v_cache=F),
                dict(q_out=S), dict(kc_row=64), dict(kc_page=1024), dict(vc_head=32), dict(o_head=8),
                # parts of one array that meet: a token's keys end in its values
                dict(q_out=Q + 2 * 64, q=Q, k=Q + 2 * 256, o_token=256)):
        assert append(**bad) == mezo.EOVERLAP, bad


def test_append_of_nothing():
    for none in (dict(n_docs=0), dict(max_q=0), dict(tokens=0), dict(tokens=0, q=0, k=0, v=0, docs=0)):
        assert append(**none) == mezo.OK
    assert append(n_docs=0, dim=60) == mezo.EINVAL


def attend(work=0, size=0, **kw):
    a = dict(q=Q, k=KC, v=VC, out=O, lse=E, docs=T, slopes=0, q_tokens=10, k_tokens=0, q_token=256, q_head=64,
             k_token=128, k_head=64, v_token=128, v_head=64, o_token=256, o_head=64, max_q=10, max_k=80, n_docs=3,
             heads=4, kv_heads=2, dim=64, dtype=mezo.BF16, causal=1, scale=0.1, softcap=0.0)
    c = dict(list=P, tree=0, n_entries=5, n_pages=6, k_page=2048, v_page=2048, rows=16, tree_words=0)
    for n, x in kw.items():
        (c if n in c else a)[n] = x
    pa, pc = mezo._ATTENTION.pack(*a.values()), mezo._PAGES.pack(*c.values())
    if size is None:
        return L.mezo_paged_attention_workspace(pa, pc)
    return L.mezo_paged_attention(pa, pc, work or None, size, None)


def test_attention_refusals():
    for bad in (dict(q=0), dict(k=0), dict(v=0), dict(out=0), dict(docs=0), dict(list=0), dict(heads=0),
                dict(kv_heads=0), dict(kv_heads=3), dict(heads=65540), dict(dim=0), dict(dim=60), dict(dim=136),
                dict(rows=4), dict(rows=48), dict(rows=1 << 17), dict(q=Q + 8), dict(k=KC + 8), dict(v=VC + 2),
                dict(out=O + 8), dict(lse=E + 2), dict(docs=T + 4), dict(list=P + 2), dict(tree=F + 4, tree_words=1),
                dict(tree=F), dict(tree=F, tree_words=1025), dict(tree=F, tree_words=1, slopes=S),
                dict(tree=F, tree_words=1, causal=0), dict(q_token=260), dict(k_page=2044), dict(v_page=1),
                dict(k_token=1 << 25), dict(v_token=1 << 63), dict(k_page=1 << 62), dict(k_page=1 << 31),
                dict(v_page=1 << 31), dict(k_token=1 << 24, rows=256), dict(n_pages=1 << 32),
                dict(n_entries=1 << 35), dict(n_docs=1 << 23), dict(max_k=1 << 31, n_entries=1 << 30)):
        assert attend(**bad) == mezo.EINVAL, bad
    assert attend(dtype=mezo.NF4) == mezo.EDTYPE
    for bad in (dict(scale=float("inf")), dict(softcap=-1.0), dict(softcap=float("nan"))):
        assert attend(**bad) == mezo.ERANGE, bad
    for bad in (dict(out=Q), dict(out=KC), dict(out=T), dict(out=P), dict(lse=O), dict(lse=VC + 64), dict(o_head=8),
                dict(tree=O, tree_words=1), dict(tree=E, tree_words=2), dict(lse=P)):
        assert attend(**bad) == mezo.EOVERLAP, bad
    for none in (dict(n_docs=0), dict(max_q=0), dict(q_tokens=0)):
        assert attend(**none) == mezo.OK


def test_attention_workspace():
    big = dict(n_docs=1, max_q=1, max_k=16384, n_entries=1024)
    need = attend(size=None, **big)
    # as for contiguous keys of as many rows
    a = mezo._ATTENTION.pack(Q, K, V, O, 0, T, 0, 10, 16384, 256, 64, 128, 64, 128, 64, 256, 64, 1, 16384, 1, 4, 2, 64,
                             mezo.BF16, 1, 0.1, 0.0)
    assert need > 0 and need == L.mezo_attention_workspace(a)
    assert attend(**big) == mezo.EINVAL
    assert attend(work=W, size=need - 1, **big) == mezo.EINVAL
    assert attend(work=W + 8, size=need, **big) == mezo.EINVAL
    assert attend(work=O, size=need, **big) == mezo.EOVERLAP
    assert attend(size=None) == 0  # short documents need none
    assert attend(size=None, max_k=1 << 20, n_docs=1, max_q=1) == 0  # (80 rows in the list)
    assert attend(size=None, rows=12, **big) == 0
    assert L.mezo_paged_attention_workspace(None, None) == 0


def test_trees():
    mask, depth = mezo.tree_mask([[-1, 0, 0, 1, -1], [], [-1]], device="cpu")
    assert mask.tolist() == [[1], [3], [5], [11], [16], [1]] and depth.tolist() == [0, 1, 1, 2, 0, 0]
    mask, depth = mezo.tree_mask([list(range(-1, 65))], device="cpu")
    assert mask.shape == (66, 2) and mask[63].tolist() == [-1, 0] and mask[65].tolist() == [-1, 3]
    assert depth.tolist() == list(range(66))
    for bad in ([[0]], [[-2]], [[-1, 1]], [[-1, 2]]):
        with pytest.raises(ValueError):
            mezo.tree_mask(bad, device="cpu")
    assert mezo.tree_mask([], device="cpu")[0].shape == (0, 1)


def test_cache_refuses_what_it_cannot_hold():
    k = torch.zeros(4, 16, 2, 64)
    pages = torch.zeros(2, 2, dtype=torch.int32)
    with pytest.raises(ValueError):  # not on a device
        mezo.PagedCache(k, k, pages)


def test_error_of_a_missing_handle_is_a_code():
    assert L.mezo_paged_attention(None, None, None, 0, None) == mezo.EINVAL
    assert ctypes.sizeof(ctypes.c_void_p) == 8


# ---- products with 4-bit weights -----------------------------------------------------

def linear(x=Q, x_dtype=mezo.BF16, ldx=256, codes=K, absmax=V, m=4, n=8, k=256, c=O, c_dtype=mezo.F32, ldc=8, work=W,
           size=None):
    if size is None:
        size = L.mezo_nf4_linear_workspace(m, n, k, x_dtype, c_dtype)
    return L.mezo_nf4_linear(x, x_dtype, ldx, codes, absmax, m, n, k, c, c_dtype, ldc, work, size, None)


def test_linear_refusals():
    for bad in (dict(x=None), dict(codes=None), dict(absmax=None), dict(c=None), dict(m=0), dict(n=0), dict(k=0),
                dict(ldx=255), dict(ldc=7), dict(x=Q + 1), dict(x_dtype=mezo.F32, x=Q + 2), dict(c=O + 2),
                dict(codes=K + 8), dict(absmax=V + 4), dict(k=(1 << 23) + 1, ldx=1 << 24), dict(m=(1 << 30) + 1),
                dict(n=(1 << 30) + 1, ldc=1 << 31), dict(n=1 << 20, k=1 << 20, ldx=1 << 20, ldc=1 << 20),
                dict(m=1 << 20, n=1 << 20, ldc=1 << 20), dict(ldx=1 << 63), dict(ldc=1 << 62), dict(x=2 ** 64 - 64),
                dict(c=2 ** 64 - 32)):
        assert linear(**bad) == mezo.EINVAL, bad
    assert linear(x_dtype=mezo.NF4) == mezo.EDTYPE
    assert linear(c_dtype=5) == mezo.EDTYPE
    for bad in (dict(c=Q), dict(c=K + 128), dict(c=V), dict(c=Q + 4 * 256 * 2 - 4)):
        assert linear(**bad) == mezo.EOVERLAP, bad


def test_linear_workspace():
    big = dict(m=500, n=1000, k=1000, ldx=1000, ldc=1000)
    need = L.mezo_nf4_linear_workspace(500, 1000, 1000, mezo.BF16, mezo.F32)
    assert need > 0
    assert linear(**big, work=None) == mezo.EINVAL
    assert linear(**big, size=need - 1) == mezo.EINVAL
    assert linear(**big, work=W + 8) == mezo.EINVAL
    for other in (Q, K, V, O):
        assert linear(**big, work=other) == mezo.EOVERLAP
    for bad in ((0, 1, 1, 0, 0), (1, 0, 1, 0, 0), (1, 1, 0, 0, 0), (1, 1, 1, 2, 0), (1, 1, 1, 0, 9), (1 << 31, 1, 1, 0, 0)):
        assert L.mezo_nf4_linear_workspace(*bad) == 0
    # a matrix of any size is expanded a slab at a time
    assert L.mezo_nf4_linear_workspace(100, 50272, 16384, mezo.BF16, mezo.BF16) < 300 << 20


def test_linear_of_more_rows_than_a_grid():
    """Rows are laid out in whole blocks of 64 columns: what fits in MAX_NUMEL so, and no more."""
    size = L.mezo_nf4_linear_workspace
    for m, n, k in ((1 << 30, 1, 16), ((1 << 28) + 1, 1, 1), (1, 1 << 30, 16), (4, (1 << 28) + 1, 64)):
        assert size(m, n, k, mezo.BF16, mezo.BF16) == 0
        assert linear(m=m, n=n, k=k, ldx=k, ldc=n, size=1 << 40) == mezo.EINVAL
    for m, n, k in ((1 << 28, 1, 1), (1 << 28, 64, 64), (255, (1 << 26) - 1, 63)):
        assert size(m, n, k, mezo.F32, mezo.BF16) > 0
