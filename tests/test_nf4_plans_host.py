"""How a product with 4-bit weights is cut into workgroups (csrc/nf4_linear_launch.hpp),
on the host: the kernel that each product of the tile tests runs on, and what every
cut has to hold to."""
import os
import shutil
import subprocess

import pytest

from nf4_tiles import PRODUCTS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r'''
#include <cstdio>
#include "nf4_linear_launch.hpp"
int main()
{
    unsigned long long m, n, k;
    int wide;
    const char* const names[] = {"thin", "64x64", "128x128", "256x256"};
    while (std::scanf("%llu %llu %llu %d", &m, &n, &k, &wide) == 4) {
        const mezo::NF4Cut c = mezo::cut_nf4(m, n, k, wide);
        if (c.tile != mezo::kThin)
            std::printf("%s %u %llu\n", names[c.tile], c.splits, (unsigned long long)c.slab);
        else if (c.thin_rows)
            std::printf("%u rows %u %llu\n", c.thin_rows, c.splits, (unsigned long long)c.slab);
        else
            std::printf("ragged %u %llu\n", c.splits, (unsigned long long)c.slab);
    }
    // every split of k has work; slabs are whole tiles but for the last; the workspace's parts
    // begin on 16 bytes and hold what is put there
    unsigned long long bad = 0;
    for (m = 1; m < 20000; m = m * 5 / 4 + 1)
        for (n = 1; n < 200000; n = n * 4 / 3 + 1)
            for (k = 1; k < 70000; k = k * 3 / 2 + 1)
                for (int i = 0; i < 4; ++i) {
                    wide = i & 1;
                    const unsigned long long kk = i & 2 ? (k + 63) / 64 * 64 : k;
                    const mezo::NF4Cut c = mezo::cut_nf4(m, n, kk, wide);
                    const mezo::NF4Space s = mezo::nf4_space(m, n, kk, wide);
                    const unsigned long long stages = mezo::nf4_columns(kk) / 64 * (wide && c.tile != mezo::kThin ? 6 : 1);
                    if (c.splits < 1 || c.splits > 16 || (c.splits > 1 && 8 * c.splits > stages)) ++bad;
                    if ((c.tile == mezo::kThin) != (c.slab == 0)) ++bad;
                    if (c.slab > n || (c.slab < n && c.slab % 256)) ++bad;
                    if (c.tile == mezo::kThin && (c.thin_rows == 0) != (kk % 64 != 0)) ++bad;
                    if (s.weights % 16 || s.partial % 16 || s.weights > s.partial || s.partial > s.bytes) ++bad;
                    if (c.splits > 1 && s.bytes - s.partial < 4 * c.splits * m * (c.slab ? c.slab : n)) ++bad;
                }
    std::printf("bad %llu\n", bad);
}
'''


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_cuts(tmp_path):
    src, exe = tmp_path / "cuts.cpp", tmp_path / "cuts"
    src.write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-D__HIP_PLATFORM_AMD__", "-isystem", "/opt/rocm/include",
                    "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2306_10015_amd", "csrc"),
                    str(src), "-o", str(exe)], check=True)
    asked = "".join(f"{m} {n} {k} {int(x == 'f32')}\n" for m, n, k, x, *_ in PRODUCTS)
    lines = subprocess.run([str(exe)], input=asked, capture_output=True, text=True, check=True).stdout.splitlines()
    assert lines[:-1] == [f"{kernel} {splits} {slab}" for _, _, _, _, kernel, splits, slab, _ in PRODUCTS]
    assert lines[-1] == "bad 0"


def test_every_kernel_is_run():
    """The tiles with k whole and split, rows of c on the alignment of four columns and off it,
    and several slabs of either type; every kernel of few activations, k whole and, where it can
    be, split (128 rows of bf16 are taken where they give every CU work)."""
    run = [(x, kernel, splits > 1, n % 4 == 0 and not wide, 0 < slab < n) for _, n, _, x, kernel, splits, slab, wide in PRODUCTS]
    for x in ("f32", "bf16"):
        for tile in ("64x64", "128x128", "256x256"):
            for split in (False, True):
                assert {aligned for *key, aligned, _ in run if key == [x, tile, split]} >= {False, True}, (x, tile, split)
        assert any(r[0] == x and r[4] for r in run)
        for kernel in ("16 rows", "64 rows", "128 rows", "ragged"):
            splits = {False} if (x, kernel) == ("bf16", "128 rows") else {False, True}
            assert {split for *key, split, _, _ in run if key == [x, kernel]} == splits, (x, kernel)
